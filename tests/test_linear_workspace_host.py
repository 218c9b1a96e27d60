"""Sizes of the dense layer's workspace (CPU)."""
import pytest

from tests.test_abi_host import _lib

F32, BF16, F16 = 0, 1, 2
ELEMENT = {F32: 4, BF16: 2, F16: 2}


@pytest.mark.parametrize("dtype,d_in,d_out,rows,most", [
    (BF16, 4096, 4096, 1, 2 << 20), (BF16, 4096, 16384, 32, 12 << 20), (F32, 256, 256, 64, 1 << 20), (F32, 64, 64, 8, 1 << 18),
    (F16, 1000, 1000, 32, 4 << 20)])
def test_small_calls_take_little(dtype, d_in, d_out, rows, most):
    """A layer for a few rows holds partial sums, not copies of W."""
    assert _lib().mlp_linear_workspace_bytes(dtype, d_in, d_out, rows) <= most


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_room_of_the_operands(dtype):
    """What a call may write there fits: g (of 16-bit types two values of up to 64 rows, or of
    fewer than eight outputs), the layouts of X and W with rows of multiples of eight (twice
    for narrow 16-bit layers, up to 64 rows), and no more than 17 MiB and 256 chunks of
    column sums over it."""
    lib, e = _lib(), ELEMENT[dtype]

    def p8(n):
        return -(-n // 8) * 8

    for d_in in (1, 5, 8, 33, 1000, 4097, 1 << 20):
        for d_out in (1, 7, 8, 129, 4096, 10001):
            for rows in (1, 31, 32, 33, 64, 65, 700, 5000, 1 << 20):
                b = lib.mlp_linear_workspace_bytes(dtype, d_in, d_out, rows)
                low = 0 if e == 4 else rows if d_out < 8 else min(rows, 64)
                narrow = min(d_in, d_out) < 8
                need = e * (rows + low) * p8(d_out)
                if narrow or rows > 32:
                    two = e == 2 and narrow
                    need += e * (rows + (low if two and d_out >= 8 else 0)) * p8(d_in) + e * d_in * (2 if two else 1) * p8(d_out)
                assert need <= b <= need + (17 << 20) + 4 * 256 * max(d_out, 1024) + 4096, (d_in, d_out, rows, b - need)
