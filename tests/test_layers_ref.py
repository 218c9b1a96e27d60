"""Pins of the layer operators' 64-bit reference (tests/layers_ref.py): the generator
against published blocks, the gradients against differences."""
import numpy as np
import pytest
import torch

from tests import layers_ref as R


@pytest.mark.parametrize("word,key,want", [
    (0x00000000, 0x00000000, (0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8)),
    (0xffffffff, 0xffffffff, (0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd))])
def test_generator_known_answers(word, key, want):
    """The known answers published with the generator (philox4x32, 10 rounds)."""
    out = R.philox(np.full((1, 4), word, np.uint32), (key, key))[0]
    assert tuple(int(v) for v in out) == want


def test_mask_rate_and_layout():
    k = R.keep_mask(5, 1 << 33, 64, 1001, 0.25)
    assert k.shape == (64, 1001) and abs(k.mean() - 0.75) < 5 * (0.25 * 0.75 / k.size) ** 0.5
    # rows start at blocks of their own: one more column in the last block changes nothing
    assert np.array_equal(R.keep_mask(5, 9, 6, 19, 0.5), R.keep_mask(5, 9, 6, 24, 0.5)[:, :19])
    # the counter goes on from row to row, and wraps
    assert np.array_equal(R.keep_mask(5, 9, 6, 24, 0.5)[2:], R.keep_mask(5, 15, 4, 24, 0.5))
    assert np.array_equal(R.keep_mask(5, -3, 2, 24, 0.5)[1], R.keep_mask(5, 0, 1, 24, 0.5)[0])
    assert not R.keep_mask(5, 9, 6, 24, 1.0).any() and R.keep_mask(5, 9, 6, 24, 0.0).all()


@pytest.mark.parametrize("act", R.ACTS)
def test_gradients_against_differences(act):
    """d/dt sum(dY * y) by central differences of the forward map, p = 0.5."""
    g = torch.Generator().manual_seed(11)
    X, W, b, dY = (torch.randn(*s, generator=g, dtype=torch.float64) for s in ((5, 7), (7, 9), (9,), (5, 9)))
    rng = (123456789012345, 77)

    def loss(X, W, b):
        return float((dY * R.forward(X, W, b, None, act, 0.5, rng, "f32")[0]).sum())

    z = X @ W + b
    ref, _ = R.backward(X, W, z, dY, act, 0.5, rng, "f32")
    assert float(z.abs().min()) > 1e-4   # no difference straddles ReLU's kink
    h = 1e-6
    for t, got in ((X, ref["dx"]), (W, ref["dw"]), (b, ref["db"])):
        for i in range(0, t.numel(), 3):
            f = t.view(-1)
            old = float(f[i])
            f[i] = old + h
            up = loss(X, W, b)
            f[i] = old - h
            down = loss(X, W, b)
            f[i] = old
            # third derivatives of order 1: truncation ~ h^2, rounding ~ 1e-16 / h
            assert abs((up - down) / (2 * h) - float(got.reshape(-1)[i])) < 1e-7
