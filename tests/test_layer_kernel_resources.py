"""Registers of the layers' built kernels, read from the objects that the build left: none
spills vector registers to memory but the fp32 256 x 128 tiles of dW, which are the faster of
two all the same. (Scalar registers spill to lanes of vector registers.)"""
import os

import pytest

from tests import test_kernel_resources as K

BUILT = os.path.join(K.ROOT, "paper_2606_30497_amd", "_build")


@pytest.mark.parametrize("source", ["linear", "linear_gemm", "linear_gemm_f32", "linear_skinny", "dropout"])
def test_no_spills(tmp_path, monkeypatch, source):
    obj = os.path.join(BUILT, source + ".hip.o")
    if not os.path.exists(obj) or not os.path.exists(K.BIN):
        pytest.skip("nothing built, or no ROCm tools")
    monkeypatch.setattr(K, "OBJ", obj)
    kernels = K._kernels(tmp_path)
    assert kernels
    for name, r in kernels.items():
        if name == "k_gemm_f32<2, 256, 128, 4, 2>":
            assert r["vgpr_spill_count"] <= 29 and r["private_segment_fixed_size"] <= 56, r
        else:
            assert r["vgpr_spill_count"] == r["private_segment_fixed_size"] == 0, (name, r)
