"""CPU-only checks of the rules that choose a kernel for an 8-bit product (256 compute units where there is no GPU to ask)."""
import pytest

from paper_2505_19115_amd import binding as nv

L = nv.lib


@pytest.mark.parametrize("M, N, K, bf16, f32", [(384, 6016, 7296, True, True), (200, 5000, 4096, True, True), (777, 1025, 8192, True, True), (64, 2048, 16384, True, True),
                                                (256, 1024, 8192, False, False), (128, 1024, 8192, False, False)])
def test_which_contractions_are_divided(M, N, K, bf16, f32):
    # against the few-row kernel at the price that it has where codes are expanded: binary32 384 x 6016 x 7296 took 75 us whole and takes 62 divided
    assert (L.nvfp4_fp8_gemm_workspace_bytes(M, N, K, nv.BF16) > 0) == bf16
    assert (L.nvfp4_fp8_gemm_workspace_bytes(M, N, K, nv.F32) > 0) == f32
