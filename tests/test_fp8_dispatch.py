"""CPU-only checks of the rules that choose a kernel for an 8-bit product (256 compute units where there is no GPU to ask)."""
import pytest
import torch

from paper_2505_19115_amd import binding as nv

L = nv.lib


@pytest.mark.parametrize("M, N, K, bf16, f32", [(384, 6016, 7296, True, True), (200, 5000, 4096, True, True), (777, 1025, 8192, True, True), (64, 2048, 16384, True, True),
                                                (256, 1024, 8192, False, False), (128, 1024, 8192, False, False)])
def test_which_contractions_are_divided(M, N, K, bf16, f32):
    # against the few-row kernel at the price that it has where codes are expanded: binary32 384 x 6016 x 7296 took 75 us whole and takes 62 divided
    assert (L.nvfp4_fp8_gemm_workspace_bytes(M, N, K, nv.BF16) > 0) == bf16
    assert (L.nvfp4_fp8_gemm_workspace_bytes(M, N, K, nv.F32) > 0) == f32


F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("call, M, N, K, groups, dtype, want", [
    ("fp8_gemm", 16, 11008, 4096, 0, BF16, ("few rows", 16, 48, 4, False)), ("fp8_gemm", 777, 4099, 384, 0, BF16, ("tiles", 128, 128, 1, False)),
    ("fp8_gemm", 4096, 4096, 11008, 0, BF16, ("wide", 256, 256, 1, False)), ("fp8_gemm", 777, 12288, 4096, 0, BF16, ("wide", 256, 192, 1, False)),
    ("fp8_gemm", 4096, 4096, 11008, 0, F32, ("wide", 256, 128, 1, False)), ("fp8_gemm", 8192, 8192, 128, 0, F32, ("wide", 256, 128, 1, True)),
    ("fp8_gemm", 512, 4096, 11008, 0, BF16, ("divided", 256, 128, 4, False)), ("fp8_gemm", 1000, 6144, 9856, 0, BF16, ("divided", 256, 192, 2, False)),
    ("fp8_gemm", 777, 4608, 9088, 0, BF16, ("divided", 256, 256, 3, False)), ("nvfp4_fp8_gemm", 777, 4608, 9088, 0, BF16, ("wide", 256, 128, 1, False)),
    ("fp8_gemm_experts", 16, 2048, 4096, 8, BF16, ("few rows", 16, 32, 4, False)), ("fp8_gemm_experts", 16384, 4096, 2048, 16, BF16, ("wide", 256, 256, 1, False)),
    ("fp8_gemm_experts_dw", 4096, 2048, 16384, 16, BF16, ("wide", 256, 256, 1, True)), ("fp8_gemm_experts_dw", 33, 40, 600, 300, F32, ("tiles", 128, 128, 1, False))])
def test_which_kernel_serves_a_product(call, M, N, K, groups, dtype, want):
    assert nv.fp8_gemm_kernel(call, M, N, K, groups, dtype) == want
    if dtype is F32:  # the kernels of binary32 results, the output of half the bytes
        assert nv.fp8_gemm_kernel(call, M, N, K, groups, BF16, exact=True)[:4] == want[:4]


def test_no_kernel():
    for args in ((0, 4, 128), (4, 0, 128), (4, 4, 100), (4, 4, -128), (1 << 31, 4, 128), (4, 4, (1 << 23) + 128)):
        assert nv.fp8_gemm_kernel("fp8_gemm", *args) is None
    assert nv.fp8_gemm_kernel("fp8_gemm", (1 << 31) - 1, (1 << 31) - 1, 128) is None and nv.fp8_gemm_kernel("fp8_gemm_experts", 4, 1 << 22, 128, 512) is None
    assert nv.fp8_gemm_kernel("fp8_gemm_experts_dw", 1 << 22, 4, 128, 512) is None and nv.fp8_gemm_kernel("fp8_gemm_experts_dw", 4, 4, 1 << 30, 2) is None
    for groups in (0, 513):
        assert nv.fp8_gemm_kernel("fp8_gemm_experts", 4, 4, 128, groups) is None and nv.fp8_gemm_kernel("fp8_gemm_experts_dw", 4, 4, 128, groups) is None
    assert L.nvfp4_host_fp8_gemm_kernel(4, 4, 4, 128, 1, nv.BF16, None) == 0 and L.nvfp4_host_fp8_gemm_kernel(0, 4, 4, 128, 1, nv.BF16, None) == 0
