"""bf16 results of exact products and binary32 sums: the binary32 results, rounded once."""
import pytest
import torch

from paper_2505_19115_amd import binding as nv

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
# waves that divide the contraction, tiles of 128 x 128 and of 256 rows inside and at edges, contractions divided among workgroups, outputs past the last cache level
SIZES = [(1, 1, 128), (3, 5, 256), (16, 4100, 640), (33, 9000, 256), (100, 12300, 128), (300, 515, 1024), (2048, 2304, 384), (2100, 2301, 384), (512, 1000, 8064), (300, 129, 16256),
         (16384, 8200, 128)]


def operands(seed, M, N, K):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [nv.fp8_quantize(torch.randn(n, K, generator=g, device="cuda"))[0] for n in (M, N)]


@pytest.mark.parametrize("M, N, K", SIZES)
def test_the_sums_of_binary32_results(M, N, K):
    a, b = operands(M + N, M, N, K)
    ref = nv.fp8_gemm(a, b, out_dtype=F32).to(BF16)
    assert torch.equal(nv.fp8_gemm(a, b, exact=True), ref)
    assert torch.equal(nv.fp8_gemm(a, b, out_dtype=F32, exact=True), nv.fp8_gemm(a, b, out_dtype=F32))
    base = torch.full((M + 1, N + 7), -7.0, dtype=BF16, device="cuda")
    nv.fp8_gemm(a, b, out=base[:M, 3: N + 3], exact=True)
    assert torch.equal(base[:M, 3: N + 3], ref) and bool((base[:, :3] == -7).all()) and bool((base[:, N + 3:] == -7).all()) and bool((base[M] == -7).all())


def test_products_that_the_instruction_cuts_off():
    # 2^16 - 2^16 and a small product beside them in a group of eight: the sum is the small product
    for M, N in ((16, 16), (200, 600), (2100, 2300)):
        a, b = torch.zeros(M, 128), torch.zeros(N, 128)
        a[:, 0], a[:, 1], a[:, 2], b[:, 0], b[:, 1], b[:, 2] = 256, -256, 0.25, 256, 256, 3
        q, r = nv.fp8_quantize(a.cuda())[0], nv.fp8_quantize(b.cuda())[0]
        assert bool((nv.fp8_gemm(q, r, exact=True) == 0.75).all()) and not bool((nv.fp8_gemm(q, r) == 0.75).any())


@pytest.mark.parametrize("M, N, K", [(5, 7, 256), (300, 515, 256), (2100, 2300, 256), (512, 1000, 8064)])
def test_blocks_that_bf16_does_not_hold(M, N, K):
    g = torch.Generator(device="cuda").manual_seed(K)
    x, w = torch.randn(M, K, generator=g, device="cuda"), torch.randn(N, K, generator=g, device="cuda") * 2.0 ** -30
    x[M // 2, 3] = torch.finfo(BF16).min
    a, b = nv.fp8_quantize(x)[0], nv.fp8_quantize(w)[0]
    out = nv.fp8_gemm(a, b, exact=True)
    assert bool(out.isfinite().all()) and torch.equal(out, nv.fp8_gemm(a, b, out_dtype=F32).to(BF16))


@pytest.mark.parametrize("T, k, E, N, K, drop", [(5, 2, 4, 40, 256, 0.3), (64, 8, 64, 96, 1024, 0.1), (300, 2, 8, 515, 384, 0.1), (3000, 2, 3, 2304, 640, 0.1), (2000, 4, 8, 1051, 260, 0.0)])
def test_experts(T, k, E, N, K, drop):
    g = torch.Generator(device="cuda").manual_seed(T)
    ids = torch.topk(torch.randn(T, E, generator=g, device="cuda"), k, dim=1).indices
    o = nv.moe_sort(torch.where(torch.rand(T, k, generator=g, device="cuda") < drop, -1, ids), E)
    a, ac = nv.fp8_quantize(torch.randn(T, K, generator=g, device="cuda"), cols=True, order=o.order, top_k=k, offsets=o.offsets)
    b = nv.fp8_quantize(torch.randn(E, N, K, generator=g, device="cuda"))[0]
    dc = nv.fp8_quantize(torch.randn(T * k, N, generator=g, device="cuda"), rows=False, cols=True, offsets=o.offsets)[1]
    assert torch.equal(nv.fp8_gemm_experts(a, b, o.offsets, exact=True), nv.fp8_gemm_experts(a, b, o.offsets, out_dtype=F32).to(BF16))
    assert torch.equal(nv.fp8_gemm_experts_dw(dc, ac, o.offsets, exact=True), nv.fp8_gemm_experts_dw(dc, ac, o.offsets, out_dtype=F32).to(BF16))


def test_other_calls_do_not_know_the_type():
    x = torch.zeros(4, 128, device="cuda")
    stream, p = torch.cuda.current_stream().cuda_stream, x.data_ptr()
    assert nv.lib.nvfp4_moe_gather(p, nv.BF16_EXACT, 4, 128, 128, p, 1, 4, p, stream) == nv.EINVAL
    assert nv.lib.nvfp4_fp8_quantize(p, nv.BF16_EXACT, 1, 4, 128, 128, None, 1, 4, None, 0, p, p, None, None, stream) == nv.EINVAL
    with pytest.raises(TypeError):
        nv.fp8_gemm(*operands(1, 4, 4, 128), out_dtype=torch.float16, exact=True)
