"""Experts' rows of one type combined into another, and the gradient of that, against 64 bits: one rounding, to the result's type.

Bounds: a combined element is a chain of top_k fused multiply-adds in binary32, top_k 2^-24 sum |w y|, dweights of D elements (D / 64 + 22) 2^-24 sum |dout y|; results
add their own rounding, half of their type's eps (the two roundings of a bf16 result, to binary32 and from there, 2^-6 of it more)."""
import pytest
import torch

from paper_2505_19115_amd import binding as nv

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
MIXED = [(F32, BF16), (BF16, F32)]  # of the rows, of the result
OWN = {t: torch.finfo(t).eps / 2 * (1 + 2.0 ** -6) for t in (BF16, F32)}


def case(seed, T, k, E, D, rows, out):
    g = torch.Generator().manual_seed(seed)
    ids = torch.randint(-1, E, (T, k), generator=g)
    o = nv.moe_sort(ids.cuda(), E)
    y, dout = torch.randn(T * k, D, generator=g).to(rows), torch.randn(T, D, generator=g).to(out)
    y[int(o.offsets[-1]):] = float("nan")
    return o, y, dout, torch.rand(T, k, generator=g)


@pytest.mark.parametrize("rows, out", MIXED)
@pytest.mark.parametrize("D", [1, 2, 3, 4, 5, 7, 8, 9, 15, 31, 64, 65, 127, 128, 129, 255, 257, 263, 511, 512, 515, 1023, 1025, 2048, 4100])
def test_mixed_types(D, rows, out):
    T, k, E = 37, 3, 4
    o, y, dout, w = case(D, T, k, E, D, rows, out)
    pos, kept = o.position.cpu().long(), int(o.offsets[-1])
    terms = torch.where((pos >= 0)[..., None], y.double()[pos.clamp(min=0)], 0.0)
    for weights in (w, None):
        got = nv.moe_combine(y.cuda(), o.position, None if weights is None else weights.cuda(), out_dtype=out).cpu()
        weighted = terms * (1.0 if weights is None else weights.double()[..., None])
        ref = weighted.sum(1)
        assert got.dtype == out and got.shape == (T, D)
        assert bool(((got.double() - ref).abs() <= k * 2.0 ** -24 * weighted.abs().sum(1) + OWN[out] * ref.abs() + 1e-300).all())
    dy, dw = (t.cpu() for t in nv.moe_combine_bwd(dout.cuda(), y.cuda(), w.cuda(), o.position, o.offsets, out_dtype=out))
    assert dy.dtype == rows and dw.dtype == F32
    ref = torch.zeros(T * k, D, dtype=torch.float64)
    t = torch.arange(T).repeat_interleave(k).view(T, k)[pos >= 0]
    ref[pos[pos >= 0]] = dout.double()[t] * w.double()[pos >= 0][:, None]
    assert bool(((dy.double() - ref).abs() <= (OWN[rows] + 2.0 ** -24) * ref.abs()).all()) and bool((dy[kept:] == 0).all())
    products = dout.double()[:, None] * terms
    assert bool(((dw.double() - products.sum(-1)).abs() <= (D / 64 + 22) * 2.0 ** -24 * products.abs().sum(-1) + 1e-300).all())
    assert bool((dw[pos < 0] == 0).all())


@pytest.mark.parametrize("rows, out", MIXED)
def test_streaming_loads(rows, out):
    # rows of large tensors come by another form of loads: the same bits as of a part by itself
    T, k, D = 4096, 2, 8192
    g = torch.Generator(device="cuda").manual_seed(1)
    o = nv.moe_sort(torch.randint(-1, 4, (T, k), generator=g, device="cuda"), 4)
    y, dout = torch.randn(T * k, D, generator=g, device="cuda").to(rows), torch.randn(T, D, generator=g, device="cuda").to(out)
    w = torch.rand(T, k, generator=g, device="cuda")
    part = lambda t: t[:, :104].contiguous()  # noqa: E731
    assert torch.equal(part(nv.moe_combine(y, o.position, w, out_dtype=out)), nv.moe_combine(part(y), o.position, w, out_dtype=out))
    dy, dw = nv.moe_combine_bwd(dout, y, w, o.position, o.offsets, out_dtype=out)
    assert torch.equal(part(dy), nv.moe_combine_bwd(part(dout), part(y), w, o.position, o.offsets, out_dtype=out)[0])
    terms = dout.double()[:, None] * torch.where((o.position >= 0)[..., None], y.double()[o.position.clamp(min=0).long()], 0)
    assert bool(((dw.double() - terms.sum(-1)).abs() <= (D / 64 + 22) * 2.0 ** -24 * terms.abs().sum(-1)).all())


def test_experts_are_rounded_once():
    # a product's binary32 rows, combined into bf16: no more than the product's own bound and one rounding, which bf16 rows pass
    T, k, E, K, N = 300, 4, 6, 256, 200
    g = torch.Generator().manual_seed(2)
    ids = torch.topk(torch.randn(T, E, generator=g), k, dim=1).indices
    o = nv.moe_sort(ids.cuda(), E)
    x, weight, w = torch.randn(T, K, generator=g), torch.randn(E, N, K, generator=g), torch.rand(T, k, generator=g)
    a, b = nv.fp8_quantize(x.cuda(), order=o.order, top_k=k)[0], nv.fp8_quantize(weight.cuda())[0]
    value = lambda q: (q.codes.cpu().double().view(q.codes.shape[0], -1, 128) * 2.0 ** (q.scales.cpu().t().double() - 127)[..., None]).view(q.codes.shape)  # noqa: E731
    A, B, pos = value(a), value(b).view(E, N, K), o.position.cpu().long()
    rows, S = torch.zeros(T, k, N, dtype=torch.float64), torch.zeros(T, k, N, dtype=torch.float64)
    for j in range(k):
        rows[:, j] = (A[pos[:, j]][:, None] * B[ids[:, j]]).sum(-1)
        S[:, j] = (A[pos[:, j]][:, None] * B[ids[:, j]]).abs().sum(-1)
    ref = (rows * w.double()[..., None]).sum(1)
    most = ((K / 32 + 48) * 2.0 ** -24 * S * w.double()[..., None]).sum(1) + k * 2.0 ** -24 * (rows * w.double()[..., None]).abs().sum(1) + OWN[BF16] * ref.abs()
    once = nv.moe_combine(nv.fp8_gemm_experts(a, b, o.offsets, out_dtype=F32), o.position, w.cuda(), out_dtype=BF16).cpu().double()
    twice = nv.moe_combine(nv.fp8_gemm_experts(a, b, o.offsets), o.position, w.cuda()).cpu().double()
    assert bool(((once - ref).abs() <= most).all()) and not bool(((twice - ref).abs() <= most).all())


def test_refusals():
    o, y, dout, w = (t.cuda() if torch.is_tensor(t) else t for t in case(3, 10, 2, 3, 16, F32, BF16))
    with pytest.raises(TypeError):
        nv.moe_combine(y, o.position, w, out_dtype=torch.float16)
    for bad in (lambda: nv.moe_combine_bwd(dout, y, w, o.position, o.offsets), lambda: nv.moe_combine_bwd(dout.float(), y, w, o.position, o.offsets, out_dtype=BF16)):
        with pytest.raises(ValueError):
            bad()
    stream, L = torch.cuda.current_stream().cuda_stream, nv.lib
    args = (y.data_ptr(), nv.F32, 20, 16, w.data_ptr(), o.position.data_ptr(), 10, 2)
    assert L.nvfp4_moe_combine_to(*args, dout.data_ptr(), 2, stream) == nv.EINVAL and L.nvfp4_moe_combine_to(*args, dout.data_ptr() + 1, nv.BF16, stream) == nv.EALIGN
    back = (y.data_ptr(), nv.F32, 20, 16, w.data_ptr(), o.position.data_ptr(), o.offsets.data_ptr(), 3, 10, 2, torch.empty_like(y).data_ptr(), w.clone().data_ptr(), stream)
    assert L.nvfp4_moe_combine_to_bwd(dout.data_ptr(), 2, *back) == nv.EINVAL and L.nvfp4_moe_combine_to_bwd(dout.data_ptr() + 1, nv.BF16, *back) == nv.EALIGN
