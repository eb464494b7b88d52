"""Products with packed 4-bit weights on every kernel that the size rules choose: each of them is asked for by a shape that reaches it, with odd numbers of rows and columns, a
contraction that ends inside a K tile, rows between others, results between guards, experts of uneven sizes.  Against 64 bits, at 1e-5 of sum |x||w| (binary32 sums, the bar of the
other products here) and one rounding of the result."""
import pytest
import torch

from paper_2505_19115_amd import binding as nv

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
FORMATS = {"nvfp4": nv.NVFP4, "mxfp4": nv.MXFP4, "e4m3_32": nv.Format(32, nv.SCALE_E4M3, 1), "e4m3_128": nv.Format(128, nv.SCALE_E4M3, 1)}
GRID = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64)
E4M3 = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double()

# x's type, its rows on 16-byte boundaries, rows, columns of the product, its kernel (of three experts' the same where the last number says so, or their rows and columns)
KERNELS = [
    (BF16, True, 16, 8201, ("few rows", 16, 16, 4)), (BF16, False, 3, 8201, ("few rows", 16, 16, 4)), (F32, True, 16, 8201, ("few rows", 16, 16, 4)), (BF16, True, 16, 300, ("few rows", 16, 16, 8)),
    (BF16, True, 65, 50, ("direct", 32, 64, 4)), (BF16, True, 9000, 50, ("direct", 64, 64, 4)), (BF16, True, 1500, 2049, ("direct", 128, 64, 4)), (BF16, True, 9000, 700, ("direct", 128, 128, 4)),
    (BF16, True, 9000, 1001, ("direct", 112, 192, 4)), (BF16, True, 9000, 3001, ("direct", 128, 256, 4)),
    (BF16, False, 65, 50, ("staged", 32, 64, 4)), (BF16, False, 9000, 130, ("staged", 64, 64, 4)), (BF16, False, 1500, 2049, ("staged", 128, 128, 4)),
    (F32, True, 65, 50, ("staged", 32, 64, 4)), (F32, True, 1280, 1921, ("staged", 32, 128, 4)), (F32, True, 2000, 6001, ("staged", 32, 256, 4)),
]
EXPERTS = [
    (BF16, True, 90, 40, 130, ("few rows", 16, 16, 8)), (BF16, True, 257, 40, 130, ("few rows", 16, 16, 4)), (BF16, False, 257, 40, 130, ("few rows", 16, 16, 4)), (F32, True, 257, 40, 130, ("few rows", 16, 16, 4)),
    (BF16, True, 65, 3, 50, ("direct", 32, 64, 4)), (BF16, True, 9000, 3, 50, ("direct", 64, 64, 4)), (BF16, True, 1500, 3, 2049, ("direct", 128, 64, 4)), (BF16, True, 9000, 3, 700, ("direct", 128, 128, 4)),
    (BF16, True, 9000, 3, 1001, ("direct", 112, 192, 4)), (BF16, True, 9000, 3, 3001, ("direct", 128, 256, 4)),
    (BF16, False, 65, 3, 50, ("staged", 32, 64, 4)), (BF16, False, 9000, 3, 130, ("staged", 64, 64, 4)), (BF16, False, 3001, 8, 1001, ("staged", 128, 128, 4)),
    (F32, True, 65, 3, 50, ("staged", 32, 64, 4)), (F32, True, 1280, 3, 1921, ("staged", 32, 128, 4)), (F32, True, 2000, 3, 6001, ("staged", 32, 256, 4)),
]


def contraction(fmt):
    return 384 if fmt.block == 128 else 416  # (416: a quarter of the last K tile)


def packed(rows, K, fmt):
    g = torch.Generator(device="cuda").manual_seed(rows)
    w = torch.randn(rows, K, generator=g, device="cuda") * 0.02
    w[torch.rand(rows, generator=g, device="cuda") < 0.1] *= 300
    return nv.quantize(w, fmt=fmt)


def values(codes, scales, fmt):
    c = GRID.cuda()[torch.stack([codes & 15, codes >> 4], dim=2).int().view(codes.shape[0], -1)]
    s = E4M3.cuda()[scales.int()] if fmt.scale == nv.SCALE_E4M3 else torch.exp2(scales.double() - 127)
    return c * s.repeat_interleave(fmt.block, dim=1)


def rows_between_others(M, K, dtype, aligned):
    """Rows of a larger pitch, on 16-byte boundaries or on none, NaN between them."""
    g = torch.Generator(device="cuda").manual_seed(M + K)
    base = torch.full((M, K + (16 if aligned else 11)), float("nan"), dtype=dtype, device="cuda")
    x = base[:, 8: 8 + K] if aligned else base[:, 5: 5 + K]
    x.copy_(torch.randn(M, K, generator=g, device="cuda") * torch.rand(M, 1, generator=g, device="cuda").mul(4).exp())
    return x


def right(got, x, w, g):
    ref, slack = x.double() @ w.t() * g, (x.double().abs() @ w.abs().t()) * (1e-5 * abs(g)) + 1e-300
    if got.dtype is F32:
        return bool(((got.double() - ref).abs() <= slack).all())
    lo, hi = (ref - slack * (1 + 1e-6)).float().bfloat16(), (ref + slack * (1 + 1e-6)).float().bfloat16()
    return bool(((got >= lo) & (got <= hi)).all())


@pytest.mark.parametrize("name", FORMATS)
@pytest.mark.parametrize("dtype, aligned, M, N, kernel", KERNELS)
def test_products(dtype, aligned, M, N, kernel, name):
    fmt = FORMATS[name]
    K = contraction(fmt)
    assert nv.gemm_w4_kernel(M, N, K, dtype=dtype, aligned=aligned) == kernel
    w, x = packed(N, K, fmt), rows_between_others(M, K, dtype, aligned)
    for out in (BF16, F32):
        room = torch.full((M + 2, N + 9), 77.0, dtype=out, device="cuda")
        got = nv.gemm_w4(x, w, fmt, out=room[1: M + 1, 3: 3 + N])
        assert right(got, x, values(w[0], w[1], fmt), float(w[2]) if fmt.tensor_scale else 1.0)
        room[1: M + 1, 3: 3 + N] = 77
        assert (room == 77).all()


@pytest.mark.parametrize("name", FORMATS)
@pytest.mark.parametrize("dtype, aligned, R, E, N, kernel", EXPERTS)
def test_experts(dtype, aligned, R, E, N, kernel, name):
    fmt, k, out = FORMATS[name], 3, F32 if N % 2 else BF16
    K = contraction(fmt)
    assert nv.gemm_w4_kernel(R, N, K, E, dtype, aligned) == kernel
    codes, scales, g = packed(E * N, K, fmt)
    if fmt.tensor_scale:
        g = torch.rand(E, generator=torch.Generator().manual_seed(E)).cuda() + 0.5
    # uneven experts, one of them of no rows; the last seven rows are nobody's
    share = torch.rand(E, generator=torch.Generator().manual_seed(R)) ** 2
    share[0] = 0
    cut = (share.cumsum(0) / share.sum() * (R - 7)).round().int()
    offsets = torch.cat([torch.zeros(1, dtype=torch.int32), cut])
    T = R // 2 + 1
    x = rows_between_others(T, K, dtype, aligned)
    order = torch.randint(0, T * k, (R,), generator=torch.Generator().manual_seed(2)).int()
    order[::7] = -1
    order[3::11] = T * k + 4  # past the last row of x
    gathered = torch.where(((order >= 0) & (order < T * k)).cuda()[:, None], x[(order.long() // k).clamp(0, T - 1).cuda()], 0)
    placed = rows_between_others(R, K, dtype, aligned)
    placed.copy_(gathered)
    v = values(codes, scales, fmt).view(E, N, K)
    for got in (nv.gemm_w4_experts(x, (codes, scales, g), offsets.cuda(), fmt, order=order.cuda(), top_k=k, out_dtype=out),
                nv.gemm_w4_experts(placed, (codes, scales, g), offsets.cuda(), fmt, out_dtype=out)):
        assert not got[R - 7:].any()
        for e in range(E):
            a, b = int(offsets[e]), int(offsets[e + 1])
            if b > a:
                assert right(got[a:b], gathered[a:b], v[e], float(g[e]) if fmt.tensor_scale else 1.0), e
