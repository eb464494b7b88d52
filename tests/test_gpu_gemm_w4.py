"""Products of tensors with packed 4-bit weights on the GPU against 64 bits: out = g sum x w, at 1e-5 of sum |x||w| (binary32 sums, the bar of the other products here)
and one rounding of the result; exactly, where every partial sum is a binary32 number."""
import numpy as np
import pytest
import torch

from gpu_util import assert_bf16_gemm_close, assert_gemm_close
from paper_2505_19115_amd import binding as nv

pytestmark = pytest.mark.gpu
FORMATS = {"nvfp4": nv.NVFP4, "mxfp4": nv.MXFP4, "e4m3_32": nv.Format(32, nv.SCALE_E4M3, 1), "e4m3_64": nv.Format(64, nv.SCALE_E4M3, 1), "e4m3_128": nv.Format(128, nv.SCALE_E4M3, 1),
           "nvfp4_no_g": nv.Format(16, nv.SCALE_E4M3, 0)}
DTYPES = [torch.bfloat16, torch.float32]
GRID = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64)
E4M3 = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double()


def values(codes, scales, fmt):
    """The numbers of a packed weight without g, [N, K] in 64 bits."""
    codes, scales = codes.cpu().long(), scales.cpu().long()
    c = GRID[torch.stack([codes & 15, codes >> 4], dim=2).view(codes.shape[0], -1)]
    s = E4M3[scales] if fmt.scale == nv.SCALE_E4M3 else torch.exp2(scales.double() - 127)
    return c * s.repeat_interleave(fmt.block, dim=1)


def packed(N, K, fmt, seed=0):
    """A weight as quantize leaves it, some blocks of zeros, some rows far larger."""
    g = torch.Generator().manual_seed(seed + N + K)
    w = torch.randn(N, K, generator=g) * 0.02
    w[torch.rand(N, generator=g) < 0.1] *= 300
    w[torch.rand(N, K // 32, generator=g).repeat_interleave(32, 1) < 0.05] = 0
    if fmt.tensor_scale or fmt.scale == nv.SCALE_E8M0:
        return nv.quantize(w.cuda(), fmt=fmt)
    codes, scales, g1 = nv.quantize(w.cuda(), fmt=nv.Format(fmt.block, fmt.scale, 1))
    return codes, scales, g1


def activation(M, K, dtype, seed=1, pad=0):
    g = torch.Generator().manual_seed(seed + M + K)
    return (torch.randn(M, K + pad, generator=g) * torch.rand(M, 1, generator=g).mul(4).exp()).to(dtype)[:, :K]


def check(got, x, w, g, what):
    ref, size = (x.double() @ w.t() * g).numpy(), (x.double().abs() @ w.abs().t() * abs(g)).numpy()
    if got.dtype == torch.bfloat16:
        assert_bf16_gemm_close(got.cpu().double().numpy(), ref, size, what)
    else:
        err = np.abs(got.cpu().double().numpy() - ref)
        assert (err <= 1e-5 * size + 1e-300).all(), f"{what}: {(err / np.maximum(size, 1e-300)).max()} of sum |x||w|"


@pytest.mark.parametrize("out", DTYPES)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("name", FORMATS)
@pytest.mark.parametrize("M, N, K", [(1, 1, 128), (1, 17, 256), (2, 64, 384), (7, 100, 640), (16, 48, 1024), (17, 33, 512), (31, 130, 256), (33, 16, 2048), (64, 257, 384), (65, 65, 896),
                                     (100, 40, 128), (130, 300, 1152), (200, 520, 256)])
def test_products(M, N, K, name, dtype, out):
    fmt = FORMATS[name]
    w = packed(N, K, fmt)
    x = activation(M, K, dtype)
    got = nv.gemm_w4(x.cuda(), w, fmt, out_dtype=out)
    assert got.shape == (M, N) and got.dtype == out
    check(got, x, values(w[0], w[1], fmt), float(w[2]) if fmt.tensor_scale else 1.0, f"{M} {N} {K} {name}")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("K", [32, 64, 96, 160, 224, 288, 992, 4064, 12320])
@pytest.mark.parametrize("M", [1, 16, 40, 129])
def test_contractions_between_k_tiles(M, K, dtype):
    for name in ("nvfp4", "mxfp4"):
        w = packed(50, K, FORMATS[name])
        x = activation(M, K, dtype)
        check(nv.gemm_w4(x.cuda(), w, FORMATS[name], out_dtype=torch.float32), x, values(w[0], w[1], FORMATS[name]), float(w[2]), f"{M} {K} {name}")


@pytest.mark.parametrize("M", [1, 5, 16, 64, 150])
def test_every_code_and_scale_exactly(M):
    # x picks single weights: row m of x is one power of two; w runs over all codes and all finite scale bytes.  Results are the weights themselves.
    N, K = 64, 2048
    for fmt in (nv.NVFP4, nv.Format(32, nv.SCALE_E4M3, 1), nv.MXFP4):
        codes = torch.arange(N * K // 2, dtype=torch.int64).mul(167).add(31).remainder(256).to(torch.uint8).view(N, K // 2)
        most = 126 if fmt.scale == nv.SCALE_E4M3 else 200
        least = 0 if fmt.scale == nv.SCALE_E4M3 else 60
        scales = (torch.arange(N * K // fmt.block) % (most - least + 1) + least).to(torch.uint8).view(N, K // fmt.block)
        v = values(codes, scales, fmt)
        g = torch.Generator().manual_seed(M)
        at = torch.randint(0, K, (M,), generator=g)
        x = torch.zeros(M, K)
        x[torch.arange(M), at] = 4.0
        for dtype in DTYPES:
            got = nv.gemm_w4(x.to(dtype).cuda(), (codes.cuda(), scales.cuda(), torch.tensor([0.25], device="cuda")), fmt, out_dtype=torch.float32)
            want = v[:, at].t() * (1 if fmt.tensor_scale else 4)
            assert torch.equal(got.cpu().double(), want)


@pytest.mark.parametrize("M", [1, 16, 33, 130])
def test_binary32_rows_keep_their_bits(M):
    # weights that are one power of two and zeros: a result is an element of x, all 24 bits of it, times that
    N, K = 96, 512
    g = torch.Generator().manual_seed(M)
    at = torch.randint(0, K, (N,), generator=g)
    codes = torch.zeros(N, K // 2, dtype=torch.uint8)
    codes[torch.arange(N), at // 2] = torch.where(at % 2 == 0, 0x02, 0x20).to(torch.uint8)  # the code of 1
    scales = torch.full((N, K // 16), 0x38, dtype=torch.uint8)  # 1
    x = torch.randn(M, K, generator=g) * torch.exp2(torch.randint(-30, 30, (M, K), generator=g).float())
    got = nv.gemm_w4(x.cuda(), (codes.cuda(), scales.cuda(), torch.tensor([2.0], device="cuda")), out_dtype=torch.float32)
    assert torch.equal(got.cpu(), 2 * x[:, at])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M", [3, 20, 140])
def test_views_and_guards(M, dtype):
    N, K = 70, 416
    w = packed(N, K, nv.NVFP4)
    x = activation(M, K, dtype)
    base = torch.full((M, K + 11), float("nan"), dtype=dtype, device="cuda")
    view = base[:, 5: 5 + K]
    view.copy_(x)
    for out in DTYPES:
        room = torch.full((M + 2, N + 9), 77.0, dtype=out, device="cuda")
        got = nv.gemm_w4(view, w, out=room[1: M + 1, 3: 3 + N])
        assert torch.equal(got, nv.gemm_w4(x.cuda(), w, out_dtype=out))
        room[1: M + 1, 3: 3 + N] = 77
        assert (room == 77).all()


@pytest.mark.parametrize("M", [1, 20, 140])
def test_infinities_stay_in_their_rows(M):
    N, K = 40, 256
    w = packed(N, K, nv.NVFP4)
    for dtype in DTYPES:
        x = activation(M + 1, K, dtype)
        clean = nv.gemm_w4(x.cuda(), w, out_dtype=torch.float32)
        x[M // 2, 7] = float("inf")
        x[M, 250] = float("nan")
        got = nv.gemm_w4(x.cuda(), w, out_dtype=torch.float32)
        rows = [i for i in range(M + 1) if i not in (M // 2, M)]
        assert torch.equal(got[rows], clean[rows]) and torch.isnan(got[M]).all()
        v = values(w[0], w[1], nv.NVFP4)[:, 7]
        want = torch.where(v == 0, float("nan"), float("inf") * v)
        if M // 2 != M:
            assert torch.equal(torch.nan_to_num(got[M // 2].cpu().double(), nan=7.0), torch.nan_to_num(want, nan=7.0))


def offsets_of(sizes, rows):
    o = [0]
    for n in sizes:
        o.append(o[-1] + n)
    assert o[-1] <= rows
    return torch.tensor(o, dtype=torch.int32)


SIZES = [[1], [0, 3, 0], [2, 0, 0, 5, 1, 0, 16, 17], [0, 0, 0, 0], [40, 0, 3, 70], [130, 1, 0, 129, 64], [1] * 40, [0] * 60 + [9] + [0] * 3, [16] * 16]


@pytest.mark.parametrize("out", DTYPES)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("name", ["nvfp4", "mxfp4", "e4m3_128"])
@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: "-".join(map(str, s))[:30])
def test_experts(sizes, name, dtype, out):
    fmt, E, N, K, T, k = FORMATS[name], len(sizes), 50, 384, 21, 3
    rows = sum(sizes) + 5  # the last five are nobody's
    codes, scales, g = packed(E * N, K, fmt)
    if fmt.tensor_scale:
        g = torch.rand(E, generator=torch.Generator().manual_seed(1)).cuda() + 0.5
    x = activation(T, K, dtype)
    order = torch.randint(0, T * k, (rows,), generator=torch.Generator().manual_seed(2)).int()
    order[::7] = -1
    order[3::11] = T * k + 4  # past the last row of x
    order[sum(sizes):] = 0
    offsets = offsets_of(sizes, rows)
    got = nv.gemm_w4_experts(x.cuda(), (codes, scales, g), offsets.cuda(), fmt, order=order.cuda(), top_k=k, out_dtype=out)
    gathered = torch.where(((order >= 0) & (order < T * k))[:, None], x[(order.long() // k).clamp(0, T - 1)], 0)
    assert not got[sum(sizes):].any()
    w = values(codes, scales, fmt).view(E, N, K)
    for e in range(E):
        a, b = int(offsets[e]), int(offsets[e + 1])
        if b > a:
            check(got[a:b], gathered[a:b], w[e], float(g[e]) if fmt.tensor_scale else 1.0, f"expert {e}")
    # rows that are there already, one g for all
    g1 = torch.tensor([1.5], device="cuda")
    got = nv.gemm_w4_experts(gathered.cuda(), (codes, scales, g1), offsets.cuda(), fmt, out_dtype=out)
    assert not got[sum(sizes):].any()
    for e in range(E):
        a, b = int(offsets[e]), int(offsets[e + 1])
        if b > a:
            check(got[a:b], gathered[a:b], w[e], 1.5 if fmt.tensor_scale else 1.0, f"expert {e}")


def test_same_bits():
    for M in (1, 16, 40, 300):
        w, x = packed(500, 2048, nv.NVFP4), activation(M, 2048, torch.bfloat16).cuda()
        first = nv.gemm_w4(x, w, out_dtype=torch.float32)
        assert all(torch.equal(first, nv.gemm_w4(x, w, out_dtype=torch.float32)) for _ in range(5))


def test_empty_and_refusals():
    w = packed(32, 256, nv.NVFP4)
    x = torch.randn(4, 256, device="cuda")
    assert nv.gemm_w4(x[:0], w).shape == (0, 32)
    assert not nv.gemm_w4(x[:, :0], (w[0][:, :0], w[1][:, :0], w[2])).any()  # a sum of nothing
    with pytest.raises(ValueError):
        nv.gemm_w4(x[:, :128], w)
    with pytest.raises(TypeError):  # (a view)
        nv.gemm_w4(x, (w[0], w[1][:, :8], w[2]))
    with pytest.raises(ValueError):
        nv.gemm_w4(x, (w[0], w[1][:, :8].contiguous(), w[2]))
    with pytest.raises(TypeError):
        nv.gemm_w4(x, (w[0], w[1], None))
    with pytest.raises(TypeError):
        nv.gemm_w4(x, (w[0].char(), w[1], w[2]))
    with pytest.raises(TypeError):
        nv.gemm_w4(x.half(), w)
    with pytest.raises(ValueError):
        nv.gemm_w4(x.cpu(), w)
    with pytest.raises(ValueError):
        nv.gemm_w4(x[:1].expand(4, 256), w)
    with pytest.raises(ValueError):
        nv.gemm_w4(x, w, out=torch.empty(4, 31, device="cuda"))
    with pytest.raises(nv.Nvfp4Error):
        nv.gemm_w4(x, (w[0], w[1], w[2]), nv.Format(16, nv.SCALE_E8M0, 0))
    o = torch.tensor([0, 2, 4], dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        nv.gemm_w4_experts(x, packed(33, 256, nv.NVFP4), o)
    with pytest.raises(TypeError):
        nv.gemm_w4_experts(x, w, o.long())
    with pytest.raises(nv.Nvfp4Error):
        nv.gemm_w4_experts(x, w, o, order=o, top_k=0)
    assert nv.gemm_w4_experts(x[:0], w, torch.zeros(3, dtype=torch.int32, device="cuda")).shape == (0, 16)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("each", [1, 9, 16, 17, 40, 130])
def test_rows_that_an_order_does_not_name_are_zeros(each, dtype):
    # whatever their expert's weight holds, in the kernel for few rows (up to 16 an expert) and in tiles: NaN scale bytes, a g that is infinite or NaN
    E, N, K, T, k = 3, 50, 384, 21, 3
    codes, scales, _ = packed(E * N, K, nv.NVFP4)
    scales[N: 2 * N] = 0x7F
    g = torch.tensor([1.0, 1.0, float("inf")], device="cuda")
    x = activation(T, K, dtype).cuda()
    rows = E * each
    order = torch.randint(0, T * k, (rows,), generator=torch.Generator().manual_seed(each)).int()
    order[::2] = -1
    order[::6] = T * k + 4
    offsets = offsets_of([each] * E, rows).cuda()
    named = ((order >= 0) & (order < T * k)).cuda()
    for out in DTYPES:
        got = nv.gemm_w4_experts(x, (codes, scales, g), offsets, order=order.cuda(), top_k=k, out_dtype=out)
        assert not torch.isnan(got[~named]).any() and not got[~named].any()
        second = torch.arange(rows, device="cuda") // each == 1
        assert torch.isnan(got[named & second]).all() and torch.isfinite(got[:each]).all()
        # g alone is not a number: the products of x that are zeros are
        got = nv.gemm_w4_experts(x, (codes, scales, g[2:] * 0), offsets, order=order.cuda(), top_k=k, out_dtype=out)
        assert not torch.isnan(got[~named]).any() and not got[~named].any() and torch.isnan(got[named]).all()


@pytest.mark.parametrize("g", [float("inf"), float("nan")])
@pytest.mark.parametrize("M", [1, 16, 17, 140])
def test_a_sum_of_nothing_is_zero_whatever_g_is(M, g):
    x = torch.randn(M, 32, device="cuda")[:, :0]
    w = (torch.empty(6, 0, dtype=torch.uint8, device="cuda"), torch.empty(6, 0, dtype=torch.uint8, device="cuda"), torch.tensor([g], device="cuda"))
    for out in DTYPES:
        got = nv.gemm_w4(x, w, out_dtype=out)
        assert got.shape == (M, 6) and (got == 0).all()
        assert (nv.gemm_w4_experts(x, w, torch.tensor([0, M, M], dtype=torch.int32, device="cuda"), out_dtype=out) == 0).all()


@pytest.mark.parametrize("top_k", [0, -1, 1 << 31, (1 << 32) + 1, -(1 << 32) + 1, (1 << 64) + 1])
def test_rows_of_a_token_that_no_call_takes(top_k):
    # also where 32 bits of the number would be a number that is allowed
    w, x = packed(32, 256, nv.NVFP4), torch.randn(4, 256, device="cuda")
    o = torch.tensor([0, 2, 4], dtype=torch.int32, device="cuda")
    with pytest.raises(nv.Nvfp4Error):
        nv.gemm_w4_experts(x, w, o, order=torch.arange(4, dtype=torch.int32, device="cuda"), top_k=top_k)


@pytest.mark.parametrize("M", [1, 17, 140])
def test_e8m0_scales_to_both_ends(M):
    # every byte that nvfp4_quantize writes (0 .. 252), and every code; x picks single weights.  Weights under 2^-126 may count as 0
    N, K = 64, 2048
    codes = torch.arange(N * K // 2, dtype=torch.int64).mul(167).add(31).remainder(256).to(torch.uint8).view(N, K // 2)
    scales = (torch.arange(N * K // 32) % 253).to(torch.uint8).view(N, K // 32)
    v = values(codes, scales, nv.MXFP4)
    at = torch.randint(0, K, (M,), generator=torch.Generator().manual_seed(M))
    x = torch.zeros(M, K)
    x[torch.arange(M), at] = 1.0
    for dtype in DTYPES:
        got = nv.gemm_w4(x.to(dtype).cuda(), (codes.cuda(), scales.cuda(), None), nv.MXFP4, out_dtype=torch.float32).cpu().double()
        want = v[:, at].t()
        assert ((got == want) | ((want.abs() < 2.0 ** -126) & (got == 0))).all()
