"""8-bit operators on the GPU against their definitions in 64 bits: the quantizer (bit for bit), the products of all kernels and their
gradients.

Bounds on products, for a contraction of K elements, with S = sum |a| |b| of the output:
  binary32: products are exact and enter binary32 sums, one rounding of at most 2^-24 S for each of K / 32 instructions, the waves'
            sums (at most 16) and, inside an instruction, for each of its 32 elements: (K / 32 + 48) 2^-24 S;
  bf16:     the 8-bit instruction adds products in groups of eight neighbours and drops of each what lies below 2^-13 of the
            power of two under the group's largest (test_groups_of_eight): 7 * 2^-13 S; its K / 8 further sums drop at most
            2^-23 S each; and the result's own rounding, half of bf16's eps of it.
"""
import pytest
import torch

from paper_2505_19115_amd import binding as nv

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float32]
ROUNDED = torch.finfo(torch.bfloat16).eps / 2  # 2^-8: eight significant bits


def two_to(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def quantized(x):
    """Row blocks of a binary64 matrix on the CPU: codes [R, P] (their values), scale bytes [P / 128, R], the values they stand for [R, K]."""
    R, K = x.shape
    P = -(-K // 128) * 128
    b = torch.zeros(R, P, dtype=torch.float64)
    b[:, :K] = x
    b = b.view(R, P // 128, 128)
    a = b.abs().amax(-1)
    e = torch.full_like(a, -127, dtype=torch.int64)
    for k in range(-126, 121):  # the smallest exponent with a <= 448 * 2^e
        e = torch.where(a > 448.0 * 2.0 ** (k - 1), k, e)
    v = b * two_to(-e)[..., None]
    step = two_to(torch.frexp(v.abs().clamp(min=2.0 ** -6)).exponent - 4)
    codes = torch.round(v / step) * step
    return codes.view(R, P), (e + 127).t().to(torch.uint8), (codes * two_to(e)[..., None]).view(R, P)[:, :K]


def values(q):
    s = two_to(q.scales.cpu().t().long() - 127)
    return (q.codes.cpu().double().view(q.codes.shape[0], -1, 128) * s[..., None]).view(q.codes.shape)


def same(q, x):
    codes, scales, _ = quantized(x)
    assert torch.equal(q.scales.cpu(), scales)
    assert torch.equal(q.codes.cpu().double(), codes)


def tensor(g, *shape, dtype=torch.bfloat16):
    x = torch.randn(*shape, generator=g, dtype=torch.float32) * torch.exp(2 * torch.rand(*shape[:-1], 1, generator=g) - 1)
    x[torch.rand(*shape, generator=g) < 0.002] *= 60
    return x.to(dtype)


def lost(K, dtype):
    return (K / 32 + 48) * 2.0 ** -24 if dtype == torch.float32 else 7 * 2.0 ** -13 + K / 8 * 2.0 ** -23


def bound(a, b, dtype):
    """Of |out - a b^T|, less the rounding of the result."""
    S = a.abs() @ b.abs().t()
    return S * lost(a.shape[1], dtype) + 1e-300


def near(out, ref, most, what=""):
    out = out.cpu().double()
    if out.numel() == 0:
        return
    most = most + (ROUNDED if what == "bf16" else 0.0) * ref.abs()
    over = (out - ref).abs() / most
    assert bool((over <= 1).all()), f"{what}: {float(over.max())} times the bound at {divmod(int(over.argmax()), out.shape[-1])}"


def check(out, a, b, dtype):
    near(out, a @ b.t(), bound(a, b, dtype), "bf16" if dtype == torch.bfloat16 else "f32")


# ---- the quantizer

@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", [(1, 1), (1, 128), (3, 127), (5, 129), (17, 640), (128, 128), (129, 257), (300, 1000), (2049, 391)])
def test_quantize(shape, dtype):
    x = tensor(torch.Generator().manual_seed(1), *shape, dtype=dtype)
    rows, cols = nv.fp8_quantize(x.cuda(), cols=True)
    same(rows, x.double())
    same(cols, x.double().t())
    alone, none = nv.fp8_quantize(x.cuda())
    assert none is None and torch.equal(alone.codes.view(torch.uint8), rows.codes.view(torch.uint8)) and torch.equal(alone.scales, rows.scales)
    none, alone = nv.fp8_quantize(x.cuda(), rows=False, cols=True)
    assert none is None and torch.equal(alone.codes.view(torch.uint8), cols.codes.view(torch.uint8)) and torch.equal(alone.scales, cols.scales)


def test_quantize_many_rows():
    # enough blocks for the kernel that keeps eight rows a group of lanes
    x = tensor(torch.Generator().manual_seed(2), 4099, 1030)
    same(nv.fp8_quantize(x.cuda())[0], x.double())


@pytest.mark.parametrize("dtype", DTYPES)
def test_quantize_rounding(dtype):
    # every bf16 magnitude of a few binades below a block's largest, which lies on and next to 448 * 2^e: ties and subnormal codes among them
    bits = torch.arange(0x3A00, 0x4400, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).double()
    rows = []
    for top in (448.0, 449.0 if dtype == torch.float32 else 450.0, 447.0 if dtype == torch.float32 else 446.0, 224.0, 256.0, 1.0, 2.0 ** -60):
        v = bits[bits <= top] if top >= 1 else bits[:500] * 2.0 ** -62
        v = v[v.abs() <= top]
        pad = -(-v.numel() // 127) * 127
        v = torch.cat([v, torch.zeros(pad - v.numel(), dtype=torch.float64)]).view(-1, 127)
        v[:, ::2] *= -1
        rows.append(torch.cat([v, torch.full((v.shape[0], 1), top, dtype=torch.float64)], 1))
    x = torch.cat(rows).to(dtype)
    same(nv.fp8_quantize(x.cuda())[0], x.double())
    same(nv.fp8_quantize(x.t().contiguous().cuda(), rows=False, cols=True)[1], x.double())


def test_quantize_extremes():
    # blocks of zeros, of the largest and of the smallest magnitudes; below 448 * 2^-127 the scale's exponent stays at its least
    x = torch.zeros(6, 128)
    x[1] = torch.finfo(torch.float32).max
    x[2] = torch.finfo(torch.float32).tiny
    x[3, 5] = -(2.0 ** -120)
    x[4] = 2.0 ** -149
    x[5] = -0.0
    q = nv.fp8_quantize(x.cuda())[0]
    assert q.scales[0].tolist()[0] == 0 and q.scales[0].tolist()[5] == 0
    codes, scales, _ = quantized(x.double())
    assert torch.equal(q.scales.cpu(), scales)
    assert torch.equal(q.codes.cpu().double()[:4], codes[:4])


@pytest.mark.parametrize("dtype", DTYPES)
def test_quantize_not_finite(dtype):
    # a block with an infinity or a NaN is NaN codes; its neighbours are as they were, and the product shows it in its row alone
    x = tensor(torch.Generator().manual_seed(3), 130, 300, dtype=dtype)
    clean = nv.fp8_quantize(x.cuda())[0]
    x[7, 140], x[9, 299], x[129, 0] = float("nan"), float("inf"), -float("inf")
    rows, cols = nv.fp8_quantize(x.cuda(), cols=True)
    for q in (rows, nv.fp8_quantize(x.cuda())[0]):
        got = q.codes.cpu().double()
        assert got[7, 128:256].isnan().all() and got[9, 256:300].isnan().all() and got[129, :128].isnan().all()
        ok = torch.ones(130, 3, dtype=torch.bool)
        ok[7, 1] = ok[9, 2] = ok[129, 0] = False
        assert torch.equal(got.view(130, 3, 128)[ok], clean.codes.cpu().double().view(130, 3, 128)[ok]) and torch.equal(q.scales.cpu().t()[ok], clean.scales.cpu().t()[ok])
    got = cols.codes.cpu().double().view(300, 2, 128).isnan().any(-1)
    assert got.nonzero().tolist() == [[0, 1], [140, 0], [299, 0]]
    w = nv.fp8_quantize(tensor(torch.Generator().manual_seed(4), 20, 300).cuda())[0]
    for out in DTYPES:
        bad = nv.fp8_gemm(rows, w, out_dtype=out).cpu().isnan()
        assert bad.all(1).nonzero().flatten().tolist() == [7, 9, 129] and int(bad.sum()) == 3 * 20


@pytest.mark.parametrize("dtype", DTYPES)
def test_quantize_strides(dtype):
    base = tensor(torch.Generator().manual_seed(5), 70, 403, dtype=dtype)
    for view in (base[:, 1:], base[3:, 2:300], base[::3, :129], base[:1, 5:], base[:, 7:8]):
        rows, cols = nv.fp8_quantize(view.cuda() if view.is_contiguous() else base.cuda().as_strided(view.shape, view.stride(), view.storage_offset()), cols=True)
        same(rows, view.double())
        same(cols, view.double().t())
    with pytest.raises(ValueError):
        nv.fp8_quantize(base.cuda().t())


def test_quantize_stack():
    # a stack of matrices: rows as one, columns each for itself
    x = tensor(torch.Generator().manual_seed(6), 3, 200, 150)
    rows, cols = nv.fp8_quantize(x.cuda(), cols=True)
    same(rows, x.double().reshape(600, 150))
    same(cols, x.double().transpose(1, 2).reshape(450, 200))
    with pytest.raises(ValueError):
        nv.fp8_quantize(x.cuda()[:, :100], cols=True)


def test_quantize_streaming_loads():
    # a tensor past the last cache level's size comes by another form of loads; its last rows as they are by themselves
    for dtype, sides in ((torch.bfloat16, dict(cols=True)), (torch.float32, {})):
        x = torch.empty((1 << 28) // (2 if dtype == torch.bfloat16 else 4) // 2048 + 128, 2048, dtype=dtype, device="cuda")
        x.normal_()
        rows, cols = nv.fp8_quantize(x, **sides)
        r, c = nv.fp8_quantize(x[-128:].contiguous(), **sides)
        assert torch.equal(rows.codes[-128:].view(torch.uint8), r.codes.view(torch.uint8)) and torch.equal(rows.scales[:, -128:], r.scales)
        if cols:
            assert torch.equal(cols.codes[:, -128:].view(torch.uint8), c.codes.view(torch.uint8)) and torch.equal(cols.scales[-1], c.scales[0])


# ---- products.  Sizes that reach: waves dividing the contraction (shapes of 1 to 4 fragments a side), tiles of 128 x 128, of 256 x 128, 192 and 256

SIZES = [(1, 1, 1), (1, 300, 128), (3, 5, 200), (16, 16, 128), (16, 4100, 640), (17, 33, 640), (33, 9000, 130), (64, 64, 2560), (65, 129, 1300), (100, 12300, 130),
         (300, 515, 1000), (1000, 2600, 100), (777, 4099, 384), (2000, 2100, 300), (2049, 4099, 130), (1100, 6000, 1100), (4096, 4096, 520)]


@pytest.mark.parametrize("dtype", DTYPES)
def test_groups_of_eight(dtype):
    # 2^16, -2^16 and one small product more, at each place of the block: binary32 outputs hold it, bf16 ones lose of it less than
    # 2^3 if it stands in one group of eight with the large ones, and nothing of a power of two down to 1 if not
    for p in (0, 5, 32, 100):
        a, b = torch.zeros(128, 128), torch.zeros(17, 128)
        a.fill_diagonal_(1.0)
        a[:, p], a[:, p + 1] = 256, -256
        b[:] = 2.0 ** (7 - torch.arange(9).repeat_interleave(2)[:17, None].float())
        b[1::2] *= 1.875
        b[:, p], b[:, p + 1] = 256, 256
        scales = torch.full((1, 128), 127, dtype=torch.uint8).cuda()
        q, r = (nv.Fp8(t.to(torch.float8_e4m3fn).cuda(), scales[:, : t.shape[0]].contiguous()) for t in (a, b))
        out, ref = nv.fp8_gemm(q, r, out_dtype=dtype).cpu().double(), a.double() @ b.double().t()
        here = torch.arange(128) // 8 == p // 8
        if dtype == torch.float32:
            assert torch.equal(out, ref)
        else:
            assert bool(((out - ref).abs()[here] < 8).all()) and torch.equal(out[~here][:, ::2], ref[~here][:, ::2])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M, N, K", SIZES)
def test_gemm(M, N, K, dtype):
    g = torch.Generator().manual_seed(M + N + K)
    a, b = (nv.fp8_quantize(tensor(g, n, K).cuda())[0] for n in (M, N))
    out = nv.fp8_gemm(a, b, out_dtype=dtype)
    A, B = values(a), values(b)
    if M * N > 1 << 20:  # rows and columns at the edges of tiles, and some others, of all of it on the GPU
        ref = values_on_gpu(a) @ values_on_gpu(b).t()
        S = values_on_gpu(a).abs() @ values_on_gpu(b).abs().t()
        most = S * lost(K + 32, dtype) + (0 if dtype == torch.float32 else ROUNDED) * ref.abs() + 1e-300
        assert bool(((out.double() - ref).abs() <= most).all())
    else:
        check(out, A, B, dtype)
    assert torch.equal(out, nv.fp8_gemm(a, b, out_dtype=dtype))  # the same bits again


def values_on_gpu(q):
    s = two_to(q.scales.t().long() - 127)
    return (q.codes.double().view(q.codes.shape[0], -1, 128) * s[..., None]).view(q.codes.shape)


def test_gemm_exact_integers():
    # small integers: every way of summing gives the same
    g = torch.Generator().manual_seed(8)
    for M, N, K in ((5, 7, 300), (130, 4200, 256), (2048, 2304, 256), (1000, 11000, 128)):
        x, w = (torch.randint(-4, 5, (n, K), generator=g).float().cuda() for n in (M, N))
        a, b = nv.fp8_quantize(x)[0], nv.fp8_quantize(w)[0]
        ref = x.double() @ w.double().t()
        assert torch.equal(nv.fp8_gemm(a, b, out_dtype=torch.float32).double(), ref)
        assert torch.equal(nv.fp8_gemm(a, b), ref.to(torch.bfloat16))


@pytest.mark.parametrize("dtype", DTYPES)
def test_gemm_output_pitch_and_empty(dtype):
    g = torch.Generator().manual_seed(9)
    for M, N in ((9, 21), (300, 4097), (2100, 2400)):
        a, b = (nv.fp8_quantize(tensor(g, n, 256).cuda())[0] for n in (M, N))
        base = torch.full((M + 1, N + 7), -7.0, dtype=dtype, device="cuda")
        nv.fp8_gemm(a, b, out=base[:M, 3: N + 3])
        assert torch.equal(base[:M, 3: N + 3], nv.fp8_gemm(a, b, out_dtype=dtype))
        assert bool((base[:, :3] == -7).all()) and bool((base[:, N + 3:] == -7).all()) and bool((base[M] == -7).all())
    empty = nv.Fp8(torch.empty(0, 256, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(2, 0, dtype=torch.uint8, device="cuda"))
    assert nv.fp8_gemm(empty, b, out_dtype=dtype).shape == (0, b.codes.shape[0])
    none = nv.Fp8(torch.empty(3, 0, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(0, 3, dtype=torch.uint8, device="cuda"))
    assert bool((nv.fp8_gemm(none, none, out_dtype=dtype) == 0).all())
    with pytest.raises(ValueError):
        nv.fp8_gemm(a, none)
    with pytest.raises(ValueError):
        nv.fp8_gemm(a, b, out=torch.empty(1, 1, device="cuda"))
    with pytest.raises(TypeError):
        nv.fp8_gemm(a, b, out_dtype=torch.float16)


@pytest.mark.parametrize("dtype", DTYPES)
def test_gemm_scales_at_any_byte(dtype):
    # few rows and odd numbers of them: scale bytes are read four at a time from any address, and not past the last
    g = torch.Generator().manual_seed(10)
    for M in (1, 2, 3, 5, 63, 66, 131):
        for N in (1, 2, 3, 67):
            for K in (100, 300):
                a, b = (nv.fp8_quantize(tensor(g, n, K).cuda())[0] for n in (M, N))
                check(nv.fp8_gemm(a, b, out_dtype=dtype), values(a), values(b), dtype)


def test_gemm_tiny_and_huge_scales():
    # scales multiply as exponents: results across the range of binary32, one side's least scale among them
    g = torch.Generator().manual_seed(11)
    for ea, eb in ((-110, 60), (100, -100), (-60, -60), (60, 50)):
        x, w = torch.randn(20, 128, generator=g, dtype=torch.float64) * 2.0 ** ea, torch.randn(24, 128, generator=g, dtype=torch.float64) * 2.0 ** eb
        a, b = nv.fp8_quantize(x.float().cuda())[0], nv.fp8_quantize(w.float().cuda())[0]
        for dtype in DTYPES:
            check(nv.fp8_gemm(a, b, out_dtype=dtype), values(a), values(b), dtype)


def test_offsets_past_32_bits():
    # operands and outputs of more than 2^32 bytes: the last rows
    a = nv.Fp8(torch.zeros(270000, 16384, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn), torch.full((128, 270000), 127, dtype=torch.uint8, device="cuda"))
    g = torch.Generator().manual_seed(12)
    tail, _ = nv.fp8_quantize(tensor(g, 500, 16384).cuda())
    a.codes[-500:] = tail.codes
    a.scales[:, -500:] = tail.scales
    b = nv.fp8_quantize(tensor(g, 40, 16384).cuda())[0]
    out = nv.fp8_gemm(a, b)
    near(out[-500:], values(tail) @ values(b).t(), bound(values(tail), values(b), torch.bfloat16), "bf16")
    assert bool((out[:-500] == 0).all())
    del a, out
    x = torch.zeros(270000, 8200, dtype=torch.bfloat16, device="cuda")
    x[-5:] = tensor(g, 5, 8200).cuda()
    q = nv.fp8_quantize(x)[0]
    same(nv.Fp8(q.codes[-5:], q.scales[:, -5:].contiguous()), x[-5:].cpu().double())
    assert int(q.codes[:-5].view(torch.uint8).max()) == 0
    del x, q
    a, b = (nv.fp8_quantize(tensor(g, n, 128).cuda())[0] for n in (270000, 8200))
    out = nv.fp8_gemm(a, b)
    last = values(nv.Fp8(a.codes[-100:], a.scales[:, -100:].contiguous()))
    near(out[-100:], last @ values(b).t(), bound(last, values(b), torch.bfloat16), "bf16")


def test_linear_gradients():
    # dX = dY W and dW = dY^T X of one layer, against the formula on the quantized operands and against differences of the layer itself.  The codes' error, 2^-4 / sqrt(12)
    # of an element at the most and 2.2e-2 of it in the mean square of a binade, on both sides: 3.2e-2 of the norm, six times that in any of some thousand elements
    g = torch.Generator().manual_seed(13)
    x, w, dy = tensor(g, 200, 300), tensor(g, 150, 300), tensor(g, 200, 150)
    X, W, D = (t.double() for t in (x, w, dy))
    xq, xc = nv.fp8_quantize(x.cuda(), cols=True)
    wq, wc = nv.fp8_quantize(w.cuda(), cols=True)
    dq, dc = nv.fp8_quantize(dy.cuda(), cols=True)
    for dtype in DTYPES:
        dx, dw = nv.fp8_gemm(dq, wc, out_dtype=dtype), nv.fp8_gemm(dc, xc, out_dtype=dtype)
        check(dx, quantized(D)[2], quantized(W.t())[2], dtype)
        check(dw, quantized(D.t())[2], quantized(X.t())[2], dtype)
        loss = lambda X, W: float((D * (X @ W.t())).sum())  # noqa: E731
        for got, at, size in ((dx, 0, X), (dw, 1, W)):
            rms = float(got.double().square().mean().sqrt())
            for i, j in torch.stack([torch.randint(0, n, (40,), generator=g) for n in size.shape], 1).tolist():
                h = torch.zeros_like(size)
                h[i, j] = 0.5
                args = [(X + s * h, W) if at == 0 else (X, W + s * h) for s in (1, -1)]
                assert abs(float(got[i, j]) - (loss(*args[0]) - loss(*args[1]))) <= 6 * 3.2e-2 * rms * max(1.0, abs(float(got[i, j])) / rms)


# ---- the experts' products

def routed(g, T, k, E, drop=0.0, only=None):
    ids = torch.topk(torch.randn(T, E, generator=g) + torch.randn(1, E, generator=g), k, dim=1).indices
    if only is not None:
        ids = torch.full_like(ids, only)
    ids = torch.where(torch.rand(T, k, generator=g) < drop, -1, ids)
    return nv.moe_sort(ids.cuda(), E), ids


EXPERTS = [(1, 1, 1, 8, 8, 0.0, None), (1, 2, 32, 40, 130, 0.0, None), (5, 2, 4, 40, 130, 0.3, None), (40, 4, 64, 100, 200, 0.0, None), (130, 1, 3, 64, 64, 1.0, None),
           (300, 2, 8, 515, 300, 0.1, None), (300, 2, 300, 33, 40, 0.1, None), (700, 1, 4, 260, 100, 0.0, 2), (1200, 3, 3, 300, 400, 0.0, None), (2000, 4, 8, 1051, 260, 0.1, None),
           (4096, 2, 5, 520, 300, 0.0, None)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T, k, E, N, K, drop, only", EXPERTS)
def test_experts(T, k, E, N, K, drop, only, dtype):
    """Forward product and both gradients, experts without a token, with one, with all of them, and dropped pairs, whose rows hold NaN."""
    g = torch.Generator().manual_seed(T + E)
    order, ids = routed(g, T, k, E, drop, only)
    R, off = T * k, order.offsets.tolist()
    x, w, dy = tensor(g, T, K), tensor(g, E, N, K), tensor(g, R, N)
    dy[off[-1]:] = float("nan")
    X = torch.zeros(R, K, dtype=torch.float64)
    picked = order.order[: off[-1]].cpu().long() // k
    X[: off[-1]] = x.double()[picked]
    a, a_cols = nv.fp8_quantize(x.cuda(), cols=True, order=order.order, top_k=k, offsets=order.offsets)
    b, b_cols = nv.fp8_quantize(w.cuda(), cols=True)
    d, d_cols = nv.fp8_quantize(dy.cuda(), cols=True, offsets=order.offsets)
    rows_alone = nv.fp8_quantize(x.cuda(), order=order.order, top_k=k)[0]
    same(rows_alone, X)
    assert torch.equal(rows_alone.codes[: off[-1]].view(torch.uint8), a.codes[: off[-1]].view(torch.uint8)) and torch.equal(rows_alone.scales[:, : off[-1]], a.scales[:, : off[-1]])
    y = nv.fp8_gemm_experts(a, b, order.offsets, out_dtype=dtype)
    dx = nv.fp8_gemm_experts(d, b_cols, order.offsets, out_dtype=dtype)
    dw = nv.fp8_gemm_experts_dw(d_cols, a_cols, order.offsets, out_dtype=dtype)
    assert bool((y[off[-1]:] == 0).all()) and bool((dx[off[-1]:] == 0).all())
    A, D = quantized(X)[2], quantized(torch.nan_to_num(dy.double()))[2]
    for e in range(E):
        s = slice(off[e], off[e + 1])
        if off[e] == off[e + 1]:
            assert bool((dw[e] == 0).all())
            continue
        W = w[e].double()
        check(y[s], A[s], quantized(W)[2], dtype)
        check(dx[s], D[s], quantized(W.t())[2], dtype)
        # blocks along the expert's own rows, from its first on
        check(dw[e], quantized(dy[s].double().t())[2], quantized(X[s].t())[2], dtype)
    assert torch.equal(dw, nv.fp8_gemm_experts_dw(d_cols, a_cols, order.offsets, out_dtype=dtype, rows=R))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M, N, K", [(1, 16384, 300), (9, 16001, 700), (16, 13000, 129), (3, 30000, 5000)])
def test_few_rows_of_many_columns(M, N, K, dtype):
    g = torch.Generator().manual_seed(M + N + K)
    a, b = (nv.fp8_quantize(tensor(g, n, K).cuda())[0] for n in (M, N))
    out = nv.fp8_gemm(a, b, out_dtype=dtype)
    A, B = values_on_gpu(a), values_on_gpu(b)
    ref = A @ B.t()
    most = A.abs() @ B.abs().t() * lost(A.shape[1], dtype) + (0 if dtype == torch.float32 else ROUNDED) * ref.abs() + 1e-300
    assert bool(((out.double() - ref).abs() <= most).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M, N, K", [(100, 4096, 11008), (257, 1000, 9001), (512, 3000, 6000), (777, 1025, 8192), (1000, 4096, 11008), (300, 129, 30000), (500, 200, 16257)])
def test_divided_contraction(M, N, K, dtype):
    # outputs of few tiles: with scratch memory their contraction is divided, without it is not; a pitched output, nothing beside it written
    g = torch.Generator().manual_seed(M + N + K)
    a, b = (nv.fp8_quantize(tensor(g, n, K).cuda())[0] for n in (M, N))
    A, B = values_on_gpu(a), values_on_gpu(b)
    ref = A @ B.t()
    # (16 parts at most: as many more roundings)
    most = A.abs() @ B.abs().t() * (lost(A.shape[1], dtype) + 16 * 2.0 ** -24) + (0 if dtype == torch.float32 else ROUNDED) * ref.abs() + 1e-300
    whole = torch.empty(M, N, dtype=dtype, device="cuda")
    P, tag = A.shape[1], 0 if dtype == torch.float32 else 1
    stream = torch.cuda.current_stream().cuda_stream
    assert nv.lib.nvfp4_fp8_gemm(M, N, P, a.codes.data_ptr(), a.scales.data_ptr(), b.codes.data_ptr(), b.scales.data_ptr(), whole.data_ptr(), tag, N, stream) == 0
    wide = torch.full((M + 2, N + 5), 7.0, dtype=dtype, device="cuda")
    out = nv.fp8_gemm(a, b, out=wide[1:-1, 3:3 + N])
    for got in (whole, out):
        assert bool(((got.double() - ref).abs() <= most).all())
    assert bool((wide[0] == 7).all()) and bool((wide[-1] == 7).all()) and bool((wide[:, :3] == 7).all()) and bool((wide[:, 3 + N:] == 7).all())
    assert torch.equal(out, nv.fp8_gemm(a, b, out_dtype=dtype))  # the same bits again
    need = nv.lib.nvfp4_fp8_gemm_workspace_bytes(M, N, P, tag)
    if need:  # too little of it is refused
        less = torch.empty(need - 1, dtype=torch.uint8, device="cuda")
        args = (M, N, P, a.codes.data_ptr(), a.scales.data_ptr(), b.codes.data_ptr(), b.scales.data_ptr(), whole.data_ptr(), tag, N)
        assert nv.lib.nvfp4_fp8_gemm_ws(*args, less.data_ptr(), need - 1, stream) == nv.lib.nvfp4_fp8_gemm_ws(*args, None, need, stream) != 0


@pytest.mark.parametrize("dtype", DTYPES)
def test_experts_large_tiles(dtype):
    # outputs of more tiles than CUs, uneven experts, weight gradients of many and of few tiles an expert
    g = torch.Generator().manual_seed(20)
    for T, k, E, N, K in ((3000, 2, 3, 2304, 640), (3000, 4, 20, 512, 512)):
        order, _ = routed(g, T, k, E, 0.05)
        off = order.offsets.tolist()
        a, a_cols = nv.fp8_quantize(tensor(g, T, K).cuda(), cols=True, order=order.order, top_k=k, offsets=order.offsets)
        b, _ = nv.fp8_quantize(tensor(g, E, N, K).cuda())
        _, d_cols = nv.fp8_quantize(tensor(g, T * k, N).cuda(), rows=False, cols=True, offsets=order.offsets)
        y, dw = nv.fp8_gemm_experts(a, b, order.offsets, out_dtype=dtype), nv.fp8_gemm_experts_dw(d_cols, a_cols, order.offsets, out_dtype=dtype)
        A, B, DC, AC = values_on_gpu(a), values_on_gpu(b).view(E, N, -1), values_on_gpu(d_cols), values_on_gpu(a_cols)
        for e in range(E):
            n, first = off[e + 1] - off[e], 128 * (off[e] // 128 + e)
            blocks = slice(first, first + -(-n // 128) * 128)
            for got, p, q in ((y[off[e]: off[e + 1]], A[off[e]: off[e + 1]], B[e]), (dw[e], DC[:, blocks], AC[:, blocks])):
                ref, S = p @ q.t(), p.abs() @ q.abs().t()
                most = S * lost(p.shape[1], dtype) + (0 if dtype == torch.float32 else ROUNDED) * ref.abs() + 1e-300
                assert bool(((got.double() - ref).abs() <= most).all()), e


def test_experts_refusals():
    order, _ = routed(torch.Generator().manual_seed(21), 10, 2, 4)
    x = torch.randn(10, 200, device="cuda")
    a, c = nv.fp8_quantize(x, cols=True, order=order.order, top_k=2, offsets=order.offsets)
    b = nv.fp8_quantize(torch.randn(4 * 7 + 1, 200, device="cuda"))[0]
    for bad in (lambda: nv.fp8_gemm_experts(a, b, order.offsets), lambda: nv.fp8_gemm_experts_dw(a, c, order.offsets), lambda: nv.fp8_gemm_experts_dw(c, c, order.offsets, rows=1000),
                lambda: nv.fp8_quantize(x, offsets=order.offsets), lambda: nv.fp8_quantize(x, rows=False), lambda: nv.fp8_quantize(x[None], order=order.order)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: nv.fp8_gemm_experts(a, b, order.offsets.long()), lambda: nv.fp8_quantize(x, order=order.order.long()), lambda: nv.fp8_quantize(x.half())):
        with pytest.raises(TypeError):
            bad()


def test_offsets_that_are_not_ascending():
    # whatever the offsets hold, rows and blocks stay inside their tensors: a call ends and what is beside its output is untouched
    g = torch.Generator().manual_seed(22)
    x = tensor(g, 300, 256).cuda()
    w = nv.fp8_quantize(tensor(g, 3, 200, 256).cuda())[0]
    for bad in ([0, 200, 100, 300], [-5, 1000, 2000, 1 << 30], [300, 200, 100, 0], [7, 7, 7, 7]):
        offsets = torch.tensor(bad, dtype=torch.int32, device="cuda")
        a, c = nv.fp8_quantize(x, cols=True, offsets=offsets)
        for dtype in DTYPES:
            assert nv.fp8_gemm_experts(nv.fp8_quantize(x)[0], w, offsets, out_dtype=dtype).shape == (300, 200)
    torch.cuda.synchronize()


# ---- streams, graphs

def step(x, w, ids, weights):
    order = nv.moe_sort(ids, w.shape[0])
    a, cols = nv.fp8_quantize(x, cols=True, order=order.order, top_k=ids.shape[1], offsets=order.offsets)
    y = nv.fp8_gemm_experts(a, nv.fp8_quantize(w)[0], order.offsets)
    out = nv.moe_combine(y, order.position, weights)
    dy, dweights = nv.moe_combine_bwd(out, y, weights, order.position, order.offsets)
    dw = nv.fp8_gemm_experts_dw(nv.fp8_quantize(dy, rows=False, cols=True, offsets=order.offsets)[1], cols, order.offsets)
    return out, dy, dweights, dw


def inputs(seed, T=600, k=2, E=6, N=300, K=260):
    g = torch.Generator().manual_seed(seed)
    return tensor(g, T, K).cuda(), tensor(g, E, N, K).cuda(), torch.topk(torch.randn(T, E, generator=g), k, 1).indices.cuda(), torch.rand(T, k, generator=g).cuda()


def test_other_stream():
    args = inputs(30)
    ref = step(*args)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        late = [a.clone() for a in args]
        got = step(*late)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(ref, got))


def test_graph():
    args = inputs(31)
    held = [a.clone() for a in args]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(*held)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(*held)
    for seed in (31, 32, 33):
        new = inputs(seed)
        for h, n in zip(held, new):
            h.copy_(n)
        graph.replay()
        ref = step(*new)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(ref, got)), seed


def test_graph_of_a_divided_contraction():
    # a product that brings its own scratch memory, on two streams and captured, replayed between eager calls with memory of their own
    g = torch.Generator().manual_seed(40)
    held = [tensor(g, 512, 8000).cuda(), tensor(g, 1000, 8000).cuda()]
    assert nv.lib.nvfp4_fp8_gemm_workspace_bytes(512, 1000, 8064, 1) > 0
    step = lambda x, w: nv.fp8_gemm(nv.fp8_quantize(x)[0], nv.fp8_quantize(w)[0])  # noqa: E731
    ref, side = step(*held), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step(*held)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert torch.equal(ref, got)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(*held)
    for _ in range(4):
        new = [tensor(g, 512, 8000).cuda(), tensor(g, 1000, 8000).cuda()]
        for h, n in zip(held, new):
            h.copy_(n)
        graph.replay()
        others = [torch.full((1 << 20,), float("nan"), device="cuda") for _ in range(8)]  # (what eager work allocates between)
        ref = step(*new)
        torch.cuda.synchronize()
        assert torch.equal(ref, got) and len(others) == 8


def test_example():
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "experts_training.py")
    spec = importlib.util.spec_from_file_location("experts_training", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    losses = module.train(steps=12, tokens=256, experts=4, width=128, hidden=256)
    assert all(b < a for a, b in zip(losses[::4], losses[4::4])) and losses[-1] < 0.9 * losses[0]
