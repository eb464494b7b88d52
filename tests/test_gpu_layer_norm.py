"""Rows' norms on the GPU against their formulas in 64 bits.

Bounds, u = 2^-24.  A sum over a row is a chain of at most C = 64 additions in a thread, 6 across lanes and 16 across waves (rows past the registers: cols / 1024 + 8 in a
thread).  The mean is off by M = u (C + 23) mean|x|; r relatively by u (C + 26) / 2 + (M r)^2 / 2 + 3 u; y by |w h| (that + 4 u) + |w| r M + 2 u (|y| + |b|) and half of its type's eps.
dx, from given statistics: u (C + 36) r (|u| + mean|u| + |h| mean|u h|) and its rounding.  Sums over rows: chains of at most 100 + rows / 10."""
import pytest
import torch

from paper_2505_19115_amd import binding as nv

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DTYPES = [torch.bfloat16, torch.float32]
HALF = {t: torch.finfo(t).eps / 2 for t in DTYPES}
# widths around those where the kernels change (pieces of 8 bf16 or 4 binary32 elements, 8 .. 1024 threads), odd ones, and beyond the registers of a workgroup
WIDTHS = [1, 2, 7, 8, 9, 31, 32, 33, 63, 64, 65, 96, 127, 128, 129, 255, 257, 511, 512, 513, 1000, 1023, 1025, 2047, 2049, 2785, 4096, 4097, 8191, 8200, 11008, 16384, 16391, 20001, 32769]


def rows_of(cols):
    return 37 if cols <= 600 else 5


def inputs(R, D, dtype, wdt, seed=0, pad=0, shift=0.0):
    g = torch.Generator().manual_seed(seed + D)
    x = (torch.randn(R, D + pad, generator=g) * torch.rand(R, 1, generator=g).mul(4).exp() + shift).to(dtype)[:, :D]
    w = None if wdt is None else (1 + 0.3 * torch.randn(D, generator=g)).to(wdt)
    b = None if wdt is None else torch.randn(D, generator=g).to(wdt)
    return x, w, b


def norm64(x, w, b, eps, center):
    x = x.double()
    D = x.shape[1]
    m = x.mean(1, keepdim=True) if center else torch.zeros(x.shape[0], 1, dtype=torch.float64)
    r = 1 / ((x - m).square().mean(1, keepdim=True) + eps).sqrt()
    h = (x - m) * r
    wd, bd = (torch.ones(D, dtype=torch.float64) if w is None else w.double()), (torch.zeros(D, dtype=torch.float64) if b is None else b.double())
    y = h * wd + bd
    C = 64 if D <= 16384 else D / 1024 + 8
    M = U * (C + 23) * x.abs().mean(1, keepdim=True) if center else 0 * r
    rel = U * (C + 26) / 2 + (M * r) ** 2 / 2 + 3 * U
    bound = (wd * h).abs() * (rel + 4 * U) + wd.abs() * r * M + 2 * U * (y.abs() + bd.abs()) + HALF[torch.float32] * 0
    return y, m[:, 0], r[:, 0], bound, M[:, 0], rel[:, 0]


@pytest.mark.parametrize("center", [True, False])
@pytest.mark.parametrize("wdt", [None, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", WIDTHS)
def test_forward(D, dtype, wdt, center):
    x, w, b = inputs(rows_of(D), D, dtype, wdt)
    cuda = lambda t: t if t is None else t.cuda()  # noqa: E731
    got = nv.layer_norm(x.cuda(), cuda(w), cuda(b), eps=1e-5, center=center)
    y, m, r, bound, M, rel = norm64(x, w, b, 1e-5, center)
    assert got.y.dtype == dtype and (got.mean is None) == (not center)
    assert ((got.y.cpu().double() - y).abs() <= bound + HALF[dtype] * y.abs() * (1 + 2 ** -7) + 2.0 ** -130).all()
    if center:
        assert ((got.mean.cpu().double() - m).abs() <= M + U * m.abs()).all()
    assert ((got.rstd.cpu().double() / r - 1).abs() <= rel + U).all()


@pytest.mark.parametrize("which", ["weight", "bias"])
@pytest.mark.parametrize("dtype", DTYPES)
def test_only_weight_or_bias(dtype, which):
    x, w, b = inputs(9, 200, dtype, torch.float32)
    w, b = (w, None) if which == "weight" else (None, b)
    got = nv.layer_norm(x.cuda(), None if w is None else w.cuda(), None if b is None else b.cuda())
    y, _, _, bound, _, _ = norm64(x, w, b, 1e-5, True)
    assert ((got.y.cpu().double() - y).abs() <= bound + HALF[dtype] * y.abs() * (1 + 2 ** -7)).all()


@pytest.mark.parametrize("D", [100, 4096, 20001])
def test_far_from_zero(D):
    # a mean a thousand times the deviations: statistics come from deviations, not from a difference of sums of squares (which would leave nothing)
    g = torch.Generator().manual_seed(D)
    x = torch.randn(4, D, generator=g) + 1000
    got = nv.layer_norm(x.cuda())
    y, _, _, bound, _, _ = norm64(x, None, None, 1e-5, True)
    assert ((got.y.cpu().double() - y).abs() <= bound + U * y.abs()).all()
    assert (got.y.cpu().double() - y).abs().max() < 2e-3


@pytest.mark.parametrize("offset, pad", [(0, 1), (1, 2), (3, 64), (5, 3)])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [33, 777, 5000, 17000])
def test_views(D, dtype, offset, pad):
    # rows of a larger pitch from any element on, NaN between them; the same bits as dense rows
    R = 7
    base = torch.full((R, offset + D + pad), float("nan"), dtype=dtype, device="cuda")
    dbase = torch.full((R, D + offset + pad + 1), float("nan"), dtype=dtype, device="cuda")
    x, w, b = inputs(R, D, dtype, torch.float32)
    dy = torch.randn(R, D, generator=torch.Generator().manual_seed(1)).to(dtype).cuda()
    view, dview = base[:, offset: offset + D], dbase[:, 1 + offset: 1 + offset + D]
    view.copy_(x)
    dview.copy_(dy)
    x, w, b = x.cuda(), w.cuda(), b.cuda()
    a, c = nv.layer_norm(view, w, b), nv.layer_norm(x, w, b)
    assert all(torch.equal(s, t) for s, t in zip(a, c))
    a, c = nv.layer_norm_bwd(dview, view, w, a.mean, a.rstd, bias=True), nv.layer_norm_bwd(dy, x, w, c.mean, c.rstd, bias=True)
    assert all(torch.equal(s, t) for s, t in zip(a, c))


def grads64(dy, x, w, mean, rstd):
    dy, x, r = dy.double(), x.double(), rstd.double()[:, None]
    h = (x - (0 if mean is None else mean.double()[:, None])) * r
    u = dy * (1 if w is None else w.double())
    mu, mh = u.mean(1, keepdim=True) if mean is not None else torch.zeros_like(r), (u * h).mean(1, keepdim=True)
    size = r * (u.abs() + (u.abs().mean(1, keepdim=True) if mean is not None else 0) + h.abs() * (u * h).abs().mean(1, keepdim=True))
    return r * (u - mu - h * mh), size, (dy * h).sum(0), (dy * h).abs().sum(0), dy.sum(0), dy.abs().sum(0)


def check_grads(got, dy, x, w, mean, rstd, dtype):
    dx, size, dw, dw_size, db, db_size = grads64(dy, x, w, mean, rstd)
    R, D = x.shape
    C = 64 if D <= 16384 else D / 1024 + 8
    assert ((got.dx.cpu().double() - dx).abs() <= U * (C + 36) * size + HALF[dtype] * dx.abs() * (1 + 2 ** -7) + 2.0 ** -130).all()
    chain = U * (100 + R / 10 + 4)
    for g, v, s in ((got.dweight, dw, dw_size), (got.dbias, db, db_size)):
        if g is not None:
            assert ((g.cpu().double() - v).abs() <= chain * s + HALF[g.dtype] * v.abs() * (1 + 2 ** -7) + 2.0 ** -130).all()


@pytest.mark.parametrize("center", [True, False])
@pytest.mark.parametrize("wdt", [None, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", WIDTHS)
def test_backward(D, dtype, wdt, center):
    R = rows_of(D)
    x, w, _ = inputs(R, D, dtype, wdt)
    dy = torch.randn(R, D, generator=torch.Generator().manual_seed(D + 1)).to(dtype)
    wg = w if w is None else w.cuda()
    stats = nv.layer_norm(x.cuda(), wg, center=center)
    got = nv.layer_norm_bwd(dy.cuda(), x.cuda(), wg, stats.mean, stats.rstd, bias=center)
    assert got.dx.dtype == dtype and (got.dweight is None) == (w is None) and (got.dbias is None) == (not center)
    check_grads(got, dy, x, w, stats.mean.cpu() if center else None, stats.rstd.cpu(), dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("R, D", [(1, 64), (2, 4096), (3, 16384), (511, 300), (4099, 40), (5000, 512), (3001, 1030), (1300, 4096), (700, 8192), (600, 16384), (40, 17000)])
def test_backward_many_rows(R, D, dtype):
    # rows that leave a workgroup's teams and the last round of workgroups half empty
    x, w, _ = inputs(R, D, dtype, torch.float32, seed=3)
    dy = torch.randn(R, D, generator=torch.Generator().manual_seed(D + R)).to(dtype)
    stats = nv.layer_norm(x.cuda(), w.cuda())
    got = nv.layer_norm_bwd(dy.cuda(), x.cuda(), w.cuda(), stats.mean, stats.rstd, bias=True)
    check_grads(got, dy, x, w, stats.mean.cpu(), stats.rstd.cpu(), dtype)
    again = nv.layer_norm_bwd(dy.cuda(), x.cuda(), w.cuda(), stats.mean, stats.rstd, bias=True)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


@pytest.mark.parametrize("center", [True, False])
def test_gradient_against_differences(center):
    # central differences with step h: the truncation is h^2 / 6 times third derivatives (below 40 in these rows of size 1), the calls' own error 60 u |y| sqrt(D) / h
    R, D, h = 3, 11, 2.0 ** -7
    g = torch.Generator().manual_seed(0)
    x, w, b, dy = torch.randn(R, D, generator=g), 1 + 0.3 * torch.randn(D, generator=g), torch.randn(D, generator=g), torch.randn(R, D, generator=g)

    def total(x, w, b):
        return float((nv.layer_norm(x.cuda(), w.cuda(), b.cuda(), center=center).y.cpu().double() * dy.double()).sum())

    stats = nv.layer_norm(x.cuda(), w.cuda(), b.cuda(), center=center)
    got = nv.layer_norm_bwd(dy.cuda(), x.cuda(), w.cuda(), stats.mean, stats.rstd, bias=True)
    for which, grad in ((0, got.dx), (1, got.dweight), (2, got.dbias)):
        flat = grad.cpu().reshape(-1)
        for i in range(flat.numel()):
            args = [[x, w, b], [x, w, b]]
            for side, sign in ((0, 1), (1, -1)):
                t = args[side][which].clone()
                t.view(-1)[i] += sign * h
                args[side][which] = t
            diff = (total(*args[0]) - total(*args[1])) / (2 * h)
            assert abs(diff - float(flat[i])) <= h * h * 40 / 6 + 60 * U * 10 / h


def test_special_rows():
    # constant rows (variance 0), zeros, infinities and NaN stay in their rows; a row that overflows to an infinite sum of squares gives zeros times the weight
    x = torch.zeros(6, 300)
    x[1] = 5
    x[2, 7] = float("inf")
    x[3, 299] = float("nan")
    x[4] = torch.randn(300, generator=torch.Generator().manual_seed(0))
    x[5] = 1e25
    for center in (True, False):
        got = nv.layer_norm(x.cuda(), center=center)
        assert not got.y[0].any() and torch.isnan(got.y[2]).any() and torch.isnan(got.y[3]).all()
        assert torch.isfinite(got.y[4]).all()
        if center:
            assert not got.y[1].any() and got.mean[1] == 5 and abs(float(got.rstd[1]) - 1e-5 ** -0.5) <= 1e-4
        y = norm64(x[4:5], None, None, 1e-5, center)
        assert ((got.y[4:5].cpu().double() - y[0]).abs() <= y[3] + U * y[0].abs()).all()
    d = nv.layer_norm_bwd(torch.ones(6, 300, device="cuda"), x.cuda(), None, got.mean, got.rstd)
    assert torch.isfinite(d.dx[4]).all() and torch.isnan(d.dx[3]).any()


def test_no_rows_and_refusals():
    x = torch.randn(4, 32, device="cuda")
    w = torch.ones(32, device="cuda")
    none = nv.layer_norm(x[:0], w)
    assert none.y.shape == (0, 32) and none.rstd.shape == (0,)
    got = nv.layer_norm_bwd(x[:0], x[:0], w, none.mean, none.rstd, bias=True)
    assert got.dx.shape == (0, 32) and not got.dweight.any() and not got.dbias.any()  # the sums of no rows
    assert nv.layer_norm(x[:, :0]).y.shape == (4, 0)
    for eps in (-1e-5, float("nan"), float("inf")):
        with pytest.raises(nv.Nvfp4Error):
            nv.layer_norm(x, eps=eps)
    with pytest.raises(TypeError):
        nv.layer_norm(x.half())
    with pytest.raises(TypeError):
        nv.layer_norm(x, w, w.bfloat16())
    for bad in (x.t(), x[:1].expand(4, 32), x[0], x.cpu()):
        with pytest.raises(ValueError):
            nv.layer_norm(bad)
    for bad in (w[:31], w[None], torch.ones(64, device="cuda")[::2]):
        with pytest.raises(ValueError):
            nv.layer_norm(x, bad)
    s = nv.layer_norm(x, w)
    for dy in (x[:3], x.bfloat16()):
        with pytest.raises(ValueError):
            nv.layer_norm_bwd(dy, x, w, s.mean, s.rstd)
    with pytest.raises(TypeError):
        nv.layer_norm_bwd(x, x, w, s.mean[:3], s.rstd)
    with pytest.raises(TypeError):
        nv.layer_norm_bwd(x, x, w, s.mean, s.rstd.double())


@pytest.mark.parametrize("center", [True, False])
@pytest.mark.parametrize("dtype", DTYPES)
def test_statistics_of_rows_without_columns(dtype, center):
    # a mean of nothing is 0 / 0, and so is what follows from it; never what the memory held before
    for R in (1, 5, 300):
        torch.full((4, R), 7.0, device="cuda")  # (freed at once: the next tensors of this size are made of it)
        got = nv.layer_norm(torch.empty(R, 0, dtype=dtype, device="cuda"), center=center)
        assert got.y.shape == (R, 0) and torch.isnan(got.rstd).all() and (torch.isnan(got.mean).all() if center else got.mean is None)
        grads = nv.layer_norm_bwd(got.y, got.y, torch.empty(0, device="cuda"), got.mean, got.rstd, bias=True)
        assert grads.dx.shape == (R, 0) and grads.dweight.shape == grads.dbias.shape == (0,)


@pytest.mark.parametrize("center", [True, False])
@pytest.mark.parametrize("D, R", [(16391, 4096), (65537, 8192), (262147, 2048)])
def test_column_sums_of_long_rows(D, R, center):
    # numbers of one sign, where every rounding of a chain of additions may fall the same way.  A term dy (x - m) r is off by 3 u, its column's sums inside a thread by 2 u (they carry what
    # their roundings leave), the 16 at most of a column's workgroups by 16 u, the result by u
    x = torch.rand(R, D, generator=torch.Generator(device="cuda").manual_seed(D), device="cuda") + 0.5
    dy = torch.full((R, D), 0.1, device="cuda")
    m, r = torch.full((R,), -0.25, device="cuda"), torch.full((R,), 0.7, device="cuda")
    got = nv.layer_norm_bwd(dy, x, torch.ones(D, device="cuda"), m if center else None, r, bias=True)
    db = float(dy[0, 0].double()) * R
    assert ((got.dbias.double() / db - 1).abs() <= 19 * U).all()
    dw = torch.zeros(D, dtype=torch.float64, device="cuda")
    for part in x.split(256):
        dw += (part.double() - (m[0].double() if center else 0)).mul_(r[0].double() * dy[0, 0].double()).sum(0)
    assert ((got.dweight.double() / dw - 1).abs() <= 22 * U).all()


def test_column_sums_of_long_rows_keep_infinities():
    D, R = 16391, 300
    x, dy = torch.ones(R, D, device="cuda"), torch.ones(R, D, device="cuda")
    dy[7, 5], dy[8, 6], dy[9, 6], dy[100, 16390] = float("inf"), float("inf"), -float("inf"), -float("inf")
    dy[40, 9] = dy[200, 9] = dy[40, 10] = dy[41, 10] = 3e38
    got = nv.layer_norm_bwd(dy, x, torch.ones(D, device="cuda"), None, torch.ones(R, device="cuda"), bias=True)
    for v in (got.dweight, got.dbias):
        assert v[5] == float("inf") and torch.isnan(v[6]) and v[16390] == -float("inf") and v[9] == v[10] == float("inf")
        v[[5, 6, 9, 10, 16390]] = R
        assert (v == R).all()


@pytest.mark.parametrize("center", [True, False])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("R, D", [(1024, 2056), (1025, 1030), (1025, 1537), (1027, 2048), (1025, 2049), (1030, 3333), (1026, 4096), (1100, 4104), (4099, 40), (1031, 12000)])
def test_forward_many_rows(R, D, dtype, center):
    # many rows, and some that leave the last workgroup half empty
    x, w, b = inputs(R, D, dtype, torch.float32, seed=2)
    got = nv.layer_norm(x.cuda(), w.cuda(), b.cuda(), center=center)
    y, m, r, bound, M, rel = norm64(x, w, b, 1e-5, center)
    assert ((got.y.cpu().double() - y).abs() <= bound + HALF[dtype] * y.abs() * (1 + 2 ** -7) + 2.0 ** -130).all()
    if center:
        assert ((got.mean.cpu().double() - m).abs() <= M + U * m.abs()).all()
    assert ((got.rstd.cpu().double() / r - 1).abs() <= rel + U).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [96, 1030, 1537, 2048, 2049, 3333, 4096, 4104, 9000])
def test_a_row_alone(D, dtype):
    # how many rows there are does not change a row's result
    x, w, b = (t.cuda() for t in inputs(1100, D, dtype, torch.float32, seed=4))
    many, few = nv.layer_norm(x, w, b), nv.layer_norm(x[:5], w, b)
    assert all(torch.equal(m[:5], f) for m, f in zip(many, few))
