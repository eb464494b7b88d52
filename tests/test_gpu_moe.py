"""Routing on the GPU against its definition in 64 bits: the sort (exactly), rows gathered, combined and the gradient of that.

Bounds: a combined element is a chain of top_k fused multiply-adds in binary32, top_k 2^-24 sum |w y|; dweights of D elements is a lane's chain of D / 64 (and up
to 8 elements a piece) and six additions across lanes, (D / 64 + 16) 2^-24 sum |dout y|; results add their own rounding, half of
their type's eps."""
import pytest
import torch

from paper_2505_19115_amd import binding as nv

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float32]
OWN = {t: torch.finfo(t).eps / 2 for t in DTYPES}


def sorted_by_hand(ids, E):
    flat = ids.reshape(-1).tolist()
    slots = [[] for _ in range(E)]
    for i, e in enumerate(flat):
        if 0 <= e < E:
            slots[e].append(i)
    offsets = [0]
    for s in slots:
        offsets.append(offsets[-1] + len(s))
    kept = [i for s in slots for i in s]
    position = [-1] * len(flat)
    for slot, i in enumerate(kept):
        position[i] = slot
    return offsets, kept + [-1] * (len(flat) - len(kept)), position


def drawn(g, T, k, E, kind):
    if kind == "even":
        return torch.randint(0, E, (T, k), generator=g)
    if kind == "one":
        return torch.full((T, k), E - 1)
    if kind == "none":
        return torch.where(torch.rand(T, k, generator=g) < 0.5, -1, E)
    ids = torch.randint(-2, E + 2, (T, k), generator=g)  # some outside
    ids[torch.rand(T, k, generator=g) < 0.5] = 0
    return ids


@pytest.mark.parametrize("dtype", [torch.int32, torch.int64])
@pytest.mark.parametrize("kind", ["even", "one", "none", "uneven"])
@pytest.mark.parametrize("T, k, E", [(1, 1, 1), (1, 8, 8), (7, 3, 5), (64, 1, 2), (65, 2, 512), (1023, 1, 7), (1024, 8, 64), (4097, 2, 3), (3000, 6, 200), (70001, 1, 33)])
def test_sort(T, k, E, kind, dtype):
    ids = drawn(torch.Generator().manual_seed(T + E), T, k, E, kind).to(dtype)
    got = nv.moe_sort(ids.cuda(), E)
    offsets, order, position = sorted_by_hand(ids, E)
    assert got.offsets.tolist() == offsets and got.order.tolist() == order and got.position.reshape(-1).tolist() == position
    assert got.position.shape == ids.shape and all(t.dtype == torch.int32 for t in got)


def test_sort_large():
    # more parts than one workgroup adds the counts of: each part grows
    g = torch.Generator(device="cuda").manual_seed(1)
    ids = torch.randint(0, 300, (1500001, 1), generator=g, device="cuda")
    got = nv.moe_sort(ids, 300)
    key, order = torch.sort(ids.view(-1), stable=True)
    assert torch.equal(got.order.long(), order) and torch.equal(got.position.view(-1).long()[order], torch.arange(1500001, device="cuda"))
    assert torch.equal(got.offsets.long(), torch.searchsorted(key, torch.arange(301, device="cuda")))


def test_sort_outside_numbers():
    # numbers whose low 32 bits are an expert's are not that expert
    ids = torch.tensor([[1 << 32, (1 << 32) + 1], [-(1 << 32), 1], [-(1 << 63), (1 << 63) - 1]])
    got = nv.moe_sort(ids.cuda(), 2)
    assert got.offsets.tolist() == [0, 0, 1] and got.position.tolist() == [[-1, -1], [-1, 0], [-1, -1]] and got.order.tolist() == [3, -1, -1, -1, -1, -1]


def test_sort_empty_and_refusals():
    got = nv.moe_sort(torch.empty(0, 4, dtype=torch.int64, device="cuda"), 5)
    assert got.offsets.tolist() == [0] * 6 and got.order.numel() == 0 and got.position.shape == (0, 4)
    ids = torch.zeros(4, 2, dtype=torch.int64, device="cuda")
    for groups in (0, -1, 513):
        with pytest.raises(nv.Nvfp4Error):
            nv.moe_sort(ids, groups)
    for bad in (ids.float(), ids.short(), ids.t()):
        with pytest.raises(TypeError):
            nv.moe_sort(bad, 3)


def case(seed, T, k, E, D, dtype, kind="uneven"):
    g = torch.Generator().manual_seed(seed)
    o = nv.moe_sort(drawn(g, T, k, E, kind).cuda(), E)
    x, y = torch.randn(T, D, generator=g).to(dtype), torch.randn(T * k, D, generator=g).to(dtype)
    y[int(o.offsets[-1]):] = float("nan")  # rows of no pair
    return o, x, y, torch.rand(T, k, generator=g)


SIZES = [(1, 1, 1, 1), (1, 2, 4, 4096), (7, 3, 5, 33), (20, 5, 3, 515), (64, 8, 9, 130), (50, 2, 3, 8200), (333, 4, 6, 1027), (1000, 1, 512, 64), (600, 7, 4, 512)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T, k, E, D", SIZES)
def test_gather(T, k, E, D, dtype):
    o, x, _, _ = case(2, T, k, E, D, dtype)
    order = o.order.cpu().long()
    ref = torch.where((order >= 0)[:, None], x[order.clamp(min=0) // k], torch.zeros((), dtype=dtype))
    assert torch.equal(nv.moe_gather(x.cuda(), o.order, k).cpu(), ref)
    wide = torch.randn(T, D + 5).to(dtype).cuda()
    assert torch.equal(nv.moe_gather(wide[:, 2: D + 2], o.order, k), nv.moe_gather(wide[:, 2: D + 2].contiguous(), o.order, k))


def test_gather_names_no_row():
    # an order may hold anything: what names no row of x is zeros
    x = torch.ones(3, 10, device="cuda")
    order = torch.tensor([0, 5, 6, -1, 1 << 30, -(1 << 31), 4], dtype=torch.int32, device="cuda")
    assert nv.moe_gather(x, order, 2)[:, 0].tolist() == [1, 1, 0, 0, 0, 0, 1]


@pytest.mark.parametrize("weighted", [True, False])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T, k, E, D", SIZES)
def test_combine(T, k, E, D, dtype, weighted):
    o, _, y, w = case(3, T, k, E, D, dtype)
    pos = o.position.cpu().long()
    rows = torch.where((pos >= 0)[..., None], y.double()[pos.clamp(min=0)], torch.zeros((), dtype=torch.float64)) * (w.double()[..., None] if weighted else 1.0)
    got = nv.moe_combine(y.cuda(), o.position, w.cuda() if weighted else None).cpu().double()
    ref = rows.sum(1)
    most = k * 2.0 ** -24 * rows.abs().sum(1) + OWN[dtype] * ref.abs() * (1 + 2.0 ** -6) + 1e-300
    assert bool(((got - ref).abs() <= most).all())
    assert bool((got[(pos < 0).all(1)] == 0).all())  # a token without a choice


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T, k, E, D", SIZES)
def test_combine_gradient(T, k, E, D, dtype):
    o, up, y, w = case(4, T, k, E, D, dtype)
    pos, kept = o.position.cpu().long(), int(o.offsets[-1])
    dy, dw = (t.cpu() for t in nv.moe_combine_bwd(up.cuda(), y.cuda(), w.cuda(), o.position, o.offsets))
    ref = torch.zeros(T * k, D, dtype=torch.float64)
    t = torch.arange(T).repeat_interleave(k).view(T, k)[pos >= 0]
    ref[pos[pos >= 0]] = up.double()[t] * w.double()[pos >= 0][:, None]
    assert bool(((dy.double() - ref).abs() <= OWN[dtype] * ref.abs() * (1 + 2.0 ** -6) + 2.0 ** -24 * ref.abs()).all()) and bool((dy[kept:] == 0).all())
    products = up.double()[:, None] * torch.where((pos >= 0)[..., None], y.double()[pos.clamp(min=0)], torch.zeros((), dtype=torch.float64))
    assert bool(((dw.double() - products.sum(-1)).abs() <= (D / 64 + 16) * 2.0 ** -24 * products.abs().sum(-1) + 1e-300).all())
    assert bool((dw[pos < 0] == 0).all())


def test_combine_gradient_by_differences():
    # the layer is linear in y and in the weights: its difference along a direction is the gradient's product with it, up to the binary32 roundings of both (of some
    # T * D outputs, each top_k 2^-24 of its terms)
    T, k, E, D = 200, 3, 5, 96
    o, up, y, w = case(5, T, k, E, D, torch.float32, "even")
    g = torch.Generator().manual_seed(6)
    dy, dw = nv.moe_combine_bwd(up.cuda(), y.cuda(), w.cuda(), o.position, o.offsets)
    f = lambda y, w: float((nv.moe_combine(y.cuda(), o.position, w.cuda()).double().cpu() * up.double()).sum())  # noqa: E731
    terms = float(up.abs().double().sum() * 8)
    for _ in range(4):
        v, u = torch.randn(y.shape, generator=g), torch.randn(w.shape, generator=g)
        assert abs((f(y + v, w) - f(y - v, w)) / 2 - float((dy.double().cpu() * v.double()).sum())) <= 16 * 2.0 ** -24 * terms
        assert abs((f(y, w + u) - f(y, w - u)) / 2 - float((dw.double().cpu() * u.double()).sum())) <= 16 * 2.0 ** -24 * terms


@pytest.mark.parametrize("dtype", DTYPES)
def test_streaming_loads(dtype):
    # rows of large tensors come by another form of loads, the results are the same bits as those of a piece by itself
    T, D = 3000, 8192 * 4 // (2 if dtype == torch.bfloat16 else 4)
    g = torch.Generator(device="cuda").manual_seed(7)
    for k in (1, 2):
        o = nv.moe_sort(torch.randint(-1, 4, (T, k), generator=g, device="cuda"), 4)
        x, y = (torch.randn(n, D, generator=g, device="cuda").to(dtype) for n in (T, T * k))
        w = torch.rand(T, k, generator=g, device="cuda")
        part = lambda t: t[:, :100].contiguous()  # noqa: E731
        assert torch.equal(part(nv.moe_gather(x, o.order, k)), nv.moe_gather(part(x), o.order, k))
        assert torch.equal(part(nv.moe_combine(y, o.position, w)), nv.moe_combine(part(y), o.position, w))
        dy, dw = nv.moe_combine_bwd(x, y, w, o.position, o.offsets)
        assert torch.equal(part(dy), nv.moe_combine_bwd(part(x), part(y), w, o.position, o.offsets)[0])
        rows = torch.where((o.position >= 0)[..., None], y.float()[o.position.clamp(min=0).long()], 0)
        ref, size = (x.double()[:, None] * rows).sum(-1), (x.double()[:, None] * rows).abs().sum(-1)
        assert bool(((dw.double() - ref).abs() <= (D / 64 + 16) * 2.0 ** -24 * size).all())


def test_refusals():
    o, x, y, w = case(8, 10, 2, 3, 16, torch.float32, "even")
    x, y, w = x.cuda(), y.cuda(), w.cuda()
    for bad in (lambda: nv.moe_gather(x.t(), o.order, 2), lambda: nv.moe_combine(y[:, ::2], o.position, w), lambda: nv.moe_combine(y, o.position[0]),
                lambda: nv.moe_combine_bwd(x[:5], y, w, o.position, o.offsets), lambda: nv.moe_combine_bwd(x.bfloat16(), y, w, o.position, o.offsets)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: nv.moe_gather(x, o.order.long(), 2), lambda: nv.moe_combine(y, o.position, w.double()), lambda: nv.moe_combine(y, o.position, w[:, :1]),
                lambda: nv.moe_combine(y.half(), o.position, w), lambda: nv.moe_combine_bwd(x, y, w, o.position, o.offsets.long())):
        with pytest.raises(TypeError):
            bad()
    with pytest.raises(nv.Nvfp4Error):
        nv.moe_gather(x, o.order, 0)
    assert nv.moe_combine(y[:, :0].contiguous(), o.position, w).shape == (10, 0)
    assert nv.moe_gather(x, o.order[:0], 2).shape == (0, 16)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [2, 3, 4, 5, 7, 8, 9, 15, 63, 64, 65, 127, 128, 129, 131, 255, 256, 257, 263, 511, 512, 513, 519, 1023, 1025])
def test_widths(D, dtype):
    # rows by 8, 16, 32 and 64 lanes, with and without a last piece that overlaps the one before; a lane adds at most 16 products of a row at a time, 64 lanes 6 sums
    T, k, E = 37, 3, 4
    o, x, y, w = case(8, T, k, E, D, dtype)
    order, pos, kept = o.order.cpu().long(), o.position.cpu().long(), int(o.offsets[-1])
    ref = torch.where((order >= 0)[:, None], x[order.clamp(min=0) // k], torch.zeros((), dtype=dtype))
    assert torch.equal(nv.moe_gather(x.cuda(), o.order, k).cpu(), ref)
    rows = torch.where((pos >= 0)[..., None], y.double()[pos.clamp(min=0)], torch.zeros((), dtype=torch.float64))
    got, ref = nv.moe_combine(y.cuda(), o.position, w.cuda()).cpu().double(), (rows * w.double()[..., None]).sum(1)
    assert bool(((got - ref).abs() <= k * 2.0 ** -24 * (rows * w.double()[..., None]).abs().sum(1) + OWN[dtype] * ref.abs() * (1 + 2.0 ** -6) + 1e-300).all())
    dy, dw = (t.cpu() for t in nv.moe_combine_bwd(x.cuda(), y.cuda(), w.cuda(), o.position, o.offsets))
    ref = torch.zeros(T * k, D, dtype=torch.float64)
    t = torch.arange(T).repeat_interleave(k).view(T, k)[pos >= 0]
    ref[pos[pos >= 0]] = x.double()[t] * w.double()[pos >= 0][:, None]
    assert bool(((dy.double() - ref).abs() <= (OWN[dtype] * (1 + 2.0 ** -6) + 2.0 ** -24) * ref.abs()).all()) and bool((dy[kept:] == 0).all())
    products = x.double()[:, None] * rows
    assert bool(((dw.double() - products.sum(-1)).abs() <= (D / 64 + 22) * 2.0 ** -24 * products.abs().sum(-1) + 1e-300).all())
