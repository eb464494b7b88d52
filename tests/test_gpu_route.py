"""The experts' router on the GPU against its formulas in 64 bits: choice, weights, balance, gradient.

Bounds, u = 2^-24.  A share exp(l - top) / sum: the difference rounds by u |l - top|, expf is off by 2 u, the sum of S + 6 additions adds (S + 6) u and the same of its
terms, the quotient u: relative error u (2 D + S + 12) with D the largest |l - top| among terms that count, S = 8 for a row (8 entries a lane) and k for the chosen.
Sums over tokens add at most 300 additions in a row (rows of a lane group, lanes, waves, parts).  Results add half of their type's eps."""
import math

import pytest
import torch

from paper_2505_19115_amd import binding as nv

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DTYPES = [torch.bfloat16, torch.float32]
SIZES = [(1, 1, 1), (1, 8, 2), (3, 8, 8), (5, 9, 4), (64, 16, 2), (65, 17, 17), (130, 61, 4), (33, 64, 6), (257, 65, 3), (100, 128, 8), (31, 200, 5), (17, 256, 1), (9, 257, 8), (6, 512, 512), (2000, 8, 2)]
MASKS = ["none", "some", "lowest", "rows", "all"]


def drawn(seed, T, E, dtype, mask, pad=0):
    """Logits with ties; some at -inf, at the type's lowest value, whole rows, or all of them."""
    g = torch.Generator().manual_seed(seed)
    l = torch.randn(T, E + pad, generator=g, dtype=torch.float64).mul(3).mul(8).round().div(8).to(dtype)
    if mask == "some":
        l[torch.rand(T, E + pad, generator=g) < 0.4] = -math.inf
    elif mask == "lowest":
        l[torch.rand(T, E + pad, generator=g) < 0.4] = torch.finfo(dtype).min
    elif mask == "rows":
        l[torch.rand(T, generator=g) < 0.4] = -math.inf
        l[0] = -math.inf
    elif mask == "all":
        l[:] = -math.inf
    return l


def chosen_by_hand(l, k):
    """The k largest of each row, of equal ones the lowest index; -1 where -inf is left."""
    out = []
    for row in l.double().tolist():
        order = sorted(range(len(row)), key=lambda e: (-row[e], e))[:k]
        out.append([e if row[e] > -math.inf else -1 for e in order])
    return torch.tensor(out, dtype=torch.int32).view(l.shape[0], k)


def shares(l, mask=None):
    """Softmax over the entries of the mask in 64 bits (zeros for rows without any), lse (0 then), and the largest distance from the top that counts."""
    l = l.double()
    if mask is not None:
        l = torch.where(mask, l, -math.inf)
    top = l.max(1, keepdim=True).values
    there = top > -math.inf
    d = torch.where(there, l - torch.where(there, top, 0), -math.inf)
    e = d.exp()
    s = e.sum(1, keepdim=True)
    far = torch.where(d > -110, -d, 0).max(1, keepdim=True).values
    return torch.where(there, e / torch.where(there, s, 1), 0), torch.where(there, s.clamp(min=1e-300).log() + torch.where(there, top, 0), 0), far, there


def picked(experts, E):
    m = torch.zeros(experts.shape[0], E + 1, dtype=torch.bool)
    m.scatter_(1, torch.where(experts < 0, E, experts).long(), True)
    return m[:, :E]


def share_bound(far, terms):
    return U * (2 * far + terms + 12)


@pytest.mark.parametrize("renormalize", [True, False])
@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T, E, k", SIZES)
def test_route(T, E, k, dtype, mask, renormalize):
    l = drawn(T + E, T, E, dtype, mask)
    got = nv.moe_route(l.cuda(), k, renormalize=renormalize)
    experts = chosen_by_hand(l, k)
    assert got.experts.dtype == torch.int32 and torch.equal(got.experts.cpu(), experts)
    p, _, far, _ = shares(l, picked(experts, E) if renormalize else None)
    want = torch.where(experts < 0, 0, p.gather(1, experts.clamp(min=0).long()))
    err = (got.weights.cpu().double() - want).abs()
    assert (err <= share_bound(far, k if renormalize else 8) * want + 2.0 ** -148).all()
    if renormalize and mask == "none":
        assert (got.weights.sum(1) - 1).abs().max() <= U * (2 * k + 4)


@pytest.mark.parametrize("pad", [1, 3, 8])
@pytest.mark.parametrize("dtype", DTYPES)
def test_route_view(dtype, pad):
    # rows of a larger pitch, from an odd element on: neighbours in the memory are infinities that nobody may take
    base = torch.full((40, 61 + pad + 1), math.inf, dtype=dtype, device="cuda")
    l = drawn(3, 40, 61, dtype, "some").cuda()
    view = base[:, 1: 62]
    view.copy_(l)
    a, b = nv.moe_route(view, 5), nv.moe_route(l, 5)
    assert torch.equal(a.experts, b.experts) and torch.equal(a.weights, b.weights)
    x, y = nv.moe_balance(view, a.experts), nv.moe_balance(l, a.experts)
    assert all(torch.equal(s, t) for s, t in zip(x, y))
    d = torch.randn(40, 5, device="cuda")
    assert torch.equal(nv.moe_route_bwd(view, a.experts, d, counts=x.counts, dlosses=x.losses), nv.moe_route_bwd(l, a.experts, d, counts=x.counts, dlosses=x.losses))


def test_route_special_values():
    inf, nan = math.inf, math.nan
    l = torch.tensor([[0.0, -0.0, -1.0, 0.0], [1.0, nan, 2.0, nan], [inf, 1.0, inf, -inf], [-inf, -inf, -3e38, -inf], [1e-45, 0.0, -1e-45, 2e-45], [3e38, -3e38, 3e38, 0.0]])
    got = nv.moe_route(l.cuda(), 3)
    # (1e-45 and 2e-45 are the same number in binary32, the smallest, and above zero)
    assert got.experts.tolist() == [[0, 1, 3], [1, 3, 2], [0, 2, 1], [2, -1, -1], [0, 3, 1], [0, 2, 3]]
    w = got.weights.cpu()
    assert torch.isnan(w[1]).all() and torch.isnan(w[2]).any()
    assert w[3].tolist() == [1, 0, 0] and w[5].tolist() == [0.5, 0.5, 0]
    assert (w[0] - 1 / 3).abs().max() <= 2 * U and (w[4] - 1 / 3).abs().max() <= 2 * U
    d = nv.moe_route_bwd(l.cuda(), got.experts, torch.ones(6, 3, device="cuda"))
    assert torch.isnan(d[1, [1, 2, 3]]).all() and d[3].tolist() == [0, 0, 0, 0] and not torch.isnan(d[5]).any()


@pytest.mark.parametrize("ids", [torch.int32, torch.int64])
@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T, E, k", SIZES + [(5000, 40, 3), (3000, 500, 2)])
def test_balance(T, E, k, dtype, mask, ids):
    l = drawn(T * 7 + E, T, E, dtype, mask)
    experts = torch.randint(-2, E + 2, (T, k), generator=torch.Generator().manual_seed(T)).to(ids)
    got = nv.moe_balance(l.cuda(), experts.cuda())
    p, lse, far, there = shares(l)
    n = int(there.sum())
    inside = experts[(experts >= 0) & (experts < E)].long()
    counts = torch.bincount(inside, minlength=E)
    assert got.counts.dtype == torch.int32 and torch.equal(got.counts.cpu().long(), torch.cat([counts, torch.tensor([n])]))
    if n == 0:
        assert not got.losses.any() and not got.probs.any()
        return
    mean = p.sum(0) / n
    bound = (share_bound(far, 8) * p).sum(0) / n + 302 * U * mean + 2.0 ** -140
    assert ((got.probs.cpu().double() - mean).abs() <= bound).all()
    f = counts.double() / (n * k)
    loss, size = E * (f * mean).sum(), (lse ** 2).sum() / n
    assert abs(float(got.losses[0]) - loss) <= E * (f * bound).sum() + (E + 20) * U * loss
    # lse is off by the sum's relative error, logf's two last places of log(sum), and its own rounding
    off = share_bound(far, 8) + U * (2 * lse.abs() + 2 * math.log(E) + 2)
    off = torch.where(there, off, 0)
    assert abs(float(got.losses[1]) - size) <= float(((2 * lse.abs() + off) * off).sum() / n + 302 * U * size)


def test_balance_even_is_one():
    # every expert as often as any other, equal logits: the loss is 1, whatever the sizes
    for T, E in ((64, 8), (4096, 64), (512, 512)):
        l = torch.full((T, E), 0.75, device="cuda")
        experts = (torch.arange(T, device="cuda")[:, None] * 2 + torch.arange(2, device="cuda")) % E
        assert abs(float(nv.moe_balance(l, experts).losses[0]) - 1) <= (302 + 8 + 12 + E) * U


def grad_by_hand(l, experts, dweights, renormalize, counts, dlosses):
    """The gradient and a bound of the terms that it is made of, in 64 bits, sums over the choices written out."""
    T, E = l.shape
    p, lse, far, there = shares(l)
    d, size = torch.zeros(T, E, dtype=torch.float64), torch.zeros(T, E, dtype=torch.float64)
    k = experts.shape[1]
    if dweights is not None:
        dw = dweights.double()
        for t in range(T):
            chosen = [(j, int(experts[t, j])) for j in range(k) if 0 <= experts[t, j] < E]
            if renormalize:
                top = max([float(l[t, e]) for _, e in chosen], default=-math.inf)
                if top == -math.inf:
                    continue
                w = {j: math.exp(float(l[t, e]) - top) for j, e in chosen}
                total = sum(w.values())
                w = {j: v / total for j, v in w.items()}
            else:
                w = {j: float(p[t, e]) for j, e in chosen}
            dot, dot_size = sum(w[j] * float(dw[t, j]) for j, _ in chosen), sum(w[j] * abs(float(dw[t, j])) for j, _ in chosen)
            for j, e in chosen:
                d[t, e] += w[j] * (float(dw[t, j]) - (dot if renormalize else 0))
                size[t, e] += w[j] * (abs(float(dw[t, j])) + dot_size)
            if not renormalize:
                d[t] -= p[t] * dot
                size[t] += p[t] * dot_size
    extra = 0
    if counts is not None:
        n = max(1, int(counts[E]))
        f = counts[:E].double() / (n * k)
        a, b = float(dlosses[0]) * E / n, float(dlosses[1]) * 2 / n
        dot = (f * p).sum(1, keepdim=True)
        d += a * p * (f - dot) + b * lse * p
        size += abs(a) * p * (f + dot) + abs(b) * lse.abs() * p
        extra = abs(b) * p * (share_bound(far, 8) + U * (2 * lse.abs() + 2 * math.log(E) + 2))
    return d, size, far, extra


@pytest.mark.parametrize("parts", ["weights", "losses", "both"])
@pytest.mark.parametrize("renormalize", [True, False])
@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T, E, k", [s for s in SIZES if s[0] * s[2] <= 1000] + [(6, 512, 40)])
def test_route_gradient(T, E, k, dtype, mask, renormalize, parts):
    l = drawn(T * 3 + E, T, E, dtype, mask)
    g = torch.Generator().manual_seed(E)
    route = nv.moe_route(l.cuda(), k, renormalize=renormalize)
    dweights = torch.randn(T, k, generator=g) if parts != "losses" else None
    counts, dlosses = (None, None) if parts == "weights" else (nv.moe_balance(l.cuda(), route.experts).counts.cpu(), torch.tensor([0.7, -0.3]))
    cuda = lambda t: t if t is None else t.cuda()  # noqa: E731
    got = nv.moe_route_bwd(l.cuda(), route.experts, cuda(dweights), renormalize=renormalize, counts=cuda(counts), dlosses=cuda(dlosses))
    assert got.dtype == dtype
    want, size, far, extra = grad_by_hand(l, route.experts.cpu(), dweights, renormalize, counts, dlosses)
    # shares twice (an entry's and those of the sum over the row), k choices added, some ten roundings
    bound = (2 * share_bound(far, max(8, k)) + (k + 30) * U) * size + extra + torch.finfo(dtype).eps / 2 * want.abs() * (1 + 1e-6) + 2.0 ** -130
    assert ((got.cpu().double() - want).abs() <= bound).all()


def test_route_gradient_lists():
    # any list of experts: the same one twice, numbers that are none, an expert that is not the largest and far below it
    l = torch.tensor([[0.0, 1.0, 2.0, 3.0], [-200.0, 1.0, 2.0, 300.0], [0.5, -math.inf, 0.0, 1.0], [-math.inf] * 4])
    experts = torch.tensor([[1, 1, 3], [0, 0, 1], [1, 4, -7], [0, 1, 2]], dtype=torch.int32)
    dw = torch.tensor([[1.0, 2.0, -1.0], [1.0, 3.0, 0.5], [1.0, 1.0, 1.0], [1.0, 1.0, 1.0]])
    for renormalize in (True, False):
        got = nv.moe_route_bwd(l.cuda(), experts.cuda(), dw.cuda(), renormalize=renormalize).cpu().double()
        want, size, far, _ = grad_by_hand(l, experts, dw, renormalize, None, None)
        assert ((got - want).abs() <= (2 * share_bound(far, 8) + 33 * U) * size + 2.0 ** -130).all()


@pytest.mark.parametrize("renormalize", [True, False])
def test_gradient_against_differences(renormalize):
    # central differences of the forward calls: step h, the formulas' third derivatives are below 1 here (h^2 / 6), the calls' own error 40 u / h
    T, E, k, h = 4, 12, 3, 2.0 ** -6
    g = torch.Generator().manual_seed(1)
    l = torch.stack([torch.randperm(E, generator=g) for _ in range(T)]).float() * 0.25  # (no choice changes within a step)
    dw, dlosses = torch.randn(T, k, generator=g), torch.tensor([0.5, 0.25])
    experts = nv.moe_route(l.cuda(), k, renormalize=renormalize).experts

    def total(l):
        r = nv.moe_route(l.cuda(), k, renormalize=renormalize)
        assert torch.equal(r.experts, experts)
        b = nv.moe_balance(l.cuda(), r.experts)
        return float((r.weights.cpu().double() * dw).sum() + (b.losses.cpu().double() * dlosses).sum())

    got = nv.moe_route_bwd(l.cuda(), experts, dw.cuda(), renormalize=renormalize, counts=nv.moe_balance(l.cuda(), experts).counts, dlosses=dlosses.cuda()).cpu()
    for t in range(T):
        for e in range(E):
            up, down = l.clone(), l.clone()
            up[t, e] += h
            down[t, e] -= h
            assert abs((total(up) - total(down)) / (2 * h) - float(got[t, e])) <= h * h * float(dw.abs().max() + 1) + 100 * U / h


def test_shards_add_up():
    # two halves of a batch, their counts added: each half's gradient is that half of the whole batch's
    l = drawn(5, 600, 24, torch.float32, "rows").cuda()
    experts = nv.moe_route(l, 2).experts
    whole, a, b = (nv.moe_balance(l[s], experts[s]) for s in (slice(None), slice(0, 250), slice(250, 600)))
    assert torch.equal(whole.counts, a.counts + b.counts)
    d = torch.tensor([0.1, 0.2], device="cuda")
    grads = [nv.moe_route_bwd(l[s], experts[s], counts=whole.counts, dlosses=d) for s in (slice(0, 250), slice(250, 600))]
    assert torch.equal(torch.cat(grads), nv.moe_route_bwd(l, experts, counts=whole.counts, dlosses=d))


def test_same_bits_and_guards():
    l = drawn(9, 3001, 61, torch.bfloat16, "some").cuda()
    r = nv.moe_route(l, 4)
    first = nv.moe_balance(l, r.experts)
    for _ in range(5):
        assert all(torch.equal(s, t) for s, t in zip(first, nv.moe_balance(l, r.experts)))
    # outputs between guards: nothing outside is written
    T, E, k = 3001, 61, 4
    ids, w = torch.full((T * k + 64,), 77, dtype=torch.int32, device="cuda"), torch.full((T * k + 64,), 77.0, device="cuda")
    d = torch.full((T * E + 64,), 77.0, dtype=torch.bfloat16, device="cuda")
    s = torch.cuda.current_stream().cuda_stream
    assert nv.lib.nvfp4_moe_route(l.data_ptr(), nv.BF16, T, E, E, k, 1, ids[32:].data_ptr(), w[32:].data_ptr(), s) == nv.OK
    dw = torch.randn(T, k, device="cuda")
    assert nv.lib.nvfp4_moe_route_bwd(l.data_ptr(), nv.BF16, T, E, E, k, 1, r.experts.data_ptr(), dw.data_ptr(), None, None, d[32:].data_ptr(), s) == nv.OK
    for t in (ids, w, d):
        assert (t[:32] == 77).all() and (t[-32:] == 77).all()
    assert torch.equal(ids[32:-32].view(T, k), r.experts) and torch.equal(w[32:-32].view(T, k), r.weights)


def test_empty_and_refusals():
    l = torch.randn(6, 8, device="cuda")
    none = l[:0]
    r = nv.moe_route(none, 2)
    assert r.experts.shape == r.weights.shape == (0, 2)
    b = nv.moe_balance(none, r.experts)
    assert b.counts.tolist() == [0] * 9 and not b.losses.any() and not b.probs.any()
    assert nv.moe_route_bwd(none, r.experts, r.weights).shape == (0, 8)
    for k in (0, -1, 9):
        with pytest.raises(nv.Nvfp4Error):
            nv.moe_route(l, k)
    with pytest.raises(nv.Nvfp4Error):
        nv.moe_route(torch.randn(2, 513, device="cuda"), 2)
    with pytest.raises(TypeError):
        nv.moe_route(l.half(), 2)
    for bad in (l.t(), l[:1].expand(6, 8), l.view(2, 3, 8)):
        with pytest.raises(ValueError):
            nv.moe_route(bad, 2)
    with pytest.raises(ValueError):
        nv.moe_route(l.cpu(), 2)
    r = nv.moe_route(l, 2)
    with pytest.raises(ValueError):
        nv.moe_balance(l, r.experts[:5])
    with pytest.raises(TypeError):
        nv.moe_balance(l, r.experts.float())
    with pytest.raises(ValueError):
        nv.moe_route_bwd(l, r.experts)
    counts, dlosses = nv.moe_balance(l, r.experts).counts, torch.ones(2, device="cuda")
    with pytest.raises(ValueError):
        nv.moe_route_bwd(l, r.experts, counts=counts)
    with pytest.raises(ValueError):
        nv.moe_route_bwd(l, r.experts, counts=counts[:8], dlosses=dlosses)
    with pytest.raises(TypeError):
        nv.moe_route_bwd(l, r.experts, r.weights.double())
    with pytest.raises(TypeError):
        nv.moe_route_bwd(l, r.experts.long(), r.weights)


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("renormalize", [True, False])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("E", [5, 100])
def test_gradient_of_padding_is_zero_whatever_comes_back(E, dtype, renormalize, bad):
    # a scaled loss that has overflown must not reach the rows that count nowhere
    l = drawn(E, 40, E, dtype, "none")
    l[::3] = -math.inf
    r = nv.moe_route(l.cuda(), 2, renormalize=renormalize)
    counts, dw = nv.moe_balance(l.cuda(), r.experts).counts, torch.full((40, 2), bad, device="cuda")
    for dlosses in ([bad, 0.0], [0.0, bad], [bad, bad]):
        for experts in (r.experts, torch.zeros_like(r.experts)):  # (also where a list names an expert for a row that has none)
            for weights in (None, dw):
                d = nv.moe_route_bwd(l.cuda(), experts, weights, renormalize=renormalize, counts=counts, dlosses=torch.tensor(dlosses, device="cuda"))
                assert (d[::3] == 0).all() and not torch.isfinite(d[1::3]).all()
                d = nv.moe_route_bwd(l.cuda(), experts, dw, renormalize=renormalize)
                assert (d[::3] == 0).all()


@pytest.mark.parametrize("k", [1 << 31, (1 << 32) + 2, 1 << 40, (1 << 64) + 2])
def test_more_experts_than_there_are(k):
    # refused before anything of that size is asked for, also where 32 bits of the number would be a number that is allowed
    with pytest.raises(nv.Nvfp4Error):
        nv.moe_route(torch.randn(1, 8, device="cuda"), k)
