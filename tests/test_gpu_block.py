"""The operators around the products in the order that a mixture-of-experts block calls them, forward, backward and with packed weights: norm, router, balance, sort, products,
combine.  Against the block written out in 64 bits; captured into a graph; on other streams."""
import os
import sys

import pytest
import torch

from paper_2505_19115_amd import binding as nv

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def inputs(T=100, D=256, F=320, E=8, k=2, seed=0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(T, D, generator=g).cuda()
    x[::9] = 0  # (a padding row: its logits are closed below)
    w = (1 + 0.1 * torch.randn(D, generator=g)).cuda()
    router = (torch.randn(E, D, generator=g) * D ** -0.5).cuda()
    packed = nv.quantize((torch.randn(E * F, D, generator=g) * 0.05).cuda())
    return x, w, router, packed, T, D, F, E, k


def serve(x, w, router, packed, k, E):
    n = nv.layer_norm(x, w, center=False)
    logits = n.y @ router.t()
    logits[::9] = float("-inf")
    route = nv.moe_route(logits, k)
    order = nv.moe_sort(route.experts, E)
    y = nv.gemm_w4_experts(n.y, packed, order.offsets, order=order.order, top_k=k, out_dtype=torch.float32)
    return nv.moe_combine(y, order.position, route.weights), logits, route, order


def test_serving_block():
    x, w, router, packed, T, D, F, E, k = inputs()
    out, logits, route, order = serve(x, w, router, packed, k, E)
    x64 = x.cpu().double()
    n = x64 / (x64.square().mean(1, keepdim=True) + 1e-5).sqrt() * w.cpu().double()
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64)
    codes, scales = packed[0].cpu().long(), packed[1].cpu().view(torch.float8_e4m3fn).double()
    wv = (grid[torch.stack([codes & 15, codes >> 4], 2).view(E * F, D)] * scales.repeat_interleave(16, 1) * packed[2].cpu().double()).view(E, F, D)
    l = logits.cpu().double()
    want, size = torch.zeros(T, F, dtype=torch.float64), torch.zeros(T, F, dtype=torch.float64)
    for t in range(T):
        if t % 9 == 0:
            assert route.experts[t].tolist() == [-1, -1]
            continue
        top = torch.topk(l[t], k)
        for p, e in zip(torch.softmax(top.values, 0), top.indices.tolist()):
            want[t] += p * (wv[e] @ n[t])
            size[t] += p * (wv[e].abs() @ n[t].abs())
    # the norm's and the shares' roundings, each within 40 u, and the products' binary32 sums, 1e-5 of sum |x||w|
    assert ((out.cpu().double() - want).abs() <= (1e-5 + 80 * 2.0 ** -24) * size + 1e-30).all()
    assert not out[::9].any()


def test_gradient_of_the_block_against_autograd():
    """norm -> router -> weights, with the balance loss: the operators' gradients chained by hand against torch's of the formulas in 64 bits."""
    x, w, router, _, T, D, F, E, k = inputs()
    g = torch.Generator().manual_seed(5)
    dweights, dlosses = torch.randn(T, k, generator=g).cuda(), torch.tensor([0.3, 0.1], device="cuda")
    n = nv.layer_norm(x, w)
    logits = n.y @ router.t()
    logits[::9] = float("-inf")
    route = nv.moe_route(logits, k)
    balance = nv.moe_balance(logits, route.experts)
    dl = nv.moe_route_bwd(logits, route.experts, dweights, counts=balance.counts, dlosses=dlosses)
    got = nv.layer_norm_bwd(dl @ router, x, w, n.mean, n.rstd, bias=True)

    X, W, B = x.cpu().double().requires_grad_(), w.cpu().double().requires_grad_(), torch.zeros(D, dtype=torch.float64, requires_grad=True)
    m = X.mean(1, keepdim=True)
    h = (X - m) / ((X - m).square().mean(1, keepdim=True) + 1e-5).sqrt() * W + B
    L = h @ router.cpu().double().t()
    live = torch.arange(T) % 9 != 0
    L = L[live]
    ids = route.experts.cpu().long()[live]
    weights = torch.softmax(L.gather(1, ids), 1)
    p, N = torch.softmax(L, 1), int(live.sum())
    f = torch.bincount(ids.reshape(-1), minlength=E).double() / (N * k)
    losses = torch.stack([E * (f * p.mean(0)).sum(), torch.logsumexp(L, 1).square().mean()])
    total = (weights * dweights.cpu().double()[live]).sum() + (losses * dlosses.cpu().double()).sum()
    total.backward()
    assert abs(balance.losses.cpu().double() - losses.detach()).max() <= 1e-5 * losses.detach().max()
    # sums of D = 256 terms on both sides of the chain, each a binary32 one: a few hundred u of their sizes
    for a, b in ((got.dx, X.grad), (got.dweight, W.grad), (got.dbias, B.grad)):
        assert (a.cpu().double() - b).norm() <= 600 * 2.0 ** -24 * b.norm()


def test_captured_and_replayed():
    # graphs of the whole chain, replayed on new inputs, with eager calls of the same between the replays; two graphs side by side
    state = inputs(T=3000)
    x, w, router, packed, T, D, F, E, k = state
    dweights, dl = torch.randn(T, k, device="cuda"), torch.tensor([0.5, 0.25], device="cuda")

    def chain():
        out, logits, route, order = serve(x, w, router, packed, k, E)
        b = nv.moe_balance(logits, route.experts)
        d = nv.moe_route_bwd(logits, route.experts, dweights, counts=b.counts, dlosses=dl)
        n = nv.layer_norm(x, w)
        g = nv.layer_norm_bwd(x, x, w, n.mean, n.rstd, bias=True)
        few = nv.gemm_w4(x[:5], packed)
        return [out, route.weights, *b, d, *g, few]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        chain()
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            kept = chain()
        graphs.append((graph, kept))
    for seed in range(3):
        x.copy_(torch.randn(T, D, generator=torch.Generator().manual_seed(seed)))
        want = chain()
        for graph, kept in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for _, kept in graphs:
            assert all(torch.equal(a, b) for a, b in zip(kept, want))


def test_other_streams():
    x, w, router, packed, T, D, F, E, k = inputs(T=2000)
    want = serve(x, w, router, packed, k, E)[0]
    bal = nv.moe_balance(x, torch.zeros(2000, 1, dtype=torch.int32, device="cuda"))
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    got, balances = [], []
    for s in streams:
        with torch.cuda.stream(s):
            got.append(serve(x, w, router, packed, k, E)[0])
            balances.append(nv.moe_balance(x, torch.zeros(2000, 1, dtype=torch.int32, device="cuda")))
    torch.cuda.synchronize()
    assert all(torch.equal(g, want) for g in got)
    assert all(torch.equal(a, b) for other in balances for a, b in zip(other, bal))


def test_example_uses_them():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import experts_training as ex
    torch.manual_seed(0)
    layer = ex.Experts(8, 2, 64, 128, balance=0.01)
    x = torch.randn(40, 64, device="cuda", dtype=torch.bfloat16, requires_grad=True)
    y = layer(x)
    (y.float().square().mean() + layer.balance_loss).backward()
    assert torch.isfinite(y).all() and layer.balance_loss > 0
    for p in layer.parameters():
        assert p.grad is not None and torch.isfinite(p.grad).all() and p.grad.any()
    # the norm's gradients against torch's, in binary32
    v = torch.randn(30, 64, device="cuda", requires_grad=True)
    weight = torch.randn(64, device="cuda", requires_grad=True)
    up = torch.randn(30, 64, device="cuda")
    ex.RMSNorm.apply(v, weight).backward(up)
    a, b = v.detach().double().requires_grad_(), weight.detach().double().requires_grad_()
    (a / (a.square().mean(1, keepdim=True) + 1e-5).sqrt() * b).backward(up.double())
    assert (v.grad - a.grad).norm() <= 100 * 2.0 ** -24 * a.grad.norm() and (weight.grad - b.grad).norm() <= 100 * 2.0 ** -24 * b.grad.norm()


def test_example_without_a_balance_loss_pays_for_none(monkeypatch):
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import experts_training as ex
    torch.manual_seed(0)
    layer = ex.Experts(8, 2, 64, 128)
    x, up = torch.randn(40, 64, device="cuda", dtype=torch.bfloat16), torch.randn(40, 2, device="cuda")
    logits = [torch.randn(40, 8, generator=torch.Generator().manual_seed(0)).cuda().requires_grad_() for _ in range(2)]
    with monkeypatch.context() as m:
        m.setattr(ex.nv, "moe_balance", lambda *a: pytest.fail("asked for the balance"))
        y = layer(x)
        (y.float().square().mean() + layer.balance_loss).backward()
        assert torch.isfinite(y).all() and layer.balance_loss == 0 and all(p.grad.any() for p in layer.parameters())
        without = ex.Route.apply(logits[0], 2, False)
        (without[0] * up).sum().backward()
    # the same choice, weights and gradient as with a balance that nothing comes back from
    beside = ex.Route.apply(logits[1], 2, True)
    (beside[0] * up).sum().backward()
    assert torch.equal(without[0], beside[0]) and torch.equal(without[2], beside[2]) and not without[1].any() and torch.equal(logits[0].grad, logits[1].grad)
