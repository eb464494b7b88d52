"""Offsets past 32 bits: the last rows of tensors of more than 2^32 bytes, against calls on these rows alone (the same kernels, the same bits); sums over long batches."""
import math

import pytest
import torch

from paper_2505_19115_amd import binding as nv

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def test_route_and_gradient():
    T, E, k, last = (1 << 24) + 5, 160, 2, 4099  # 5 GB of logits
    l = torch.zeros(T, E, dtype=torch.bfloat16, device="cuda")
    l[-last:] = torch.randn(last, E, generator=torch.Generator().manual_seed(0)).cuda()
    r, small = nv.moe_route(l, k), nv.moe_route(l[-last:], k)
    assert torch.equal(r.experts[-last:], small.experts) and torch.equal(r.weights[-last:], small.weights)
    assert (r.experts[:1000] == torch.tensor([0, 1], device="cuda")).all()
    b = nv.moe_balance(l, r.experts)
    assert int(b.counts[E]) == T and int(b.counts[:E].sum()) == T * k
    d = nv.moe_route_bwd(l, r.experts, r.weights, counts=b.counts, dlosses=b.losses)
    assert torch.equal(d[-last:], nv.moe_route_bwd(l[-last:], small.experts, small.weights, counts=b.counts, dlosses=b.losses))


def test_norm():
    R, D, last = (1 << 19) + 3, 4104, 1500  # 4.3 GB
    x = torch.ones(R, D, dtype=torch.bfloat16, device="cuda")
    x[-last:] = torch.randn(last, D, generator=torch.Generator().manual_seed(0)).cuda()
    w = torch.randn(D, device="cuda")
    a, b = nv.layer_norm(x, w), nv.layer_norm(x[-last:], w)
    assert torch.equal(a.y[-last:], b.y) and torch.equal(a.rstd[-last:], b.rstd) and not a.y[0].any()
    g = nv.layer_norm_bwd(x, x, w, a.mean, a.rstd)
    assert torch.equal(g.dx[-last:], nv.layer_norm_bwd(x[-last:], x[-last:], w, b.mean, b.rstd).dx)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_packed_products(dtype):
    # x and the result past 2^32 bytes; an order that names rows past them
    M, K, N = (1 << 21) + 7, 1056, 40
    x = torch.zeros(M, K, dtype=dtype, device="cuda")
    x[-300:] = torch.randn(300, K, generator=torch.Generator().manual_seed(0)).cuda()
    w = nv.quantize(torch.randn(2 * N, K, generator=torch.Generator().manual_seed(1)).cuda())
    order = torch.arange(M - 300, M, dtype=torch.int32, device="cuda")
    offsets = torch.tensor([0, 100, 300], dtype=torch.int32, device="cuda")
    got = nv.gemm_w4_experts(x, w, offsets, order=order, out_dtype=torch.float32)
    want = nv.gemm_w4_experts(x[-300:].contiguous(), w, offsets, out_dtype=torch.float32)
    assert got.any() and ((got - want).abs() <= 1e-5 * want.abs().max()).all()
    one = (w[0][:N].contiguous(), w[1][:N].contiguous(), w[2])
    y = nv.gemm_w4(x, one, out_dtype=torch.float32)
    few = nv.gemm_w4(x[-300:], one, out_dtype=torch.float32)
    assert not y[:-300].any() and ((y[-300:] - few).abs() <= 1e-5 * few.abs().max()).all()


def test_balance_of_a_long_batch():
    # 2^23 tokens, 4096 for each group of lanes, all alike: every rounding of a chain of additions falls the same way.  Sums of 64, of 64 of these, of those; then 3 lanes' groups,
    # 8 waves and 256 parts (in three slices): 64 + 64 + 1 + 3 + 8 + 86 + 3 additions at most one after the other, 12 u for a share
    T, E = 1 << 23, 290
    l = torch.zeros(T, E, dtype=torch.bfloat16, device="cuda")
    got = nv.moe_balance(l, torch.zeros(T, 1, dtype=torch.int32, device="cuda"))
    bound = (64 + 64 + 1 + 3 + 8 + 86 + 3 + 12) * U
    assert got.counts.tolist() == [T] + [0] * (E - 1) + [T]
    assert ((got.probs.double() * E - 1).abs() <= bound).all() and abs(float(got.losses[0]) - 1) <= bound + (E + 20) * U
    size = math.log(E) ** 2
    assert abs(float(got.losses[1]) / size - 1) <= bound + 12 * U
