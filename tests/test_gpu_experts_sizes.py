"""Routing, quantizer and products at numbers of rows whose launches have more threads than are counted in 32 bits, one row at a time a row of a small table, so
that all of the answer can be looked at."""
import pytest
import torch

from paper_2505_19115_amd import binding as nv

pytestmark = pytest.mark.gpu
ROWS = (1 << 29) + 37  # eight lanes a row
TABLE = 1000           # the order's other 24 numbers name no row


@pytest.fixture(autouse=True)
def memory():
    yield
    torch.cuda.empty_cache()


def order_of(n):
    return torch.arange(n, dtype=torch.int32, device="cuda").bitwise_and_(1023)


def table(seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(TABLE, 1, generator=g, device="cuda").bfloat16()


def pieces(n, size=1 << 26):
    return ((i, min(n, i + size)) for i in range(0, n, size))


def test_gather():
    x, order = table(1), order_of(ROWS)
    out = nv.moe_gather(x, order, 1)
    padded = torch.cat([x[:, 0], x.new_zeros(24)])
    assert all(torch.equal(out[i:j, 0], padded[order[i:j].long()]) for i, j in pieces(ROWS))


def test_combine():
    y, position = table(2), order_of(ROWS).view(-1, 1)
    position[position >= TABLE] = -1
    weights = torch.full((ROWS, 1), 0.5, device="cuda")
    out = nv.moe_combine(y, position, weights)
    padded = torch.cat([y[:, 0] * 0.5, y.new_zeros(1)])  # (halving is exact)
    assert all(torch.equal(out[i:j, 0], padded[position[i:j, 0].long()]) for i, j in pieces(ROWS))


def test_combine_gradient():
    # the pairs that are kept stand at both ends
    y, dout = table(3), torch.ones(ROWS, 1, dtype=torch.bfloat16, device="cuda")
    position = torch.full((ROWS, 1), -1, dtype=torch.int32, device="cuda")
    position[:500, 0] = torch.arange(500, dtype=torch.int32, device="cuda")
    position[-400:, 0] = torch.arange(500, 900, dtype=torch.int32, device="cuda")
    weights = torch.full((ROWS, 1), 0.25, device="cuda")
    dy, dw = nv.moe_combine_bwd(dout, y, weights, position, torch.tensor([0, 900], dtype=torch.int32, device="cuda"))
    assert bool((dy[:900] == 0.25).all()) and bool((dy[900:] == 0).all())
    assert torch.equal(dw[:500, 0], y[:500, 0].float()) and torch.equal(dw[-400:, 0], y[500:900, 0].float())
    assert all(bool((dw[max(i, 500): min(j, ROWS - 400)] == 0).all()) for i, j in pieces(ROWS))


def test_quantize_rows():
    x, order = table(4), order_of(ROWS)
    q = nv.fp8_quantize(x, order=order, top_k=1)[0]
    few = nv.fp8_quantize(x, order=order[:1024].contiguous(), top_k=1)[0]
    codes, scales = few.codes.view(torch.uint8), few.scales[0]
    for i, j in pieces(ROWS, 1 << 24):
        assert torch.equal(q.codes[i:j].view(torch.uint8).view(torch.int64), codes[order[i:j].long()].view(torch.int64)), i
        assert torch.equal(q.scales[0, i:j], scales[order[i:j].long()]), i


def test_products_without_a_contraction():
    # the most rows, and the most columns of one expert: zeros
    most = (1 << 31) - 1
    e4m3 = lambda n: nv.Fp8(torch.empty(n, 0, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(0, n, dtype=torch.uint8, device="cuda"))  # noqa: E731
    out = torch.full((most, 1), 3.0, dtype=torch.bfloat16, device="cuda")
    nv.fp8_gemm(e4m3(most), e4m3(1), out=out)
    assert int(out.count_nonzero()) == 0
    out.fill_(3.0)
    nv.fp8_gemm(e4m3(1), e4m3(most), out=out.view(1, most))
    assert int(out.count_nonzero()) == 0
    del out
    offsets = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    assert int(nv.fp8_gemm_experts(e4m3(1), e4m3(most), offsets).count_nonzero()) == 0


@pytest.mark.parametrize("kept", [(1 << 31) - 1, 5])
def test_an_expert_of_the_most_rows(kept):
    # a group's rows (an expert's, or those of none) and a tile's more than 32 bits hold with a sign
    most = (1 << 31) - 1
    out = torch.full((most, 1), 3.0, dtype=torch.bfloat16, device="cuda")
    offsets = torch.tensor([0, kept], dtype=torch.int32, device="cuda")
    assert nv.lib.nvfp4_fp8_gemm_experts(most, 1, 0, 1, offsets.data_ptr(), None, None, None, None, out.data_ptr(), nv.BF16, 1, torch.cuda.current_stream().cuda_stream) == nv.OK
    assert int(out.count_nonzero()) == 0
