"""CPU-only checks of the 8-bit operators' and the routing's host side: sizes, and every refusal of the C ABI, which happens before
anything is launched (pointers here are numbers that nobody follows)."""
import ctypes as C

import pytest
import torch

from paper_2505_19115_amd import binding as nv

L = nv.lib
P, Q = 0x10000, 0x20000  # 16-byte aligned
F32, BF16 = nv.F32, nv.BF16


def test_sizes():
    assert L.nvfp4_fp8_codes_bytes(5, 1) == 5 * 128 and L.nvfp4_fp8_codes_bytes(5, 129) == 5 * 256 and L.nvfp4_fp8_codes_bytes(5, 0) == 0
    assert L.nvfp4_fp8_scales_bytes(5, 129) == 10 and L.nvfp4_fp8_scales_bytes(0, 129) == 0
    assert L.nvfp4_fp8_codes_bytes(1 << 20, 1 << 13) == 1 << 33
    # whole blocks of a matrix; of groups one more each
    assert [L.nvfp4_fp8_slots(n, 0) for n in (0, 1, 128, 129)] == [0, 1, 1, 2]
    assert [L.nvfp4_fp8_slots(n, 3) for n in (0, 1, 128, 129)] == [3, 3, 4, 4]
    assert L.nvfp4_fp8_slots(-1, 0) == 0
    # one workgroup needs no counts, many leave one for each expert
    assert L.nvfp4_moe_sort_workspace_bytes(8192, 8) == 0
    assert L.nvfp4_moe_sort_workspace_bytes(8193, 8) == 3 * 8 * 4
    assert L.nvfp4_moe_sort_workspace_bytes(-1, 8) == L.nvfp4_moe_sort_workspace_bytes(1 << 20, 0) == L.nvfp4_moe_sort_workspace_bytes(1 << 20, 513) == 0


def test_group_slots_do_not_overlap():
    # group e's blocks start at floor(first / 128) + e: no two groups share one, whatever the lengths, and all lie below fp8_slots
    g = torch.Generator().manual_seed(0)
    for _ in range(200):
        lengths = torch.randint(0, 300, (int(torch.randint(1, 9, (1,), generator=g)),), generator=g).tolist()
        first, free = 0, 0
        for e, n in enumerate(lengths):
            start = first // 128 + e
            assert start >= free
            free = start + -(-n // 128)
            first += n
        assert free <= L.nvfp4_fp8_slots(first, len(lengths))


def quantize(x=P, dt=BF16, batch=1, rows=4, cols=256, ld=256, order=None, top_k=1, x_rows=4, offsets=None, groups=0, cr=P, sr=P, cc=P, sc=P):
    return L.nvfp4_fp8_quantize(x, dt, batch, rows, cols, ld, order, top_k, x_rows, offsets, groups, cr, sr, cc, sc, None)


@pytest.mark.parametrize("change, status", [
    (dict(dt=2), nv.EINVAL), (dict(dt=-1), nv.EINVAL), (dict(rows=-1), nv.ESHAPE), (dict(cols=-1), nv.ESHAPE), (dict(batch=-1), nv.ESHAPE), (dict(ld=255), nv.ESHAPE),
    (dict(rows=1 << 31), nv.ESHAPE), (dict(cols=(1 << 23) + 1, ld=1 << 24), nv.ESHAPE), (dict(batch=1 << 20, rows=1 << 20), nv.ESHAPE),
    (dict(rows=(1 << 23) + 1), nv.ESHAPE), (dict(x=None), nv.EINVAL), (dict(cr=None, sr=None, cc=None, sc=None), nv.EINVAL), (dict(sr=None), nv.EINVAL), (dict(cc=None), nv.EINVAL),
    (dict(order=Q, top_k=0), nv.EINVAL), (dict(order=Q, x_rows=-1), nv.EINVAL), (dict(order=Q, batch=2), nv.ESHAPE),
    (dict(offsets=Q, groups=0), nv.EINVAL), (dict(offsets=Q, groups=513), nv.EINVAL), (dict(offsets=Q, groups=2, cc=None, sc=None), nv.EINVAL),
    (dict(offsets=Q, groups=2, batch=2), nv.ESHAPE), (dict(x=P + 1), nv.EALIGN), (dict(dt=F32, x=P + 2), nv.EALIGN), (dict(cr=P + 8), nv.EALIGN), (dict(cc=P + 4), nv.EALIGN),
    (dict(order=Q + 2), nv.EALIGN), (dict(offsets=Q + 1, groups=2), nv.EALIGN),
    (dict(rows=0), nv.OK), (dict(cols=0, ld=0), nv.OK), (dict(batch=0), nv.OK), (dict(rows=0, x=None, cr=None, sr=None, cc=None, sc=None), nv.OK)])
def test_quantize_refusals(change, status):
    assert quantize(**change) == status


def gemm(M=4, N=4, K=256, a=P, sa=P, b=P, sb=P, out=Q, dt=BF16, ldc=None):
    return L.nvfp4_fp8_gemm(M, N, K, a, sa, b, sb, out, dt, N if ldc is None else ldc, None)


@pytest.mark.parametrize("change, status", [
    (dict(dt=2), nv.EINVAL), (dict(M=-1), nv.ESHAPE), (dict(N=-1, ldc=0), nv.ESHAPE), (dict(K=-128), nv.ESHAPE), (dict(K=129), nv.ESHAPE), (dict(K=(1 << 23) + 128), nv.ESHAPE),
    (dict(ldc=3), nv.ESHAPE), (dict(M=1 << 31), nv.ESHAPE), (dict(a=None), nv.EINVAL), (dict(sa=None), nv.EINVAL), (dict(b=None), nv.EINVAL), (dict(sb=None), nv.EINVAL),
    (dict(out=None), nv.EINVAL), (dict(a=P + 8), nv.EALIGN), (dict(b=P + 1), nv.EALIGN), (dict(out=Q + 1), nv.EALIGN), (dict(dt=F32, out=Q + 2), nv.EALIGN),
    (dict(M=(1 << 31) - 1, N=(1 << 31) - 1), nv.ESHAPE),  # more tiles than a launch has workgroups
    (dict(M=0), nv.OK), (dict(N=0), nv.OK), (dict(M=0, a=None, out=None), nv.OK)])
def test_gemm_refusals(change, status):
    assert gemm(**change) == status


def experts(rows=4, N=4, K=256, groups=2, offsets=P, a=P, sa=P, b=P, sb=P, out=Q, dt=BF16, ldc=4):
    return L.nvfp4_fp8_gemm_experts(rows, N, K, groups, offsets, a, sa, b, sb, out, dt, ldc, None)


def experts_dw(M=4, N=4, rows=300, groups=2, offsets=P, a=P, sa=P, b=P, sb=P, out=Q, dt=BF16, ldc=4):
    return L.nvfp4_fp8_gemm_experts_dw(M, N, rows, groups, offsets, a, sa, b, sb, out, dt, ldc, None)


@pytest.mark.parametrize("call", [experts, experts_dw])
@pytest.mark.parametrize("change, status", [
    (dict(groups=0), nv.EINVAL), (dict(groups=513), nv.EINVAL), (dict(offsets=None), nv.EINVAL), (dict(offsets=P + 2), nv.EALIGN), (dict(rows=-1), nv.ESHAPE), (dict(N=-1), nv.ESHAPE),
    (dict(ldc=3), nv.ESHAPE), (dict(dt=7), nv.EINVAL), (dict(a=None), nv.EINVAL), (dict(sb=None), nv.EINVAL), (dict(out=None), nv.EINVAL), (dict(out=Q + 1), nv.EALIGN),
    (dict(a=P + 4), nv.EALIGN), (dict(N=0, ldc=0), nv.OK)])
def test_experts_refusals(call, change, status):
    assert call(**change) == status


def test_experts_sizes():
    assert experts(rows=0) == nv.OK and experts_dw(M=0) == nv.OK
    assert experts(groups=512, N=1 << 22, ldc=1 << 22) == nv.ESHAPE and experts_dw(groups=512, M=1 << 22) == nv.ESHAPE  # rows of all experts' weights past 2^31 - 1
    assert experts_dw(rows=1 << 31) == nv.ESHAPE
    assert experts_dw(rows=1 << 30) == nv.ESHAPE  # a contraction past 2^23


def sort(ids=P, size=8, pairs=64, groups=8, offsets=P, order=P, position=P, ws=None, ws_bytes=0):
    return L.nvfp4_moe_sort(ids, size, pairs, groups, offsets, order, position, ws, ws_bytes, None)


@pytest.mark.parametrize("change, status", [
    (dict(size=2), nv.EINVAL), (dict(pairs=-1), nv.ESHAPE), (dict(pairs=1 << 31), nv.ESHAPE), (dict(groups=0), nv.EINVAL), (dict(groups=513), nv.EINVAL), (dict(ids=None), nv.EINVAL),
    (dict(offsets=None), nv.EINVAL), (dict(order=None), nv.EINVAL), (dict(position=None), nv.EINVAL), (dict(ids=P + 4), nv.EALIGN), (dict(size=4, ids=P + 2), nv.EALIGN),
    (dict(order=P + 1), nv.EALIGN), (dict(pairs=1 << 20), nv.EWORKSPACE), (dict(pairs=1 << 20, ws=P, ws_bytes=8191), nv.EWORKSPACE), (dict(ws=P + 1), nv.EALIGN)])
def test_sort_refusals(change, status):
    assert sort(**change) == status


def gather(x=P, dt=BF16, x_rows=4, cols=8, ld=8, order=P, top_k=2, rows=8, out=Q):
    return L.nvfp4_moe_gather(x, dt, x_rows, cols, ld, order, top_k, rows, out, None)


def combine(y=P, dt=BF16, rows=8, cols=8, weights=P, position=P, tokens=4, top_k=2, out=Q):
    return L.nvfp4_moe_combine(y, dt, rows, cols, weights, position, tokens, top_k, out, None)


def combine_bwd(dout=P, y=P, dt=BF16, rows=8, cols=8, weights=P, position=P, offsets=P, groups=2, tokens=4, top_k=2, dy=Q, dweights=Q):
    return L.nvfp4_moe_combine_bwd(dout, y, dt, rows, cols, weights, position, offsets, groups, tokens, top_k, dy, dweights, None)


@pytest.mark.parametrize("change, status", [
    (dict(dt=2), nv.EINVAL), (dict(top_k=0), nv.EINVAL), (dict(x_rows=-1), nv.ESHAPE), (dict(cols=-1), nv.ESHAPE), (dict(ld=7), nv.ESHAPE), (dict(rows=-1), nv.ESHAPE),
    (dict(rows=1 << 31), nv.ESHAPE), (dict(x=None), nv.EINVAL), (dict(order=None), nv.EINVAL), (dict(out=None), nv.EINVAL), (dict(x=P + 1), nv.EALIGN), (dict(order=P + 2), nv.EALIGN),
    (dict(dt=F32, out=Q + 2), nv.EALIGN), (dict(rows=0), nv.OK), (dict(cols=0), nv.OK)])
def test_gather_refusals(change, status):
    assert gather(**change) == status


@pytest.mark.parametrize("change, status", [
    (dict(dt=2), nv.EINVAL), (dict(top_k=0), nv.EINVAL), (dict(rows=-1), nv.ESHAPE), (dict(cols=-1), nv.ESHAPE), (dict(tokens=-1), nv.ESHAPE), (dict(tokens=1 << 30), nv.ESHAPE),
    (dict(y=None), nv.EINVAL), (dict(position=None), nv.EINVAL), (dict(out=None), nv.EINVAL), (dict(y=P + 1), nv.EALIGN), (dict(weights=P + 2), nv.EALIGN), (dict(position=P + 1), nv.EALIGN),
    (dict(tokens=0), nv.OK), (dict(cols=0), nv.OK)])
def test_combine_refusals(change, status):
    assert combine(**change) == status


@pytest.mark.parametrize("change, status", [
    (dict(dt=2), nv.EINVAL), (dict(top_k=0), nv.EINVAL), (dict(groups=0), nv.EINVAL), (dict(groups=513), nv.EINVAL), (dict(rows=-1), nv.ESHAPE), (dict(tokens=-1), nv.ESHAPE),
    (dict(dout=None), nv.EINVAL), (dict(y=None), nv.EINVAL), (dict(weights=None), nv.EINVAL), (dict(position=None), nv.EINVAL), (dict(offsets=None), nv.EINVAL), (dict(dy=None), nv.EINVAL),
    (dict(dweights=None), nv.EINVAL), (dict(dout=P + 1), nv.EALIGN), (dict(dt=F32, dy=Q + 2), nv.EALIGN), (dict(dweights=Q + 2), nv.EALIGN), (dict(offsets=P + 3), nv.EALIGN),
    (dict(tokens=0, rows=0), nv.OK), (dict(tokens=0, cols=0), nv.OK)])
def test_combine_gradient_refusals(change, status):
    assert combine_bwd(**change) == status


def test_binding_refuses_host_tensors_and_wrong_types():
    x, ids = torch.zeros(4, 128), torch.zeros(4, 2, dtype=torch.int64)
    codes, scales = torch.zeros(4, 128, dtype=torch.float8_e4m3fn), torch.zeros(1, 4, dtype=torch.uint8)
    for call in (lambda: nv.fp8_quantize(x), lambda: nv.moe_sort(ids, 2), lambda: nv.moe_gather(x, ids.int(), 1), lambda: nv.moe_combine(x, ids.int()),
                 lambda: nv.moe_combine_bwd(x, x, torch.zeros(4, 2), ids.int(), ids.int()), lambda: nv.Fp8(codes, scales)):
        with pytest.raises(ValueError, match="GPU"):
            call()
    for bad in ((codes.view(torch.uint8), scales), (codes, scales.int()), (codes.t(), scales)):
        with pytest.raises(TypeError):
            nv.Fp8(*bad)


def test_abi_types():
    # sizes come back whole, past 32 bits
    assert L.nvfp4_fp8_codes_bytes.restype is C.c_size_t and L.nvfp4_fp8_slots.restype is C.c_int64


def test_divided_contraction_workspace():
    # an output of few tiles and a long contraction wants scratch memory; a large one, a short contraction and no output do not
    bytes_ = L.nvfp4_fp8_gemm_workspace_bytes
    assert bytes_(512, 4096, 11008, 1) > 0 and bytes_(1000, 4096, 4096, 0) > 0
    assert bytes_(512, 4096, 11008, 1) % (256 * 128 * 4) == 0
    for M, N, K, dt in ((4096, 4096, 11008, 1), (512, 4096, 256, 1), (16, 4096, 4096, 1), (0, 4096, 11008, 1), (512, 0, 11008, 1), (512, 4096, 0, 1), (512, 4096, 11000, 1),
                        (512, 4096, 11008, 5), (-1, 4096, 11008, 1), (1 << 40, 4096, 11008, 1)):
        assert bytes_(M, N, K, dt) == 0
