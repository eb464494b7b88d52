"""CPU-only checks of the host side of the router, the norms and the products with packed 4-bit weights: sizes, and every refusal of the C ABI, which
happens before anything is launched (pointers here are numbers that nobody follows)."""
import ctypes as C
import os
import shutil
import subprocess

import pytest
import torch

from paper_2505_19115_amd import binding as nv
from test_device_code import LLVM, code_object, unwaited_loads

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CLANG = "/opt/rocm/lib/llvm/bin/clang++"

L = nv.lib
P, Q = 0x10000, 0x20000  # 16-byte aligned
F32, BF16 = nv.F32, nv.BF16


def route(logits=P, dt=BF16, tokens=4, groups=8, ld=8, top_k=2, renormalize=1, experts=Q, weights=Q):
    return L.nvfp4_moe_route(logits, dt, tokens, groups, ld, top_k, renormalize, experts, weights, None)


def route_bwd(logits=P, dt=BF16, tokens=4, groups=8, ld=8, top_k=2, renormalize=1, experts=P, dweights=P, counts=P, dlosses=P, dlogits=Q):
    return L.nvfp4_moe_route_bwd(logits, dt, tokens, groups, ld, top_k, renormalize, experts, dweights, counts, dlosses, dlogits, None)


def balance(logits=P, dt=BF16, tokens=4, groups=8, ld=8, experts=P, size=8, top_k=2, losses=Q, counts=Q, probs=Q, ws=None, ws_bytes=0):
    return L.nvfp4_moe_balance(logits, dt, tokens, groups, ld, experts, size, top_k, losses, counts, probs, ws, ws_bytes, None)


@pytest.mark.parametrize("call", [route, route_bwd, balance])
@pytest.mark.parametrize("change, status", [
    (dict(dt=2), nv.EINVAL), (dict(dt=3), nv.EINVAL), (dict(groups=0, ld=0), nv.EINVAL), (dict(groups=513, ld=513), nv.EINVAL), (dict(top_k=0), nv.EINVAL), (dict(top_k=9), nv.EINVAL),
    (dict(tokens=-1), nv.ESHAPE), (dict(tokens=1 << 30), nv.ESHAPE), (dict(ld=7), nv.ESHAPE), (dict(logits=None), nv.EINVAL), (dict(logits=P + 1), nv.EALIGN), (dict(dt=F32, logits=P + 2), nv.EALIGN)])
def test_logits_refusals(call, change, status):
    assert call(**change) == status


@pytest.mark.parametrize("change, status", [
    (dict(experts=None), nv.EINVAL), (dict(weights=None), nv.EINVAL), (dict(experts=Q + 2), nv.EALIGN), (dict(weights=Q + 1), nv.EALIGN), (dict(tokens=0, logits=None, experts=None), nv.OK)])
def test_route_refusals(change, status):
    assert route(**change) == status


@pytest.mark.parametrize("change, status", [
    (dict(counts=None), nv.EINVAL), (dict(dlosses=None), nv.EINVAL), (dict(counts=None, dlosses=None, dweights=None), nv.EINVAL), (dict(experts=None), nv.EINVAL),
    (dict(dlogits=None), nv.EINVAL), (dict(dlogits=Q + 1), nv.EALIGN), (dict(dweights=P + 2), nv.EALIGN), (dict(counts=P + 2), nv.EALIGN), (dict(dlosses=P + 2), nv.EALIGN),
    (dict(experts=P + 2), nv.EALIGN), (dict(tokens=0, dweights=None, logits=None), nv.OK), (dict(tokens=0, dlosses=None), nv.EINVAL)])
def test_route_bwd_refusals(change, status):
    assert route_bwd(**change) == status


@pytest.mark.parametrize("change, status", [
    (dict(size=2), nv.EINVAL), (dict(experts=None), nv.EINVAL), (dict(losses=None), nv.EINVAL), (dict(counts=None), nv.EINVAL), (dict(probs=None), nv.EINVAL), (dict(experts=P + 4), nv.EALIGN),
    (dict(size=4, experts=P + 2), nv.EALIGN), (dict(losses=Q + 2), nv.EALIGN), (dict(tokens=1 << 20), nv.EWORKSPACE), (dict(tokens=1 << 20, ws=P, ws_bytes=63), nv.EWORKSPACE),
    (dict(tokens=1 << 20, ws=P + 2, ws_bytes=1 << 30), nv.EALIGN), (dict(tokens=0, losses=None), nv.EINVAL)])
def test_balance_refusals(change, status):
    assert balance(**change) == status


def test_balance_workspace():
    # few tokens need none; sums and counts of at most 256 workgroups otherwise
    assert L.nvfp4_moe_balance_workspace_bytes(1, 512) == L.nvfp4_moe_balance_workspace_bytes(0, 8) == L.nvfp4_moe_balance_workspace_bytes(5, 513) == 0
    for tokens in (1 << 14, 1 << 20, (1 << 31) - 1):
        for groups in (1, 8, 61, 512):
            n = L.nvfp4_moe_balance_workspace_bytes(tokens, groups)
            assert n % (8 * (groups + 1)) == 0 and 0 < n <= 256 * 8 * (groups + 1)


def norm(x=P, dt=BF16, rows=4, cols=64, ld=64, weight=P, bias=P, wdt=F32, center=1, eps=1e-5, y=Q, mean=Q, rstd=Q):
    return L.nvfp4_layer_norm(x, dt, rows, cols, ld, weight, bias, wdt, center, eps, y, mean, rstd, None)


def norm_bwd(dy=P, ldy=64, x=P, ld=64, dt=BF16, rows=4, cols=64, weight=P, wdt=F32, mean=P, rstd=P, dx=Q, dweight=Q, dbias=Q, ws=P, ws_bytes=1 << 30):
    return L.nvfp4_layer_norm_bwd(dy, ldy, x, ld, dt, rows, cols, weight, wdt, mean, rstd, dx, dweight, dbias, ws, ws_bytes, None)


@pytest.mark.parametrize("change, status", [
    (dict(dt=2), nv.EINVAL), (dict(wdt=5), nv.EINVAL), (dict(eps=-1.0), nv.EINVAL), (dict(eps=float("nan")), nv.EINVAL), (dict(eps=float("inf")), nv.EINVAL), (dict(rows=-1), nv.ESHAPE),
    (dict(rows=1 << 31), nv.ESHAPE), (dict(cols=-1), nv.ESHAPE), (dict(cols=(1 << 23) + 1, ld=1 << 24), nv.ESHAPE), (dict(ld=63), nv.ESHAPE), (dict(x=None), nv.EINVAL), (dict(y=None), nv.EINVAL),
    (dict(x=P + 1), nv.EALIGN), (dict(y=Q + 1), nv.EALIGN), (dict(weight=P + 2), nv.EALIGN), (dict(bias=P + 2), nv.EALIGN), (dict(wdt=BF16, bias=P + 1), nv.EALIGN), (dict(mean=Q + 2), nv.EALIGN),
    (dict(rstd=Q + 2), nv.EALIGN), (dict(rows=0, x=None, y=None), nv.OK), (dict(cols=0, ld=0, x=None), nv.OK)])
def test_norm_refusals(change, status):
    assert norm(**change) == status


@pytest.mark.parametrize("change, status", [
    (dict(dt=2), nv.EINVAL), (dict(wdt=5), nv.EINVAL), (dict(rows=-1), nv.ESHAPE), (dict(rows=1 << 31), nv.ESHAPE), (dict(cols=(1 << 23) + 1, ld=1 << 24, ldy=1 << 24), nv.ESHAPE),
    (dict(ld=63), nv.ESHAPE), (dict(ldy=63), nv.ESHAPE), (dict(dy=None), nv.EINVAL), (dict(x=None), nv.EINVAL), (dict(rstd=None), nv.EINVAL), (dict(dx=None), nv.EINVAL),
    (dict(dy=P + 1), nv.EALIGN), (dict(dx=Q + 1), nv.EALIGN), (dict(dweight=Q + 2), nv.EALIGN), (dict(dbias=Q + 1), nv.EALIGN), (dict(mean=P + 1), nv.EALIGN), (dict(ws=P + 8), nv.EALIGN),
    (dict(ws=None), nv.EWORKSPACE), (dict(ws_bytes=64 * 4), nv.EWORKSPACE), (dict(cols=0, ld=0, ldy=0, dy=None), nv.OK)])
def test_norm_bwd_refusals(change, status):
    assert norm_bwd(**change) == status


def test_norm_workspace():
    q = L.nvfp4_layer_norm_bwd_workspace_bytes
    assert q(100, 64, BF16, 0, 0) == q(0, 64, BF16, 1, 1) == q(4, 0, BF16, 1, 1) == q(4, 64, 2, 1, 1) == 0
    for rows in (1, 5, 1000, 1 << 20, (1 << 31) - 1):
        for cols in (1, 64, 4097, 16385, 1 << 23):
            one = q(rows, cols, F32, 1, 0)
            assert 0 < one <= 1024 * 4 * cols and one % (4 * cols) == 0 and q(rows, cols, F32, 1, 1) == 2 * one == 2 * q(rows, cols, F32, 0, 1)


def fmt(block=16, scale=0, g=1):
    return C.byref(nv._Format(block, scale, g))


def w4(M=4, N=4, K=256, f=None, x=P, dt=BF16, ldx=None, codes=P, scales=P, g=P, out=Q, odt=BF16, ldc=None):
    return L.nvfp4_gemm_w4(M, N, K, f or fmt(), x, dt, K if ldx is None else ldx, codes, scales, g, out, odt, N if ldc is None else ldc, None)


def w4_experts(M=4, N=4, K=256, groups=2, offsets=P, f=None, x=P, dt=BF16, ldx=None, x_rows=4, order=None, top_k=1, codes=P, scales=P, g=P, step=0, out=Q, odt=BF16, ldc=None):
    return L.nvfp4_gemm_w4_experts(M, N, K, groups, offsets, f or fmt(), x, dt, K if ldx is None else ldx, x_rows, order, top_k, codes, scales, g, step, out, odt,
                                   N if ldc is None else ldc, None)


@pytest.mark.parametrize("call", [w4, w4_experts])
@pytest.mark.parametrize("change, status", [
    (dict(dt=2), nv.EINVAL), (dict(odt=3), nv.EINVAL), (dict(f=fmt(16, 2)), nv.EINVAL), (dict(f=fmt(16, 0, 2)), nv.EINVAL), (dict(f=fmt(8)), nv.EUNSUPPORTED), (dict(f=fmt(16, 1, 0)), nv.EUNSUPPORTED),
    (dict(f=fmt(64, 1, 0)), nv.EUNSUPPORTED), (dict(f=fmt(32, 1, 1)), nv.EUNSUPPORTED), (dict(M=-1, x_rows=4), nv.ESHAPE), (dict(N=-1, ldc=4), nv.ESHAPE), (dict(K=-32, ldx=0), nv.ESHAPE),
    (dict(K=48), nv.ESHAPE), (dict(K=160, f=fmt(64)), nv.ESHAPE), (dict(K=(1 << 23) + 32), nv.ESHAPE), (dict(N=1 << 31), nv.ESHAPE), (dict(ldx=255), nv.ESHAPE), (dict(ldc=3), nv.ESHAPE),
    (dict(x=None), nv.EINVAL), (dict(codes=None), nv.EINVAL), (dict(scales=None), nv.EINVAL), (dict(g=None), nv.EINVAL), (dict(out=None), nv.EINVAL), (dict(x=P + 1), nv.EALIGN),
    (dict(dt=F32, x=P + 2), nv.EALIGN), (dict(codes=P + 8), nv.EALIGN), (dict(scales=P + 2), nv.EALIGN), (dict(g=P + 2), nv.EALIGN), (dict(out=Q + 1), nv.EALIGN), (dict(odt=F32, out=Q + 2), nv.EALIGN),
    (dict(N=0), nv.OK), (dict(N=0, codes=None, out=None), nv.OK)])
def test_w4_refusals(call, change, status):
    if call is w4:
        change = {k: v for k, v in change.items() if k != "x_rows"}
    assert call(**change) == status


def test_w4_null_format_and_sizes():
    assert L.nvfp4_gemm_w4(4, 4, 256, None, P, BF16, 256, P, P, P, Q, BF16, 4, None) == nv.EINVAL
    assert w4(M=0) == nv.OK and w4(M=1 << 31) == nv.ESHAPE
    assert w4(M=(1 << 31) - 1, N=(1 << 31) - 1) == nv.ESHAPE  # more tiles than a launch has workgroups


@pytest.mark.parametrize("change, status", [
    (dict(groups=0), nv.EINVAL), (dict(groups=513), nv.EINVAL), (dict(offsets=None), nv.EINVAL), (dict(offsets=P + 2), nv.EALIGN), (dict(order=P, top_k=0), nv.EINVAL), (dict(order=P + 1), nv.EALIGN),
    (dict(step=2), nv.EINVAL), (dict(x_rows=3), nv.ESHAPE), (dict(order=P, x_rows=-1), nv.ESHAPE), (dict(groups=512, N=1 << 22), nv.ESHAPE), (dict(M=0, x_rows=0, x=None), nv.OK)])
def test_w4_experts_refusals(change, status):
    assert w4_experts(**change) == status


def test_binding_refuses_tensors_off_the_gpu():
    x = torch.randn(4, 32)
    w = (torch.zeros(8, 16, dtype=torch.uint8), torch.zeros(8, 2, dtype=torch.uint8), torch.ones(1))
    ids = torch.zeros(4, 2, dtype=torch.int32)
    for call in (lambda: nv.moe_route(x, 2), lambda: nv.moe_balance(x, ids), lambda: nv.moe_route_bwd(x, ids, torch.ones(4, 2)), lambda: nv.layer_norm(x),
                 lambda: nv.layer_norm_bwd(x, x, None, None, torch.ones(4)), lambda: nv.gemm_w4(x, w), lambda: nv.gemm_w4_experts(x, w, ids[0])):
        with pytest.raises(ValueError):
            call()


@pytest.mark.skipif(not shutil.which(CLANG), reason="needs the ROCm compilers")
def test_launches_count_their_threads_in_32_bits(tmp_path):
    exe = str(tmp_path / "launch_grid")
    subprocess.check_call([CLANG, "-std=c++17", "-O1", "-x", "hip", "--offload-host-only", "-I/opt/rocm/include", "-o", exe, os.path.join(ROOT, "tests", "launch_grid_main.cpp"), "-L/opt/rocm/lib", "-lamdhip64"])
    p = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert p.returncode == 0 and "grids ok" in p.stdout, p.stderr


B, F = torch.bfloat16, torch.float32


@pytest.mark.parametrize("args, kernel", [
    ((1, 4096, 11008), ("few rows", 16, 16, 8)), ((16, 12288, 4096), ("few rows", 16, 16, 4)), ((32, 4096, 2048, 8), ("few rows", 16, 16, 4)), ((16, 300, 416, 0, F), ("few rows", 16, 16, 8)),
    ((128, 40, 416, 8), ("few rows", 16, 16, 8)), ((17, 40, 416), ("direct", 32, 64, 4)), ((135, 40, 416, 8), ("few rows", 16, 16, 8)), ((136, 40, 416, 8), ("direct", 32, 64, 4)),
    ((9000, 50, 416), ("direct", 64, 64, 4)), ((1500, 2049, 416), ("direct", 128, 64, 4)), ((9000, 700, 416), ("direct", 128, 128, 4)), ((777, 12288, 4096), ("direct", 112, 192, 4)),
    ((4096, 4096, 4096), ("direct", 128, 256, 4)), ((17, 40, 416, 0, B, False), ("staged", 32, 64, 4)), ((9000, 130, 416, 0, B, False), ("staged", 64, 64, 4)),
    ((1500, 2049, 416, 0, B, False), ("staged", 128, 128, 4)), ((65, 50, 416, 0, F), ("staged", 32, 64, 4)), ((1280, 1920, 2048, 0, F), ("staged", 32, 128, 4)), ((2000, 6001, 416, 0, F), ("staged", 32, 256, 4)),
    ((777, 12288, 4096, 0, F), ("staged", 32, 256, 4)), ((300, 12288, 4096, 0, F), ("staged", 32, 256, 4)), ((64, 12288, 4096, 0, F), ("staged", 32, 64, 4))])
def test_which_kernel_serves_a_packed_product(args, kernel):
    # (256 compute units where there is no GPU to ask)
    assert nv.gemm_w4_kernel(*args) == kernel


def test_no_packed_product_kernel():
    for args in ((0, 4, 128), (4, 0, 128), (4, 4, 100), (4, 4, -32), (1 << 31, 4, 128), (4, 4, (1 << 23) + 32), ((1 << 31) - 1, (1 << 31) - 1, 128), (4, 1 << 22, 128, 512), (4, 4, 128, -1), (4, 4, 128, 513)):
        assert nv.gemm_w4_kernel(*args) is None
    assert L.nvfp4_host_gemm_w4_kernel(4, 4, 128, 0, BF16, 1, None) == 0 and L.nvfp4_host_gemm_w4_kernel(4, 4, 128, 0, 3, 1, (C.c_int32 * 4)()) == 0


def test_direct_loads_of_packed_products_wait_for_their_address(tmp_path):
    # (a tile's first row may come of a lane read, and the loads stand in inline assembly, whose waits the compiler does not make)
    asm = subprocess.run([os.path.join(LLVM, "llvm-objdump"), "-d", code_object("gemm_w4_tiles", tmp_path)], capture_output=True, text=True, check=True).stdout
    loads, unwaited = unwaited_loads(asm)
    assert loads > 0 and not unwaited
