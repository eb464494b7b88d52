"""8-bit operators on the GPU at the sizes at which each kernel and each of its ways is taken, against 64 bits.

Bounds on products, with S = sum |a| |b| of the output: binary32 (K / 32 + 48) 2^-24 S, 2^-24 S more for each part of a divided contraction (16 at the most);
bf16 (7 * 2^-13 + K / 8 * 2^-23) S and half of bf16's eps of the result."""
import pytest
import torch

from paper_2505_19115_amd import binding as nv

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float32]


def test_quantize_empty_stacks():
    # no matrix, matrices without rows, without columns, whole or as views: operands without elements
    base = torch.ones(3, 4, 5, device="cuda")
    for x in (torch.empty(0, 4, 5, device="cuda"), torch.empty(3, 0, 5, device="cuda"), torch.empty(3, 4, 0, device="cuda"), base[:, :0], base[:, :, :0], base[:0], base[:, :1][:, :0]):
        E, R, C = x.shape
        rows, cols = nv.fp8_quantize(x, cols=True)
        assert rows.codes.shape == (E * R, -(-C // 128) * 128) and rows.scales.shape == (-(-C // 128), E * R)
        assert cols.codes.shape == (E * C, -(-R // 128) * 128) and cols.scales.shape == (-(-R // 128), E * C)


# ---- products, each on the kernel that the test is about

def two_to(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def values(q):
    s = two_to(q.scales.t().long() - 127)
    return (q.codes.double().view(q.codes.shape[0], -1, 128) * s[..., None]).view(q.codes.shape)


def tensor(g, *shape):
    x = torch.randn(*shape, generator=g, device="cuda") * torch.exp(2 * torch.rand(*shape[:-1], 1, generator=g, device="cuda") - 1)
    return x * (1 + 59 * (torch.rand(*shape, generator=g, device="cuda") < 0.002))


def near(out, A, B, dtype, parts=0):
    ref, K = A @ B.t(), A.shape[1]
    S = A.abs() @ B.abs().t()
    most = S * ((K / 32 + 48 + parts) * 2.0 ** -24 if dtype == torch.float32 else 7 * 2.0 ** -13 + K / 8 * 2.0 ** -23 + parts * 2.0 ** -24) + 1e-300
    if dtype == torch.bfloat16:
        most += torch.finfo(dtype).eps / 2 * ref.abs()
    return bool(((out.double() - ref).abs() <= most).all())


def operands(seed, M, N, K):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [nv.fp8_quantize(tensor(g, n, K))[0] for n in (M, N)]


def inside(M, N, dtype):
    """An output inside a larger tensor of sevens, and whether what is beside it still is that."""
    base = torch.full((M + 2, N + 5), 7.0, dtype=dtype, device="cuda")
    return base[1:-1, 3:3 + N], lambda: all(bool((t == 7).all()) for t in (base[0], base[-1], base[:, :3], base[:, 3 + N:]))


# rows and columns of a workgroup, K tiles of a batch (a wave's last batch is not full)
FEW_ROWS = [(5, 18, 384, 16, 16, 1), (13, 100, 2304, 16, 16, 2), (3, 33, 4480, 16, 16, 4), (1, 4506, 384, 16, 32, 1), (9, 4530, 2304, 16, 32, 2), (15, 4180, 4480, 16, 32, 4),
            (7, 9153, 384, 16, 48, 1), (3, 8888, 2304, 16, 48, 2), (16, 8473, 4480, 16, 48, 4), (1, 13666, 384, 16, 64, 1), (5, 13101, 2304, 16, 64, 2), (11, 13166, 4480, 16, 64, 4),
            (410, 298, 384, 32, 16, 1), (462, 258, 2304, 32, 16, 2), (599, 197, 4608, 32, 16, 4), (53, 3269, 384, 32, 32, 1), (19, 6202, 2304, 32, 32, 2), (22, 9107, 384, 32, 48, 1),
            (20, 8725, 2304, 32, 48, 2), (36, 6437, 384, 32, 64, 1), (34, 6781, 2304, 32, 64, 2), (191, 2692, 768, 64, 32, 1), (312, 1623, 2432, 64, 32, 2), (36, 10180, 384, 64, 48, 1),
            (66, 6511, 384, 64, 64, 1)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M, N, K, rows, cols, batch", FEW_ROWS)
def test_few_rows(M, N, K, rows, cols, batch, dtype):
    assert nv.fp8_gemm_kernel("fp8_gemm", M, N, K, out_dtype=dtype)[:4] == ("few rows", rows, cols, batch)
    a, b = operands(M + N, M, N, K)
    out, untouched = inside(M, N, dtype)
    nv.fp8_gemm(a, b, out=out)
    assert near(out, values(a), values(b), dtype) and untouched() and torch.equal(out, nv.fp8_gemm(a, b, out_dtype=dtype))


@pytest.mark.parametrize("dtype, M, N, K, cols, parts", [
    (torch.bfloat16, 510, 4004, 7808, 128, 4), (torch.bfloat16, 391, 370, 12032, 128, 16), (torch.bfloat16, 990, 6100, 9856, 192, 2), (torch.bfloat16, 775, 1297, 15872, 192, 9),
    (torch.bfloat16, 777, 4601, 9088, 256, 3), (torch.bfloat16, 266, 5076, 14720, 256, 6), (torch.float32, 384, 6016, 7296, 128, 2), (torch.float32, 512, 4090, 11008, 128, 4)])
def test_divided_contraction(M, N, K, cols, parts, dtype):
    assert nv.fp8_gemm_kernel("fp8_gemm", M, N, K, out_dtype=dtype)[:4] == ("divided", 256, cols, parts)
    assert nv.fp8_gemm_kernel("nvfp4_fp8_gemm", M, N, K, out_dtype=dtype).name != "divided"
    a, b = operands(M + N, M, N, K)
    out, untouched = inside(M, N, dtype)
    nv.fp8_gemm(a, b, out=out)
    assert near(out, values(a), values(b), dtype, parts) and untouched() and torch.equal(out, nv.fp8_gemm(a, b, out_dtype=dtype))


# outputs past the last cache level: whole tiles by streaming stores, those at the edges by others
@pytest.mark.parametrize("dtype, M, N, cols", [(torch.bfloat16, 16400, 8200, 192), (torch.bfloat16, 8200, 16700, 256), (torch.float32, 8200, 8260, 128)])
def test_streamed_output(M, N, cols, dtype):
    kernel = nv.fp8_gemm_kernel("fp8_gemm", M, N, 256, out_dtype=dtype)
    assert kernel == ("wide", 256, cols, 1, True) and (M // 256) * (N // cols) > 256
    a, b = operands(M + N, M, N, 256)
    out = nv.fp8_gemm(a, b, out_dtype=dtype)
    A, B = values(a), values(b)
    assert all(near(out[i:i + 2048], A[i:i + 2048], B, dtype) for i in range(0, M, 2048))


def routed(seed, T, k, E, drop=0.0, without=()):
    """Pairs of T tokens sorted by expert, some dropped, none to the experts of `without`."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    logits = torch.randn(T, E, generator=g, device="cuda") + torch.randn(1, E, generator=g, device="cuda")
    for e in without:
        logits[:, e] = -float("inf")
    ids = torch.topk(logits, k, dim=1).indices
    return g, nv.moe_sort(torch.where(torch.rand(T, k, generator=g, device="cuda") < drop, -1, ids), E)


# few rows an expert, in batches of one, two and four K tiles of a wave, the last not full
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T, k, E, N, K, batch", [(40, 4, 64, 100, 500, 1), (40, 4, 64, 100, 1100, 2), (8, 2, 8, 333, 2100, 4), (30, 3, 32, 64, 4200, 4), (1, 2, 8, 500, 4096, 4)])
def test_experts_of_few_rows(T, k, E, N, K, batch, dtype):
    assert nv.fp8_gemm_kernel("fp8_gemm_experts", T * k, N, -(-K // 128) * 128, E, dtype)[:4] == ("few rows", 16, 32, batch)
    g, o = routed(T + K, T, k, E, 0.2 if T > 1 else 0.0)
    off = o.offsets.tolist()
    a, b = nv.fp8_quantize(tensor(g, T, K), order=o.order, top_k=k)[0], nv.fp8_quantize(tensor(g, E, N, K))[0]
    y = nv.fp8_gemm_experts(a, b, o.offsets, out_dtype=dtype)
    A, B = values(a), values(b).view(E, N, -1)
    assert all(near(y[off[e]:off[e + 1]], A[off[e]:off[e + 1]], B[e], dtype) for e in range(E)) and bool((y[off[-1]:] == 0).all())


# more tiles than CUs, so that workgroups walk from one to the next; the widths of a tile; dropped rows at the end
@pytest.mark.parametrize("dtype, T, k, E, N, K, cols", [(torch.bfloat16, 3500, 2, 5, 3000, 640, 192), (torch.bfloat16, 3000, 2, 4, 4500, 384, 256), (torch.bfloat16, 12000, 1, 20, 512, 512, 128),
                                                        (torch.float32, 3500, 2, 5, 3000, 640, 128)])
def test_experts_of_many_tiles(T, k, E, N, K, cols, dtype):
    assert nv.fp8_gemm_kernel("fp8_gemm_experts", T * k, N, K, E, dtype)[:3] == ("wide", 256, cols)
    g, o = routed(T + N, T, k, E, 0.1, without=(1,))
    off = o.offsets.tolist()
    if cols > 128 or dtype == torch.float32:
        assert sum(-(-(j - i) // 256) for i, j in zip(off, off[1:] + [T * k])) * -(-N // cols) > 256
    a, b = nv.fp8_quantize(tensor(g, T, K), order=o.order, top_k=k)[0], nv.fp8_quantize(tensor(g, E, N, K))[0]
    y = nv.fp8_gemm_experts(a, b, o.offsets, out_dtype=dtype)
    A, B = values(a), values(b).view(E, N, -1)
    assert all(near(y[off[e]:off[e + 1]], A[off[e]:off[e + 1]], B[e], dtype) for e in range(E)) and bool((y[off[-1]:] == 0).all())
    assert torch.equal(y, nv.fp8_gemm_experts(a, b, o.offsets, out_dtype=dtype))


# of many and of few tiles an expert, walked by more workgroups than there are and not; experts without rows first, between and last; outputs streamed
@pytest.mark.parametrize("dtype, M, N, T, k, E, cols, streamed", [
    (torch.bfloat16, 2300, 2048, 1300, 2, 5, 192, False), (torch.bfloat16, 2080, 2100, 1500, 2, 6, 256, False), (torch.bfloat16, 520, 512, 6000, 2, 20, 128, False),
    (torch.bfloat16, 4096, 2048, 3000, 2, 16, 256, True), (torch.bfloat16, 4100, 2048, 3000, 2, 17, 192, True),
    (torch.float32, 2300, 2048, 1300, 2, 6, 128, False), (torch.float32, 4100, 2060, 2000, 2, 8, 128, True)])
def test_weight_gradients_of_many_tiles(M, N, T, k, E, cols, streamed, dtype):
    kernel = nv.fp8_gemm_kernel("fp8_gemm_experts_dw", M, N, T * k, E, dtype)
    assert kernel == ("wide", 256, cols, 1, streamed)
    each = -(-M // 256) * -(-N // cols)
    assert (each >= 64 and each * E > 256) or (each < 64 and M == 520)
    g, o = routed(M + T, T, k, E, 0.1, without=(0, E // 2, E - 1))
    off = o.offsets.tolist()
    d = nv.fp8_quantize(tensor(g, T * k, M), rows=False, cols=True, offsets=o.offsets)[1]
    c = nv.fp8_quantize(tensor(g, T, N), rows=False, cols=True, order=o.order, top_k=k, offsets=o.offsets)[1]
    dw = nv.fp8_gemm_experts_dw(d, c, o.offsets, out_dtype=dtype, rows=T * k)
    for e in range(E):
        first, n = 128 * (off[e] // 128 + e), -(-(off[e + 1] - off[e]) // 128) * 128
        part = lambda q: values(nv.Fp8(q.codes[:, first:first + n].contiguous(), q.scales[first // 128:(first + n) // 128].contiguous()))  # noqa: E731
        assert near(dw[e], part(d), part(c), dtype) if n else bool((dw[e] == 0).all()), e
    assert torch.equal(dw, nv.fp8_gemm_experts_dw(d, c, o.offsets, out_dtype=dtype, rows=T * k))


# ---- offsets that are none

class Guarded:
    """Bytes between guards of NaN codes and scales, and whether these still are that."""

    def __init__(self, *shape, fill):
        n = 1
        for s in shape:
            n *= s
        self.base = torch.full((n + 8192,), 0xFF, dtype=torch.uint8, device="cuda")
        self.inner = self.base[4096:4096 + n]
        self.inner.copy_(fill.reshape(-1).view(torch.uint8) if torch.is_tensor(fill) else torch.full_like(self.inner, fill))
        self.ptr = self.inner.data_ptr()

    def whole(self):
        return bool((self.base[:4096] == 0xFF).all()) and bool((self.base[4096 + self.inner.numel():] == 0xFF).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows, N, K, kernel, kernel_dw", [(20, 200, 256, "few rows", "tiles"), (300, 200, 256, "tiles", "tiles"), (3300, 1100, 1024, "wide", "wide")])
@pytest.mark.parametrize("bad", [[0, 0.67, 0.33, 1], [-5, 3.3, 6.7, 1 << 30], [1, 0.67, 0.33, 0], [0.02, 0.02, 0.02, 0.02]])
def test_offsets_that_are_not_ascending(bad, rows, N, K, kernel, kernel_dw, dtype):
    # whatever the offsets hold, nothing is read or written outside the tensors: what is beside them stays, and none of its NaN comes in
    E = 3
    if kernel == "few rows":
        E = 16
        bad = bad + [bad[1 + i % 3] for i in range(E - 3)]
    assert nv.fp8_gemm_kernel("fp8_gemm_experts", rows, N, K, E, dtype).name == kernel and nv.fp8_gemm_kernel("fp8_gemm_experts_dw", K, N, rows, E, dtype).name == kernel_dw
    offsets = torch.tensor([int(b * rows) if abs(b) < 7 and b != -5 else b for b in bad], dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(rows)
    slots, stream, L, tag, size = rows // 128 + E, torch.cuda.current_stream().cuda_stream, nv.lib, nv.F32 if dtype == torch.float32 else nv.BF16, torch.finfo(dtype).bits // 8
    x = torch.randn(rows, K, generator=g, device="cuda")
    # the quantizer
    codes_r, scales_r, codes_c, scales_c = (Guarded(*s, fill=0) for s in ((rows, K), (K // 128, rows), (K, 128 * slots), (slots, K)))
    assert L.nvfp4_fp8_quantize(x.data_ptr(), nv.F32, 1, rows, K, K, None, 1, rows, offsets.data_ptr(), E, codes_r.ptr, scales_r.ptr, codes_c.ptr, scales_c.ptr, stream) == nv.OK
    assert all(t.whole() for t in (codes_r, scales_r, codes_c, scales_c))
    # the products, of operands without a NaN
    q = nv.fp8_quantize(x)[0]
    a, sa = Guarded(rows, K, fill=q.codes), Guarded(K // 128, rows, fill=q.scales)
    w = nv.fp8_quantize(torch.randn(E * N, K, generator=g, device="cuda"))[0]
    b, sb = Guarded(E * N, K, fill=w.codes), Guarded(K // 128, E * N, fill=w.scales)
    out = Guarded(rows, N, size, fill=0)
    assert L.nvfp4_fp8_gemm_experts(rows, N, K, E, offsets.data_ptr(), a.ptr, sa.ptr, b.ptr, sb.ptr, out.ptr, tag, N, stream) == nv.OK
    assert all(t.whole() for t in (a, sa, b, sb, out)) and bool(out.inner.view(dtype).isfinite().all())
    d, c = (nv.fp8_quantize(torch.randn(n, 128 * slots, generator=g, device="cuda"))[0] for n in (K, N))
    a, sa, b, sb = Guarded(K, 128 * slots, fill=d.codes), Guarded(slots, K, fill=d.scales), Guarded(N, 128 * slots, fill=c.codes), Guarded(slots, N, fill=c.scales)
    out = Guarded(E, K, N, size, fill=0)
    assert L.nvfp4_fp8_gemm_experts_dw(K, N, rows, E, offsets.data_ptr(), a.ptr, sa.ptr, b.ptr, sb.ptr, out.ptr, tag, N, stream) == nv.OK
    assert all(t.whole() for t in (a, sa, b, sb, out)) and bool(out.inner.view(dtype).isfinite().all())
