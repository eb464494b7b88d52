"""Products of 8-bit operands whose scales stand at the ends of their range, on every kernel, against 64 bits.

Bounds, with S = sum |a| |b| of the output: binary32, where a block's sum takes its scales afterwards, one rounding more for each of K / 128 blocks than
the products' own (K / 32 + 48) 2^-24 S, and each of these roundings 2^-149 at the least; bf16 as everywhere, 7 * 2^-13 S, K / 8 sums of 2^-23 S, and half of
bf16's eps of the result."""
import pytest
import torch

from paper_2505_19115_amd import binding as nv

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float32]
# waves that divide the contraction, tiles of 128 x 128, of 256 rows, and a contraction divided among workgroups
SIZES = [(3, 5, 256), (16, 700, 384), (40, 200, 2560), (300, 515, 256), (2100, 2300, 384), (512, 1000, 8064)]
ENDS = [((0, 1, 2, 3, 4), (246, 247, 250, 254)), ((246, 247, 250, 254), (0, 1, 2, 3, 4)), ((0, 100, 247), (100, 101))]


def two_to(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def values(q):
    s = two_to(q.scales.t().long() - 127)
    return (q.codes.double().view(q.codes.shape[0], -1, 128) * s[..., None]).view(q.codes.shape)


def operand(g, rows, K, bytes_):
    """Codes of all magnitudes, each block's scale byte one of bytes_; some blocks of zeros, whose byte is 0."""
    codes = torch.randint(0, 256, (rows, K // 128, 128), generator=g, device="cuda", dtype=torch.uint8)
    codes[(codes & 127) == 127] = 8
    scales = torch.tensor(bytes_, dtype=torch.uint8, device="cuda")[torch.randint(0, len(bytes_), (K // 128, rows), generator=g, device="cuda")]
    none = torch.rand(K // 128, rows, generator=g, device="cuda") < 0.1
    codes[none.t()] = 0
    scales[none] = 0
    return nv.Fp8(codes.view(rows, K).view(torch.float8_e4m3fn), scales)


def check(out, A, B, dtype):
    ref, S, K = A @ B.t(), A.abs() @ B.abs().t(), A.shape[1]
    if dtype == torch.float32:
        most = (K / 32 + K / 128 + 48) * (2.0 ** -24 * S + 2.0 ** -149)
    else:
        most = (7 * 2.0 ** -13 + K / 8 * 2.0 ** -23) * S + torch.finfo(torch.bfloat16).eps / 2 * ref.abs() + K / 128 * 2.0 ** -133
    assert bool(out.isfinite().all()) and bool(((out.double() - ref).abs() <= most).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("ends", ENDS)
@pytest.mark.parametrize("M, N, K", SIZES)
def test_scales_at_the_ends(M, N, K, ends, dtype):
    g = torch.Generator(device="cuda").manual_seed(M + N + K)
    a, b = operand(g, M, K, ends[0]), operand(g, N, K, ends[1])
    out = nv.fp8_gemm(a, b, out_dtype=dtype)
    check(out, values(a), values(b), dtype)
    assert torch.equal(out, nv.fp8_gemm(a, b, out_dtype=dtype))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows, E, N, K", [(20, 6, 200, 256), (300, 4, 300, 256), (3000, 3, 1100, 384)])
def test_experts_scales_at_the_ends(rows, E, N, K, dtype):
    g = torch.Generator(device="cuda").manual_seed(rows)
    kept = rows - rows // 8  # the rest are of no expert
    cut = torch.sort(torch.randint(0, kept + 1, (E - 1,), generator=g, device="cuda")).values.tolist()
    off = [0, *cut, kept]
    offsets = torch.tensor(off, dtype=torch.int32, device="cuda")
    a, b = operand(g, rows, K, ENDS[0][0]), operand(g, E * N, K, ENDS[0][1])
    y = nv.fp8_gemm_experts(a, b, offsets, out_dtype=dtype)
    A, B = values(a), values(b).view(E, N, K)
    for e in range(E):
        if off[e] < off[e + 1]:
            check(y[off[e]: off[e + 1]], A[off[e]: off[e + 1]], B[e], dtype)
    assert bool((y[kept:] == 0).all())
    slots = rows // 128 + E
    d, c = operand(g, N, 128 * slots, ENDS[1][0]), operand(g, K, 128 * slots, ENDS[1][1])
    dw = nv.fp8_gemm_experts_dw(d, c, offsets, out_dtype=dtype, rows=rows)
    D, C = values(d), values(c)
    for e in range(E):
        first, n = 128 * (off[e] // 128 + e), -(-(off[e + 1] - off[e]) // 128) * 128
        check(dw[e], D[:, first: first + n], C[:, first: first + n], dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M, N, K", SIZES)
def test_the_least_and_the_largest_tensors(M, N, K, dtype):
    # a type's lowest value, as masks hold it, against small weights: the product is finite; and a tensor of binary32's least magnitudes against large ones
    g = torch.Generator(device="cuda").manual_seed(M + N)
    x, w = torch.randn(M, K, generator=g, device="cuda"), torch.randn(N, K, generator=g, device="cuda")
    big, small = x.bfloat16(), (w * 2.0 ** -30).bfloat16()
    big[torch.rand(M, K, generator=g, device="cuda") < 0.01] = torch.finfo(torch.bfloat16).min
    a, b = nv.fp8_quantize(big)[0], nv.fp8_quantize(small)[0]
    assert int(a.scales.max()) == 247
    check(nv.fp8_gemm(a, b, out_dtype=dtype), values(a), values(b), dtype)
    a, b = nv.fp8_quantize(x * 2.0 ** -127)[0], nv.fp8_quantize(w * 2.0 ** 122)[0]
    assert int(a.scales.max()) < 3 and int(a.codes.view(torch.uint8).max()) > 0
    check(nv.fp8_gemm(a, b, out_dtype=dtype), values(a), values(b), dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M, N, K", SIZES)
def test_a_scale_that_is_no_number(M, N, K, dtype):
    # byte 255 on either side: its row or column alone
    g = torch.Generator(device="cuda").manual_seed(M * N)
    a, b = operand(g, M, K, (120, 127)), operand(g, N, K, (120, 127))
    a.codes.view(torch.uint8).clamp_(min=1)
    b.codes.view(torch.uint8).clamp_(min=1)
    ref = nv.fp8_gemm(a, b, out_dtype=dtype)
    a.scales[K // 128 - 1, M // 2] = 255
    b.scales[0, N - 2] = 255
    out = nv.fp8_gemm(a, b, out_dtype=dtype)
    bad = torch.zeros(M, N, dtype=torch.bool, device="cuda")
    bad[M // 2], bad[:, N - 2] = True, True
    assert torch.equal(out.isnan(), bad)
    A, B = values(a), values(b)
    A[M // 2], B[N - 2] = 0, 0
    check(torch.where(bad, 0, out), A, B, dtype)
    assert bool(ref.isfinite().all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M, N, K", SIZES)
def test_blocks_of_zeros_change_no_other_row(M, N, K, dtype):
    # their byte is 0 as that of the least magnitudes is, and the rows beside them have the same bits
    g = torch.Generator(device="cuda").manual_seed(M + K)
    a, b = operand(g, M, K, (120, 127)), operand(g, N, K, (120, 127))
    ref = nv.fp8_gemm(a, b, out_dtype=dtype)
    rows = torch.rand(M, generator=g, device="cuda") < 0.3
    rows[0] = True
    a.codes.view(torch.uint8)[rows] = 0
    a.scales[:, rows] = 0
    out = nv.fp8_gemm(a, b, out_dtype=dtype)
    assert bool((out[rows] == 0).all()) and torch.equal(out[~rows], ref[~rows])


@pytest.mark.parametrize("M, N, K", SIZES)
def test_the_least_tensors_against_ordinary_ones(M, N, K):
    # of blocks under 2^-118, whose codes pass bf16's least, a product with magnitudes up to 224 may be off by 2^-126
    g = torch.Generator(device="cuda").manual_seed(M + 2 * N)
    a, b = operand(g, M, K, (0, 1, 2, 120)), operand(g, N, K, (110, 120, 126))
    out, A, B = nv.fp8_gemm(a, b, out_dtype=torch.float32), values(a), values(b)
    most = (K / 32 + K / 128 + 48) * (2.0 ** -24 * (A.abs() @ B.abs().t()) + 2.0 ** -149) + K * 2.0 ** -126
    assert bool(((out.double() - A @ B.t()).abs() <= most).all())
