"""The operators of a mixture-of-experts linear layer in 8 bits, and the 8-bit linear layer itself, as a program
that trains or serves one calls them through ``paper_2505_19115_amd.binding``, each beside its plain form.

Kinds of case
  sort           (token, choice) pairs sorted by expert: offsets, order, positions.
  route          rows moved between the tokens' order and the experts': step "gather" (a token's row to each of its
                 experts), "combine" (back, weighted and summed), "combine_bwd" (gradient of the latter).
  quantize       a tensor to E4M3 codes with one power-of-two scale per 128 elements, along its rows, its columns or both.
  linear         an activation quantized and multiplied with a packed weight.
  train          one linear layer, forward and backward, from tensors: six quantized operands, three products.
  experts        serving: sort, activations gathered and quantized, every expert's product, results combined.
  experts_train  the same layer's forward product and its gradients with respect to tokens and experts' weights.

The operators, in full.  Quantized operand of an [R, K] tensor: with P the next multiple of 128 of K, codes [R, P]
(zero past K) and scale bytes [P / 128, R]; for a block's largest magnitude a, the scale is 2^(byte - 127) with the
smallest exponent that keeps a <= 448 * scale (byte 0 at the least), the code E4M3(x / scale), ties to even.
Product: out[i, j] = sum over blocks of scaleA * scaleB * sum of code products.  Sort: stable, by expert; an expert
outside 0 .. E-1 drops its pair (position -1), order is -1 past the last kept pair.  Rows of a product past the last kept
pair are zero.
"""
import math

import torch

own = False

BLOCK = 128
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # a decode step's routing: 16 sequences, two of 8 experts each; launches and host work are everything
        dict(name="sort_decode", kind="sort", T=16, k=2, E=8, drop=False),
        # a training batch over many experts, some tokens beyond their expert's capacity and dropped
        dict(name="sort_batch", kind="sort", T=32768, k=8, E=128, drop=True),
        # tokens to their experts in binary32 with an odd width, some dropped
        dict(name="gather_odd", kind="route", step="gather", T=1777, k=4, E=16, D=1027, dtype="f32", drop=True),
        # experts' results back to the tokens, a training batch of the 7B width
        dict(name="combine", kind="route", step="combine", T=8192, k=2, E=8, D=4096, dtype="bf16", drop=False),
        # and its gradient
        dict(name="combine_grad", kind="route", step="combine_bwd", T=8192, k=2, E=8, D=4096, dtype="bf16", drop=False),
        # the output gradient of the 7B down projection's input, wanted along both axes
        dict(name="quantize_both", kind="quantize", rows=4096, cols=11008, sides="both", dtype="bf16", pad=0),
        # a view with a larger row pitch and an odd number of rows and columns, binary32
        dict(name="quantize_ragged", kind="quantize", rows=2049, cols=2785, sides="rows", dtype="f32", pad=64),
        # generation through the 7B gate projection, 16 sequences
        dict(name="linear_decode", kind="linear", M=16, N=11008, K=4096, dtype="bf16", out="bf16"),
        # a prompt of odd length through the 7B QKV projection
        dict(name="linear_prompt", kind="linear", M=777, N=12288, K=4096, dtype="bf16", out="bf16"),
        # the 7B down projection in a training step of 4096 tokens
        dict(name="train_down", kind="train", M=4096, N=4096, K=11008, dtype="bf16", out="bf16"),
        # generation through 8 experts, 8 sequences
        dict(name="experts_decode", kind="experts", T=8, k=2, E=8, D=4096, F=2048, dtype="bf16", out="bf16", drop=False),
        # a training batch through 16 experts
        dict(name="experts_train", kind="experts_train", T=8192, k=2, E=16, D=2048, F=4096, dtype="bf16", out="bf16", drop=False),
    ]


def _size(rng, lo, hi):
    """Log-uniform between lo and hi."""
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def _width(rng, lo, hi):
    """Such a size; half of them a multiple of 64, as layers have them."""
    v = _size(rng, lo, hi)
    return v if rng.random() < 0.5 else max(lo, v // 64 * 64)


MOST_PRODUCTS = 3 * 4096 * 4096 * 11008  # multiply-adds of the largest listed case
MOST_MOVED = 2 * 8192 * 4096             # elements moved by the largest routing case


def draw(rng):
    kind = rng.choice(["sort", "route", "route", "quantize", "linear", "linear", "train", "experts", "experts", "experts_train"])
    dtype, out = rng.choice(["bf16", "bf16", "f32"]), rng.choice(["bf16", "bf16", "f32"])
    drop = rng.random() < 0.25
    while True:
        if kind == "sort":
            c = dict(kind=kind, T=_size(rng, 1, 32768), k=rng.randint(1, 8), E=_size(rng, 8, 256), drop=drop)
            return c
        if kind == "route":
            c = dict(kind=kind, step=rng.choice(["gather", "combine", "combine_bwd"]), T=_size(rng, 1, 16384), k=rng.randint(1, 8),
                     E=_size(rng, 8, 64), D=_width(rng, 64, 8192), dtype=dtype, drop=drop)
            if c["T"] * c["k"] * c["D"] <= MOST_MOVED * (2 if dtype == "bf16" else 1) // 2:
                return c
        elif kind == "quantize":
            c = dict(kind=kind, rows=_size(rng, 1, 16384), cols=_width(rng, 64, 16384), sides=rng.choice(["rows", "cols", "both"]), dtype=dtype,
                     pad=rng.choice([0, 0, 64, 3]))
            if c["rows"] * c["cols"] <= 4096 * 11008:
                return c
        elif kind in ("linear", "train"):
            c = dict(kind=kind, M=_size(rng, 1 if kind == "linear" else 16, 8192), N=_width(rng, 64, 12288), K=_width(rng, 64, 12288), dtype=dtype, out=out)
            if (3 if kind == "train" else 1) * c["M"] * c["N"] * c["K"] <= MOST_PRODUCTS:
                return c
        else:
            c = dict(kind=kind, T=_size(rng, 1 if kind == "experts" else 32, 8192), k=rng.randint(1, 8), E=_size(rng, 8, 64), D=_width(rng, 128, 4096),
                     F=_width(rng, 128, 4096), dtype=dtype, out=out, drop=drop)
            tokens = 3 * c["T"] * c["k"] + (64 * c["E"] if kind == "experts_train" else 0)
            if tokens * c["D"] * c["F"] <= MOST_PRODUCTS // 4 and c["E"] * c["D"] * c["F"] <= 16 * 2048 * 4096:
                return c


# ---- inputs: activations N(0, 1) whose rows differ in size, weights N(0, 0.02), gradients N(0, 1e-3) with 0.05 % of entries
# 50 times larger; experts chosen as the k largest of router logits that favour some experts

def _activation(g, rows, cols, dtype, pad=0):
    x = torch.randn((rows, cols + pad), generator=g, device="cuda")
    x.mul_(torch.rand((rows, 1), generator=g, device="cuda").mul_(2).sub_(1).exp_())
    return x.to(dtype)[:, :cols]


def _gradient(g, rows, cols, dtype):
    x = torch.randn((rows, cols), generator=g, device="cuda").mul_(1e-3)
    x.mul_(torch.rand((rows, cols), generator=g, device="cuda").lt_(5e-4).mul_(49.0).add_(1.0))
    return x.to(dtype)


def _router(g, case):
    T, k, E = case["T"], case["k"], case["E"]
    logits = torch.randn((T, E), generator=g, device="cuda") + 0.5 * torch.randn((1, E), generator=g, device="cuda")
    top = torch.topk(logits, k, dim=1)
    experts = top.indices
    if case["drop"]:
        experts = torch.where(torch.rand((T, k), generator=g, device="cuda") < 1 / 16, -1, experts)
    return experts.contiguous(), torch.softmax(top.values, dim=1)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    S, kind = dict(case=case), case["kind"]
    dtype = DTYPES[case["dtype"]] if "dtype" in case else None
    if "E" in case:
        S["experts"], S["weights"] = _router(g, case)
    if kind == "route":  # what the sort of this batch has left
        T, k, D = case["T"], case["k"], case["D"]
        S["offsets"], S["order"], S["position"] = _sort(S["experts"], case["E"])
        if case["step"] != "combine":
            S["x"] = _activation(g, T, D, dtype)
        if case["step"] != "gather":
            S["y"] = _activation(g, T * k, D, dtype)
    elif kind == "quantize":
        S["x"] = _activation(g, case["rows"], case["cols"], dtype, case["pad"])
    elif kind in ("linear", "train"):
        M, N, K = case["M"], case["N"], case["K"]
        S["x"] = _activation(g, M, K, dtype)
        w = torch.randn((N, K), generator=g, device="cuda").mul_(0.02).to(dtype)
        if kind == "linear":  # the packed weight that a serving program loads
            S["w_codes"], S["w_scales"] = _quantize(w)
        else:
            S["w"], S["dy"] = w, _gradient(g, M, N, dtype)
    elif kind in ("experts", "experts_train"):
        T, k, E, D, F = (case[n] for n in ("T", "k", "E", "D", "F"))
        S["x"] = _activation(g, T, D, dtype)
        w = torch.randn((E, F, D), generator=g, device="cuda").mul_(0.02).to(dtype)
        if kind == "experts":
            S["w_codes"], S["w_scales"] = _quantize(w.view(E * F, D))
        else:
            S["w"], S["dy"] = w, _gradient(g, T * k, F, dtype)  # the gradient of the products, in the experts' order
    return S


# ---- the plain forms: elementary operations in 32 bits

def _padded(n):
    return -(-n // BLOCK) * BLOCK


def _quantize(x):
    """Row blocks of [R, K]: codes [R, P], scale bytes [P / 128, R]."""
    R, K = x.shape
    b = torch.zeros((R, _padded(K)), dtype=torch.float32, device=x.device)
    b[:, :K] = x
    b = b.view(R, -1, BLOCK)
    fraction, exponent = torch.frexp(b.abs().amax(-1))  # magnitude = fraction * 2^exponent, 448 = 0.875 * 2^9
    byte = (exponent - 9 + (fraction > 0.875).int() + 127).clamp(0, 254)
    byte = torch.where(fraction == 0, 0, byte)
    codes = (b * ((254 - byte) << 23).view(torch.float32)[..., None]).to(torch.float8_e4m3fn)
    return codes.view(R, -1), byte.t().to(torch.uint8).contiguous()


def _values(codes, scales):
    """The numbers that a quantized operand stands for, [R, P]."""
    s = (scales.t().int() << 23).contiguous().view(torch.float32)
    return (codes.float().view(codes.shape[0], -1, BLOCK) * s[..., None]).view(codes.shape)


def _sort(experts, E):
    n = experts.numel()
    ids = experts.reshape(-1)
    key, order = torch.sort(torch.where((ids >= 0) & (ids < E), ids, E), stable=True)
    offsets = torch.searchsorted(key, torch.arange(E + 1, device=ids.device)).int()
    slots = torch.arange(n, device=ids.device, dtype=torch.int32)
    position = torch.empty(n, dtype=torch.int32, device=ids.device)
    position[order] = torch.where(key < E, slots, -1)
    return offsets, torch.where(key < E, order, -1).int(), position.view(experts.shape)


def _gathered(x, order, k):
    return torch.where((order >= 0)[:, None], x.float()[order.clamp(min=0) // k], 0)


def _combined(y, position, weights):
    rows = torch.where((position >= 0)[..., None], y.float()[position.clamp(min=0)], 0)
    return (rows if weights is None else rows * weights[..., None]).sum(1)


def _combine_gradient(dout, y, weights, position, offsets):
    T, k = position.shape
    kept = position >= 0
    at = position.clamp(min=0)
    dout = dout.float()[:, None, :]
    dy = torch.zeros((y.shape[0] + 1, y.shape[1]), dtype=torch.float32, device=y.device)
    dy[torch.where(kept, position, y.shape[0]).view(-1)] = (dout * weights[..., None]).view(T * k, -1)
    dweights = torch.where(kept, (dout * y.float()[at]).sum(-1), 0)
    return dy[:-1], dweights


def _by_expert(rows, offsets, length):
    """The experts' rows of [R, C], each expert's padded with zeros to `length`: [E, length, C]; and every row's place."""
    E = offsets.numel() - 1
    r = torch.arange(rows.shape[0], device=rows.device, dtype=torch.int32)
    e = torch.searchsorted(offsets[1:].contiguous(), r, right=True)
    kept = e < E
    e = e.clamp(max=E - 1)
    at = torch.where(kept, e * length + r - offsets[e], E * length)
    block = torch.zeros((E * length + 1, rows.shape[1]), dtype=torch.float32, device=rows.device)
    block[at] = rows.float()
    return block[:-1].view(E, length, -1), at, kept


def _longest(offsets):
    return max(1, int((offsets[1:] - offsets[:-1]).max()))


def _experts_product(a, w, offsets):
    """[R, K] rows against their experts' [E, N, K]."""
    blocks, at, kept = _by_expert(a, offsets, _longest(offsets))
    y = torch.bmm(blocks, w.transpose(1, 2).contiguous()).view(-1, w.shape[1])
    return torch.where(kept[:, None], y[torch.where(kept, at, 0)], 0)


def _experts_gradient(a, b, offsets):
    """Each expert's sum over its rows r of a[r] (x) b[r], both quantized along r in blocks that start at its first row: [E, A, B]."""
    length, E = _padded(_longest(offsets)), offsets.numel() - 1
    a = _by_expert(a, offsets, length)[0].transpose(1, 2).reshape(-1, length)
    b = _by_expert(b, offsets, length)[0].transpose(1, 2).reshape(-1, length)
    a, b = _values(*_quantize(a)).view(E, -1, length), _values(*_quantize(b)).view(E, -1, length)
    return torch.bmm(a, b.transpose(1, 2).contiguous())


def _run_plain(S):
    case, kind = S["case"], S["case"]["kind"]
    if kind == "sort":
        return _sort(S["experts"], case["E"])
    dtype = DTYPES[case["dtype"]]
    if kind == "route":
        if case["step"] == "gather":
            return _gathered(S["x"], S["order"], case["k"]).to(dtype)
        if case["step"] == "combine":
            return _combined(S["y"], S["position"], S["weights"]).to(dtype)
        dy, dweights = _combine_gradient(S["x"], S["y"], S["weights"], S["position"], S["offsets"])
        return dy.to(dtype), dweights
    if kind == "quantize":
        return [_quantize(S["x"]) if case["sides"] != "cols" else None, _quantize(S["x"].t()) if case["sides"] != "rows" else None]
    out = DTYPES[case["out"]]
    if kind == "linear":
        return (_values(*_quantize(S["x"])) @ _values(S["w_codes"], S["w_scales"]).t()).to(out)
    if kind == "train":
        x, w, dy = S["x"], S["w"], S["dy"]
        y = _values(*_quantize(x)) @ _values(*_quantize(w)).t()
        dx = _values(*_quantize(dy)) @ _values(*_quantize(w.t())).t()
        dw = _values(*_quantize(dy.t())) @ _values(*_quantize(x.t())).t()
        return y.to(out), dx.to(out), dw.to(out)
    E, D, F = case["E"], case["D"], case["F"]
    offsets, order, position = _sort(S["experts"], E)
    rows = _gathered(S["x"], order, case["k"])
    if kind == "experts":
        y = _experts_product(_values(*_quantize(rows)), _values(S["w_codes"], S["w_scales"]).view(E, F, -1), offsets)
        return _combined(y, position, S["weights"]).to(out)
    w, dy = S["w"], S["dy"]
    y = _experts_product(_values(*_quantize(rows)), _values(*_quantize(w.view(E * F, D))).view(E, F, -1), offsets)
    dxs = _experts_product(_values(*_quantize(dy)), _values(*_quantize(w.transpose(1, 2).reshape(E * D, F))).view(E, D, -1), offsets)
    return y.to(out), _combined(dxs, position, None).to(out), _experts_gradient(dy, rows, offsets).to(out)


# ---- the framework's operators

def _run_own(S):
    from paper_2505_19115_amd import binding as nv
    case, kind = S["case"], S["case"]["kind"]
    if kind == "sort":
        return tuple(nv.moe_sort(S["experts"], case["E"]))
    if kind == "route":
        if case["step"] == "gather":
            return nv.moe_gather(S["x"], S["order"], case["k"])
        if case["step"] == "combine":
            return nv.moe_combine(S["y"], S["position"], S["weights"])
        return nv.moe_combine_bwd(S["x"], S["y"], S["weights"], S["position"], S["offsets"])
    if kind == "quantize":
        q = nv.fp8_quantize(S["x"], rows=case["sides"] != "cols", cols=case["sides"] != "rows")
        return [side and (side.codes, side.scales) for side in q]
    out = DTYPES[case["out"]]
    if kind == "linear":
        a, _ = nv.fp8_quantize(S["x"])
        return nv.fp8_gemm(a, nv.Fp8(S["w_codes"], S["w_scales"]), out_dtype=out)
    if kind == "train":
        x, xt = nv.fp8_quantize(S["x"], cols=True)
        w, wt = nv.fp8_quantize(S["w"], cols=True)
        y = nv.fp8_gemm(x, w, out_dtype=out)
        dy, dyt = nv.fp8_quantize(S["dy"], cols=True)
        return y, nv.fp8_gemm(dy, wt, out_dtype=out), nv.fp8_gemm(dyt, xt, out_dtype=out)
    E, k = case["E"], case["k"]
    offsets, order, position = nv.moe_sort(S["experts"], E)
    if kind == "experts":
        a, _ = nv.fp8_quantize(S["x"], order=order, top_k=k)
        y = nv.fp8_gemm_experts(a, nv.Fp8(S["w_codes"], S["w_scales"]), offsets, out_dtype=out)
        return nv.moe_combine(y, position, S["weights"])
    x, xt = nv.fp8_quantize(S["x"], cols=True, order=order, top_k=k, offsets=offsets)
    w, wt = nv.fp8_quantize(S["w"], cols=True)
    y = nv.fp8_gemm_experts(x, w, offsets, out_dtype=out)
    dy, dyt = nv.fp8_quantize(S["dy"], cols=True, offsets=offsets)
    dx = nv.moe_combine(nv.fp8_gemm_experts(dy, wt, offsets, out_dtype=out), position)
    return y, dx, nv.fp8_gemm_experts_dw(dyt, xt, offsets, out_dtype=out)


def run(S):
    return _run_own(S) if own else _run_plain(S)


def work(case):
    kind = case["kind"]
    packed = 1 + 1 / BLOCK  # bytes per element of a quantized operand
    if kind == "sort":
        return {"bytes": case["T"] * case["k"] * (8 + 4 + 4) + 4 * (case["E"] + 1), "flops": 0}
    e = 2 if case["dtype"] == "bf16" else 4
    if kind == "route":
        T, k, D = case["T"], case["k"], case["D"]
        rows = {"gather": T + T * k, "combine": T + T * k, "combine_bwd": T + 2 * T * k}[case["step"]]
        return {"bytes": rows * D * e + T * k * {"gather": 4, "combine": 8, "combine_bwd": 12}[case["step"]], "flops": 0}
    if kind == "quantize":
        return {"bytes": case["rows"] * case["cols"] * (e + packed * (2 if case["sides"] == "both" else 1)), "flops": 0}
    o = 2 if case["out"] == "bf16" else 4
    if kind in ("linear", "train"):
        M, N, K = case["M"], case["N"], case["K"]
        if kind == "linear":
            return {"bytes": M * K * e + N * K * packed + M * N * o, "flops": 2 * M * N * K}
        return {"bytes": (M * K + N * K + M * N) * (e + o), "flops": 6 * M * N * K}
    T, k, E, D, F = (case[n] for n in ("T", "k", "E", "D", "F"))
    if kind == "experts":  # of the weights, those of the experts that tokens can reach
        return {"bytes": T * k * 12 + T * D * e + min(E, T * k) * D * F * packed + T * F * o, "flops": 2 * T * k * D * F}
    return {"bytes": T * k * 8 + (T * D + E * D * F) * (e + o) + T * k * F * (e + o), "flops": 6 * T * k * D * F}


# ---- the operators in 64 bits, from their definitions

def _two_to(e):
    """2^e in binary64, exactly."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _e4m3(v):
    """The nearest number of the E4M3 grid, ties to even, magnitudes up to 448."""
    exponent = torch.frexp(v.abs().clamp(min=2.0 ** -6)).exponent - 1
    return torch.round(v * _two_to(3 - exponent)) * _two_to(exponent - 3)


def _blocked64(x):
    """Codes, scale exponents and values of the rows of a binary64 tensor, blocks along its last axis."""
    R, K = x.shape
    P = -(-K // 128) * 128
    b = torch.cat([x, x.new_zeros(R, P - K)], dim=1).reshape(R, P // 128, 128)
    largest = b.abs().max(dim=-1, keepdim=True).values
    e = torch.ceil(torch.log2(largest / 448.0)).clamp(-126, 127)  # off by one at most, where the quotient is next to a power of two
    e = torch.where(largest <= 448.0 * _two_to(e - 1), e - 1, torch.where(largest > 448.0 * _two_to(e), e + 1, e))
    e = torch.where(largest == 0, -127, e)
    codes = _e4m3(b * _two_to(-e))
    return codes.reshape(R, P), (e[..., 0] + 127).t(), (codes * _two_to(e)).reshape(R, P)[:, :K]


def _groups64(experts, E):
    """For each expert the flat (token, choice) indices that chose it, in order."""
    flat = experts.reshape(-1)
    return [torch.nonzero(flat == e).reshape(-1) for e in range(E)]


def exact(case, seed):
    S = prepare(case, seed)
    kind = case["kind"]
    if kind == "sort":
        return None
    if kind == "route":
        T, k, D = case["T"], case["k"], case["D"]
        if case["step"] == "gather":
            out = torch.zeros((T * k, D), dtype=torch.float64, device="cuda")
            picked = torch.cat(_groups64(S["experts"], case["E"]))
            out[: picked.numel()] = S["x"].double()[picked // k]
            return out
        groups = torch.cat(_groups64(S["experts"], case["E"]))
        place = torch.arange(groups.numel(), device="cuda")
        if case["step"] == "combine":
            out = torch.zeros((T, D), dtype=torch.float64, device="cuda")
            return out.index_add_(0, groups // k, S["y"].double()[place] * S["weights"].double().reshape(-1)[groups][:, None])
        dy = torch.zeros((T * k, D), dtype=torch.float64, device="cuda")
        up = S["x"].double()[groups // k]
        dy[place] = up * S["weights"].double().reshape(-1)[groups][:, None]
        dw = torch.zeros(T * k, dtype=torch.float64, device="cuda")
        dw[groups] = (up * S["y"].double()[place]).sum(-1)
        return dy, dw.view(T, k)
    if kind == "quantize":
        x = S["x"].double()
        sides = [_blocked64(x)[:2] if case["sides"] != "cols" else None, _blocked64(x.t().contiguous())[:2] if case["sides"] != "rows" else None]
        return [side and (side[0], None) for side in sides]
    if kind == "linear":  # the packed weight is an input
        w = S["w_codes"].double() * _two_to(S["w_scales"].t().long() - 127).repeat_interleave(128, dim=1)
        return _blocked64(S["x"].double())[2] @ w[:, : case["K"]].t()
    if kind == "train":
        x, w, dy = S["x"].double(), S["w"].double(), S["dy"].double()
        q = lambda t: _blocked64(t)[2]  # noqa: E731
        c = lambda t: _blocked64(t.t().contiguous())[2]  # noqa: E731
        return q(x) @ q(w).t(), q(dy) @ c(w).t(), c(dy) @ c(x).t()
    T, k, E, D, F = (case[n] for n in ("T", "k", "E", "D", "F"))
    groups = _groups64(S["experts"], E)
    q = lambda t: _blocked64(t)[2]  # noqa: E731
    x = S["x"].double()
    if kind == "experts":
        w = S["w_codes"].double() * _two_to(S["w_scales"].t().long() - 127).repeat_interleave(128, dim=1)
        w = w[:, :D].reshape(E, F, D)
        out = torch.zeros((T, F), dtype=torch.float64, device="cuda")
        for e, picked in enumerate(groups):
            if picked.numel():
                out.index_add_(0, picked // k, (q(x[picked // k]) @ w[e].t()) * S["weights"].double().reshape(-1)[picked][:, None])
        return out
    y = torch.zeros((T * k, F), dtype=torch.float64, device="cuda")
    dx = torch.zeros((T, D), dtype=torch.float64, device="cuda")
    dw = torch.zeros((E, F, D), dtype=torch.float64, device="cuda")
    at = 0
    for e, picked in enumerate(groups):
        n = picked.numel()
        if n:
            xe, we, dye = x[picked // k], S["w"][e].double(), S["dy"][at: at + n].double()
            y[at: at + n] = q(xe) @ q(we).t()
            dx.index_add_(0, picked // k, q(dye) @ q(we.t().contiguous()).t())
            dw[e] = q(dye.t().contiguous()) @ q(xe.t().contiguous()).t()
        at += n
    return y, dx, dw
