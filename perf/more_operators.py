"""The operators that stand between the products of a mixture-of-experts block, and its products with packed 4-bit weights, as a
program that trains or serves one calls them through ``paper_2505_19115_amd.binding``, each beside its plain form.

Kinds of case
  route        router logits to each token's experts and their weights.
  route_grad   the gradient of the logits: of the experts' weights, of the balance loss and of the logits' size.
  balance      both losses, the pairs of each expert and the experts' mean probabilities.
  norm         rows normalised (with or without their mean taken off), scaled, shifted; with the rows' statistics.
  norm_grad    its gradient with respect to rows, weight and (where there is one) bias.
  w4           bf16 or binary32 activations against a packed 4-bit weight: out = g sum_k x c s.
  w4_experts   the same with a weight for each expert, tokens gathered into the experts' order.

The operators, in full.  Route: the k largest logits, ties to the lower expert; an expert at -inf is never chosen (-1, weight 0 in
its place); weights exp(l - lse), lse over the row or, renormalised, over the chosen.  Balance: N tokens have a logit above -inf, f[e]
= pairs of e / (N k), P[e] = mean of softmax(row)[e] over these; losses (E sum f P, mean of lse^2); counts holds the pairs and then N.
Norm: h = (x - m) r, m the row's mean (or 0), r = 1 / sqrt(mean (x - m)^2 + eps), out = h w + b.  Packed weight of [N, K]: codes [N, K / 2] (two
E2M1 numbers a byte, the even one low), a scale byte per block of K (E4M3, or E8M0), one binary32 scale g.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
FORMATS = {"nvfp4": (16, "e4m3"), "mxfp4": (32, "e8m0"), "e4m3_32": (32, "e4m3"), "e4m3_64": (64, "e4m3"), "e4m3_128": (128, "e4m3")}
EPS = 1e-5


def listed():
    return [
        # a decode step's routing: 16 sequences, two of 8 experts each; launches and host work are everything
        dict(name="route_decode", kind="route", T=16, E=8, k=2, dtype="f32", renormalize=True, masked=False, pad=0),
        # a training batch over many experts; padding tokens, and experts that some tokens may not use
        dict(name="route_batch", kind="route", T=32768, E=128, k=8, dtype="bf16", renormalize=True, masked=True, pad=0),
        # the logits' gradient in that batch's backward pass, weights that are shares of all experts
        dict(name="route_grad", kind="route_grad", T=32768, E=128, k=8, dtype="f32", renormalize=False, masked=True, pad=0),
        # the balance of an odd batch over an odd number of experts, logits a view of wider rows
        dict(name="balance_odd", kind="balance", T=1777, E=61, k=4, dtype="f32", masked=True, pad=3),
        # and of a large one
        dict(name="balance_batch", kind="balance", T=32768, E=256, k=8, dtype="bf16", masked=False, pad=0),
        # generation: 16 rows of the 7B width before a projection
        dict(name="norm_decode", kind="norm", rows=16, cols=4096, dtype="bf16", weight="bf16", center=False, bias=False, pad=0),
        # a view with a larger row pitch and an odd number of rows and columns, binary32
        dict(name="norm_ragged", kind="norm", rows=2049, cols=2785, dtype="f32", weight="f32", center=True, bias=True, pad=64),
        # a training batch's backward pass at the 7B width
        dict(name="norm_grad", kind="norm_grad", rows=8192, cols=4096, dtype="bf16", weight="f32", center=True, bias=True, pad=0),
        # many short rows: a head's width, in a backward pass
        dict(name="norm_grad_narrow", kind="norm_grad", rows=65536, cols=96, dtype="bf16", weight="bf16", center=False, bias=False, pad=0),
        # generation of one sequence through the 7B down projection
        dict(name="w4_token", kind="w4", M=1, N=4096, K=11008, dtype="bf16", out="bf16", format="nvfp4"),
        # generation through 8 experts, 16 sequences
        dict(name="w4_experts", kind="w4_experts", T=16, k=2, E=8, N=4096, K=2048, dtype="bf16", out="bf16", format="mxfp4", drop=False),
        # a prompt of odd length through the 7B QKV projection
        dict(name="w4_prompt", kind="w4", M=777, N=12288, K=4096, dtype="bf16", out="bf16", format="nvfp4"),
    ]


def _size(rng, lo, hi):
    """Log-uniform between lo and hi."""
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def _width(rng, lo, hi):
    """Such a size; half of them a multiple of 64, as layers have them."""
    v = _size(rng, lo, hi)
    return v if rng.random() < 0.5 else max(lo, v // 64 * 64)


def draw(rng):
    kind = rng.choice(["route", "route_grad", "balance", "norm", "norm_grad", "w4", "w4", "w4", "w4_experts", "w4_experts"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    while True:
        if kind in ("route", "route_grad", "balance"):
            c = dict(kind=kind, T=_size(rng, 1, 32768), E=_size(rng, 8, 512), k=rng.randint(1, 8), dtype=dtype, masked=rng.random() < 0.5, pad=rng.choice([0, 0, 3, 8]))
            if kind != "balance":
                c["renormalize"] = rng.random() < 0.5
            if c["T"] * c["E"] <= 32768 * 128:
                return c
        elif kind in ("norm", "norm_grad"):
            c = dict(kind=kind, rows=_size(rng, 1, 65536), cols=_width(rng, 64, 16384), dtype=dtype, weight=rng.choice([dtype, "f32"]), center=rng.random() < 0.5,
                     pad=rng.choice([0, 0, 64, 3]))
            c["bias"] = c["center"] and rng.random() < 0.75
            if c["rows"] * c["cols"] <= 2048 * 8192:
                return c
        elif kind == "w4":
            name = rng.choice(["nvfp4", "nvfp4", "mxfp4", "e4m3_32", "e4m3_64", "e4m3_128"])
            step = max(32, FORMATS[name][0])
            c = dict(kind=kind, M=_size(rng, 1, 777), N=_width(rng, 64, 12288), K=_size(rng, 256, 12288) // step * step, dtype=dtype, out=rng.choice(["bf16", "f32"]), format=name)
            if c["M"] * c["N"] * c["K"] <= 777 * 12288 * 4096 // (1 if dtype == "bf16" else 2):
                return c
        else:
            name = rng.choice(["nvfp4", "nvfp4", "mxfp4", "e4m3_32", "e4m3_128"])
            step = max(32, FORMATS[name][0])
            c = dict(kind=kind, T=_size(rng, 1, 256), k=rng.randint(1, 8), E=_size(rng, 8, 64), N=_width(rng, 64, 8192), K=_size(rng, 128, 8192) // step * step, dtype=dtype,
                     out=rng.choice(["bf16", "f32"]), format=name, drop=rng.random() < 0.25)
            if c["E"] * c["N"] * c["K"] <= 16 * 2048 * 4096 and c["T"] * c["k"] * c["N"] * c["K"] <= 512 * 2048 * 4096:
                return c


# ---- inputs: router logits that favour some experts; activations N(0, 1) whose rows differ in size, gradients N(0, 1e-3) with
# 0.05 % of entries 50 times larger, norms' weights near 1; packed weights are N(0, 0.02), quantized

def _activation(g, rows, cols, dtype, pad=0):
    x = torch.randn((rows, cols + pad), generator=g, device="cuda")
    x.mul_(torch.rand((rows, 1), generator=g, device="cuda").mul_(2).sub_(1).exp_())
    return x.to(dtype)[:, :cols]


def _gradient(g, rows, cols, dtype):
    x = torch.randn((rows, cols), generator=g, device="cuda").mul_(1e-3)
    x.mul_(torch.rand((rows, cols), generator=g, device="cuda").lt_(5e-4).mul_(49.0).add_(1.0))
    return x.to(dtype)


def _logits(g, case):
    T, E = case["T"], case["E"]
    l = torch.randn((T, E + case.get("pad", 0)), generator=g, device="cuda")
    l += 0.5 * torch.randn((1, E + case.get("pad", 0)), generator=g, device="cuda")
    l = l.to(DTYPES[case["dtype"]])[:, :E]
    if case.get("masked"):  # an eighth of the experts closed to a token, a sixteenth of the tokens padding
        l.masked_fill_(torch.rand((T, E), generator=g, device="cuda") < 1 / 8, -math.inf)
        l.masked_fill_(torch.rand((T, 1), generator=g, device="cuda") < 1 / 16, -math.inf)
    return l


def _packed(w, name):
    """Codes, scale bytes and g of [N, K] in a format, to nearest."""
    block, scale = FORMATS[name]
    N, K = w.shape
    b = w.view(N, K // block, block)
    top = b.abs().amax(-1)
    if scale == "e4m3":
        g = (top.amax() / (6 * 448)).reshape(1)
        s = (top / (6 * g)).to(torch.float8_e4m3fn)
        scales, value = s.view(torch.uint8), s.float() * g
    else:
        g = torch.ones(1, device=w.device)
        exponent = torch.floor(torch.log2(top.clamp(min=1e-30))).int() - 2
        scales, value = (exponent + 127).to(torch.uint8), torch.exp2(exponent.float())
    m = (b / value.clamp(min=1e-30)[..., None]).clamp_(-6, 6)
    code = torch.bucketize(m.abs(), torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device=w.device)).to(torch.uint8)
    code |= (m < 0).to(torch.uint8) << 3
    code = code.view(N, K // 2, 2)
    return (code[..., 0] | code[..., 1] << 4).contiguous(), scales.contiguous(), g


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    S, kind = dict(case=case), case["kind"]
    dtype = DTYPES[case["dtype"]]
    if kind in ("route", "route_grad", "balance"):
        S["logits"] = _logits(g, case)
        if kind != "route":  # what the forward pass has left, and the gradients that come back
            S["experts"], S["weights"] = _route(S["logits"], case["k"], case.get("renormalize", True))
            S["losses"], S["counts"], S["probs"] = _balance(S["logits"], S["experts"])
        if kind == "route_grad":
            S["dweights"] = _gradient(g, case["T"], case["k"], torch.float32)
            S["dlosses"] = torch.tensor([1e-2, 1e-3], device="cuda") * torch.rand(2, generator=g, device="cuda")
    elif kind in ("norm", "norm_grad"):
        R, D = case["rows"], case["cols"]
        S["x"] = _activation(g, R, D, dtype, case["pad"])
        S["weight"] = (1 + 0.1 * torch.randn(D, generator=g, device="cuda")).to(DTYPES[case["weight"]])
        S["bias"] = (0.1 * torch.randn(D, generator=g, device="cuda")).to(DTYPES[case["weight"]]) if case["bias"] else None
        if kind == "norm_grad":
            S["dy"] = _gradient(g, R, D, dtype)
            _, S["mean"], S["rstd"] = _norm(S["x"], S["weight"], S["bias"], case["center"])
    else:
        N, K, E = case["N"], case["K"], case.get("E", 1)
        S["codes"], S["scales"], S["g"] = _packed(torch.randn((E * N, K), generator=g, device="cuda").mul_(0.02), case["format"])
        if kind == "w4":
            S["x"] = _activation(g, case["M"], K, dtype)
        else:  # what the sort of this batch has left
            S["x"] = _activation(g, case["T"], K, dtype)
            experts = torch.topk(_logits(g, case), case["k"], dim=1).indices
            if case["drop"]:
                experts = torch.where(torch.rand(experts.shape, generator=g, device="cuda") < 1 / 16, -1, experts)
            S["offsets"], S["order"] = _sort(experts, E)
    return S


# ---- the plain forms: elementary operations in 32 bits

def _route(logits, k, renormalize):
    l = logits.float()
    top, index = torch.sort(l, dim=1, descending=True, stable=True)
    top, index = top[:, :k], index[:, :k]
    chosen = top > -math.inf
    base = torch.where(chosen[:, :1], top[:, :1], 0)
    e = torch.exp(top - base)
    total = (e if renormalize else torch.exp(l - base)).sum(1, keepdim=True)
    return torch.where(chosen, index, -1).int(), torch.where(chosen, e / total, 0)


def _softmax(l):
    """Probabilities and lse of the rows, zeros for those without a logit; which rows have one."""
    top = l.amax(1, keepdim=True)
    kept = top > -math.inf
    base = torch.where(kept, top, 0)
    e = torch.exp(l - base)
    total = torch.where(kept, e.sum(1, keepdim=True), 1)
    return e / total, torch.where(kept, torch.log(total) + base, 0), kept


def _counts(experts, E):
    at = torch.where(experts < 0, E, experts).reshape(-1).long()
    return torch.zeros(E + 1, dtype=torch.long, device=experts.device).scatter_add_(0, at, torch.ones_like(at))[:E]


def _balance(logits, experts):
    E = logits.shape[1]
    p, lse, kept = _softmax(logits.float())
    tokens, pairs = kept.sum(), _counts(experts, E)
    n = tokens.clamp(min=1).float()
    probs = p.sum(0) / n
    f = pairs.float() / (n * experts.shape[1])
    return torch.stack([E * (f * probs).sum(), (lse * lse).sum() / n]), torch.cat([pairs, tokens[None]]).int(), probs


def _route_grad(logits, experts, dweights, renormalize, counts, dlosses):
    l, E, k = logits.float(), logits.shape[1], experts.shape[1]
    p, lse, kept = _softmax(l)
    chosen = experts >= 0
    at = experts.clamp(min=0).long()
    if renormalize:
        e = torch.where(chosen, torch.exp(l.gather(1, at) - lse), 0)
        w = e / torch.where(kept, e.sum(1, keepdim=True), 1)
    else:
        w = torch.where(chosen, p.gather(1, at), 0)
    wd = w * dweights
    s = wd.sum(1, keepdim=True)
    d = torch.zeros_like(l).scatter_add_(1, at, wd - w * s if renormalize else wd)
    if not renormalize:
        d -= p * s
    n = counts[E].clamp(min=1).float()
    f = counts[:E].float() / (n * k)
    d += dlosses[0] * E / n * p * (f - (f * p).sum(1, keepdim=True))
    return d + dlosses[1] * 2 / n * lse * p


def _norm(x, weight, bias, center):
    x = x.float()
    m = x.mean(1) if center else None
    h = x - m[:, None] if center else x
    r = 1 / torch.sqrt((h * h).mean(1) + EPS)
    y = h * r[:, None] * weight.float()
    return y if bias is None else y + bias.float(), m, r


def _norm_grad(dy, x, weight, mean, rstd):
    dy, x = dy.float(), x.float()
    h = (x if mean is None else x - mean[:, None]) * rstd[:, None]
    u = dy * weight.float()
    dx = u - h * (u * h).mean(1, keepdim=True)
    if mean is not None:
        dx = dx - u.mean(1, keepdim=True)
    return dx * rstd[:, None], (dy * h).sum(0), dy.sum(0)


def _sort(experts, E):
    ids = experts.reshape(-1)
    key, order = torch.sort(torch.where((ids >= 0) & (ids < E), ids, E), stable=True)
    return torch.searchsorted(key, torch.arange(E + 1, device=ids.device)).int(), torch.where(key < E, order, -1).int()


def _weight(codes, scales, name):
    """The numbers that a packed weight stands for, without g: [N, K]."""
    block, scale = FORMATS[name]
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], device=codes.device)
    c = grid[torch.stack([codes & 15, codes >> 4], dim=2).int()].view(codes.shape[0], -1, block)
    s = scales.view(torch.float8_e4m3fn).float() if scale == "e4m3" else torch.exp2(scales.float() - 127)
    return (c * s[..., None]).view(codes.shape[0], -1)


def _experts_product(x, w, offsets, order, k):
    """[T, K] rows gathered by order against their experts' [E, N, K]; zeros for pairs of no expert."""
    E, R = w.shape[0], order.numel()
    r = torch.arange(R, device=x.device, dtype=torch.int32)
    e = torch.searchsorted(offsets[1:].contiguous(), r, right=True)
    kept = (e < E)[:, None]
    rows = torch.where(kept, x[order.clamp(min=0) // k], 0)
    most = max(1, int((offsets[1:] - offsets[:-1]).max()))
    e = e.clamp(max=E - 1)
    at = torch.where(kept[:, 0], e * most + r - offsets[e], E * most)
    blocks = torch.zeros((E * most + 1, x.shape[1]), device=x.device)
    blocks[at] = rows
    y = torch.bmm(blocks[:-1].view(E, most, -1), w.transpose(1, 2).contiguous()).view(E * most, -1)
    return torch.where(kept, y[at.clamp(max=E * most - 1)], 0)


def _run_plain(S):
    case, kind = S["case"], S["case"]["kind"]
    if kind == "route":
        return _route(S["logits"], case["k"], case["renormalize"])
    if kind == "route_grad":
        return _route_grad(S["logits"], S["experts"], S["dweights"], case["renormalize"], S["counts"], S["dlosses"]).to(DTYPES[case["dtype"]])
    if kind == "balance":
        return _balance(S["logits"], S["experts"])
    dtype = DTYPES[case["dtype"]]
    if kind == "norm":
        y, m, r = _norm(S["x"], S["weight"], S["bias"], case["center"])
        return y.to(dtype), m, r
    if kind == "norm_grad":
        dx, dw, db = _norm_grad(S["dy"], S["x"], S["weight"], S["mean"], S["rstd"])
        w = DTYPES[case["weight"]]
        return dx.to(dtype), dw.to(w), db.to(w) if case["bias"] else None
    w, out = _weight(S["codes"], S["scales"], case["format"]), DTYPES[case["out"]]
    if kind == "w4":
        return (S["x"].float() @ w.t() * S["g"]).to(out)
    return (_experts_product(S["x"].float(), w.view(case["E"], case["N"], -1), S["offsets"], S["order"], case["k"]) * S["g"]).to(out)


# ---- the framework's operators

def _run_own(S):
    from paper_2505_19115_amd import binding as nv
    case, kind = S["case"], S["case"]["kind"]
    if kind == "route":
        return tuple(nv.moe_route(S["logits"], case["k"], renormalize=case["renormalize"]))
    if kind == "route_grad":
        return nv.moe_route_bwd(S["logits"], S["experts"], S["dweights"], renormalize=case["renormalize"], counts=S["counts"], dlosses=S["dlosses"])
    if kind == "balance":
        return tuple(nv.moe_balance(S["logits"], S["experts"]))
    if kind == "norm":
        return tuple(nv.layer_norm(S["x"], S["weight"], S["bias"], eps=EPS, center=case["center"]))
    if kind == "norm_grad":
        return tuple(nv.layer_norm_bwd(S["dy"], S["x"], S["weight"], S["mean"], S["rstd"], bias=case["bias"]))
    block, scale = FORMATS[case["format"]]
    fmt = nv.Format(block, nv.SCALE_E4M3, 1) if scale == "e4m3" else nv.Format(block, nv.SCALE_E8M0, 0)
    w = (S["codes"], S["scales"], S["g"])
    if kind == "w4":
        return nv.gemm_w4(S["x"], w, fmt, out_dtype=DTYPES[case["out"]])
    return nv.gemm_w4_experts(S["x"], w, S["offsets"], fmt, order=S["order"], top_k=case["k"], out_dtype=DTYPES[case["out"]])


def run(S):
    return _run_own(S) if own else _run_plain(S)


def work(case):
    kind = case["kind"]
    e = 2 if case["dtype"] == "bf16" else 4
    if kind in ("route", "route_grad", "balance"):
        T, E, k = case["T"], case["E"], case["k"]
        return {"bytes": T * E * e * (2 if kind == "route_grad" else 1) + T * k * (4 if kind == "balance" else 8), "flops": 0}
    if kind in ("norm", "norm_grad"):
        R, D, w = case["rows"], case["cols"], 2 if case["weight"] == "bf16" else 4
        return {"bytes": R * D * e * (2 if kind == "norm" else 3) + R * (8 if case["center"] else 4) + D * w * (1 + case["bias"] + (kind == "norm_grad")), "flops": 0}
    N, K, o = case["N"], case["K"], 2 if case["out"] == "bf16" else 4
    packed = 0.5 + 1 / FORMATS[case["format"]][0]
    if kind == "w4":
        M = case["M"]
        return {"bytes": N * K * packed + M * K * e + M * N * o, "flops": 2 * M * N * K}
    T, k = case["T"], case["k"]  # of the weights, those of the experts that tokens can reach
    return {"bytes": min(case["E"], T * k) * N * K * packed + T * K * e + T * k * (N * o + 4), "flops": 2 * T * k * N * K}


# ---- the operators in 64 bits, from their definitions

def _choose64(l, k):
    """The k largest of every row, one after the other, the lowest index of equal ones; -1 where only -inf is left."""
    rest, index = l.clone(), torch.arange(l.shape[1], device=l.device)
    out = []
    for _ in range(min(k, l.shape[1])):
        top = rest.max(dim=1, keepdim=True).values
        first = torch.where(rest == top, index, l.shape[1]).min(dim=1, keepdim=True).values
        out.append(torch.where(top == -math.inf, -1, first))
        rest.scatter_(1, first, -math.inf)
    return torch.cat(out, dim=1)


def _log_share64(l, mask):
    """log of softmax over the entries in `mask`, -inf outside; rows without one: all -inf."""
    l = torch.where(mask, l, -math.inf)
    lse = torch.logsumexp(l, dim=1, keepdim=True)
    return torch.where(lse > -math.inf, l - lse, -math.inf), lse


def exact(case, seed):
    S, kind = prepare(case, seed), case["kind"]
    if kind in ("route", "route_grad", "balance"):
        l, E, k = S["logits"].double(), case["E"], case["k"]
        share, lse = _log_share64(l, torch.ones_like(l, dtype=torch.bool))
        p = share.exp()
        there = lse > -math.inf
        n = max(1, int(there.sum()))
        if kind == "route":
            experts = _choose64(l, k)
            picked = torch.zeros((case["T"], E + 1), dtype=torch.bool, device="cuda").scatter_(1, torch.where(experts < 0, E, experts), True)[:, :E]
            w = (_log_share64(l, picked)[0].exp() if case["renormalize"] else p).gather(1, experts.clamp(min=0))
            return experts, torch.where(experts < 0, 0, w)
        experts = S["experts"].long()
        pairs = torch.bincount(experts[experts >= 0], minlength=E)
        f = pairs.double() / (n * k)
        z = torch.where(there, lse, 0)
        if kind == "balance":
            probs = p.sum(0) / n
            return torch.stack([E * (f * probs).sum(), (z ** 2).sum() / n]), torch.cat([pairs, there.sum().reshape(1)]), probs
        # by the chain rule through log shares: d share[e] / d l[i] = [e = i] - share weight of i
        up = torch.zeros((case["T"], E + 1), dtype=torch.float64, device="cuda")
        up.scatter_add_(1, torch.where(experts < 0, E, experts), S["dweights"].double())
        picked = torch.zeros((case["T"], E + 1), dtype=torch.bool, device="cuda").scatter_(1, torch.where(experts < 0, E, experts), True)[:, :E]
        w = _log_share64(l, picked)[0].exp() if case["renormalize"] else p
        d_share = w * up[:, :E]
        d = d_share - w * d_share.sum(1, keepdim=True)
        loss, size = S["dlosses"].double()
        d_share = loss * E / n * f * p
        return d + d_share - p * d_share.sum(1, keepdim=True) + size * 2 / n * z * p
    if kind in ("norm", "norm_grad"):
        x, w = S["x"].double(), S["weight"].double()
        m = x.mean(1, keepdim=True) if case["center"] else torch.zeros_like(x[:, :1])
        r = ((x - m).square().mean(1, keepdim=True) + EPS).rsqrt()
        if kind == "norm":
            y = (x - m) * r * w
            return y + S["bias"].double() if case["bias"] else y, m[:, 0] if case["center"] else None, r[:, 0]
        # the saved statistics are inputs
        m, r, dy = S["mean"].double()[:, None] if case["center"] else m, S["rstd"].double()[:, None], S["dy"].double()
        h = (x - m) * r
        dh = dy * w
        dx = r * (dh - (dh.mean(1, keepdim=True) if case["center"] else 0) - h * (dh * h).mean(1, keepdim=True))
        return dx, (dy * h).sum(0), dy.sum(0) if case["bias"] else None
    block, scale = FORMATS[case["format"]]
    def weight(rows):
        c, s = S["codes"][rows].long(), S["scales"][rows].long()
        c = torch.stack([c % 16, c // 16], dim=-1).flatten(1)
        m = c % 8
        v = torch.where(m < 2, m * 0.5, (1 + (m % 2) * 0.5) * torch.exp2((m // 2 - 1).double())) * (1 - 2 * (c // 8))
        if scale == "e4m3":
            s = torch.where(s < 8, (s % 8) * 2.0 ** -9, (1 + (s % 8) / 8.0) * torch.exp2((s // 8 - 7).double()))
        else:
            s = torch.exp2((s - 127).double())
        return v * s.repeat_interleave(block, dim=1) * S["g"].double()
    x, N = S["x"].double(), case["N"]
    if kind == "w4":
        return x @ weight(slice(0, N)).t()
    out = torch.zeros((case["T"] * case["k"], N), dtype=torch.float64, device="cuda")
    ends = S["offsets"].tolist()
    for e in range(case["E"]):
        if ends[e + 1] > ends[e]:
            out[ends[e]: ends[e + 1]] = x[S["order"][ends[e]: ends[e + 1]].long() // case["k"]] @ weight(slice(e * N, (e + 1) * N)).t()
    return out
