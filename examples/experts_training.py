"""A mixture-of-experts MLP trained with the 8-bit operators: tokens sorted by expert, gathered into quantized operands, each
expert's products, and the results back with their weights -- forward and backward.

    python examples/experts_training.py [steps]

Every product of the layer, forward and backward, runs on E4M3 operands with a scale per 128 elements; the weights, the
activations between the layers and the router stay in the precision they have.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2505_19115_amd import binding as nv


class ExpertsLinear(torch.autograd.Function):
    """Rows in the experts' order times their experts' weights [E, N, K].  x: [T, K] with order (gathered here, top_k rows a token), or rows
    that are in that order already (order None)."""

    @staticmethod
    def forward(ctx, x, weight, offsets, order, position, top_k):
        a, a_cols = nv.fp8_quantize(x, cols=True, order=order, top_k=top_k, offsets=offsets)
        w, w_cols = nv.fp8_quantize(weight, cols=True)
        ctx.a_cols, ctx.w_cols, ctx.offsets, ctx.position = a_cols, w_cols, offsets, position if order is not None else None
        ctx.dtype = x.dtype
        return nv.fp8_gemm_experts(a, w, offsets, out_dtype=x.dtype)

    @staticmethod
    def backward(ctx, dy):
        dy, dy_cols = nv.fp8_quantize(dy.contiguous(), cols=True, offsets=ctx.offsets)
        dx = nv.fp8_gemm_experts(dy, ctx.w_cols, ctx.offsets, out_dtype=ctx.dtype)
        if ctx.position is not None:
            dx = nv.moe_combine(dx, ctx.position)  # a token's gradient: the sum over its experts
        return dx, nv.fp8_gemm_experts_dw(dy_cols, ctx.a_cols, ctx.offsets, out_dtype=ctx.dtype), None, None, None, None


class Combine(torch.autograd.Function):
    @staticmethod
    def forward(ctx, y, weights, position, offsets):
        ctx.save_for_backward(y, weights, position, offsets)
        return nv.moe_combine(y, position, weights)

    @staticmethod
    def backward(ctx, dout):
        y, weights, position, offsets = ctx.saved_tensors
        return (*nv.moe_combine_bwd(dout.contiguous(), y, weights, position, offsets), None, None)


class Experts(torch.nn.Module):
    """SwiGLU experts: out[t] = sum over the token's top_k experts of weight * down(silu(gate(x)) * up(x))."""

    def __init__(self, experts: int, top_k: int, width: int, hidden: int, dtype=torch.bfloat16, device="cuda"):
        super().__init__()
        self.top_k = top_k
        self.router = torch.nn.Linear(width, experts, bias=False, dtype=torch.float32, device=device)
        make = lambda n, k: torch.nn.Parameter(torch.randn(experts, n, k, device=device).mul_(k ** -0.5).to(dtype))  # noqa: E731
        self.gate_up, self.down = make(2 * hidden, width), make(width, hidden)  # (gate over up: one gather, one product)

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        top = torch.topk(self.router(x.float()), self.top_k, dim=1)
        weights = torch.softmax(top.values, dim=1)
        offsets, order, position = nv.moe_sort(top.indices, self.down.shape[0])
        g, u = ExpertsLinear.apply(x, self.gate_up, offsets, order, position, self.top_k).chunk(2, dim=1)
        y = ExpertsLinear.apply(torch.nn.functional.silu(g) * u, self.down, offsets, None, None, 1)
        return Combine.apply(y, weights, position, offsets)


def train(steps: int = 20, tokens: int = 512, experts: int = 8, top_k: int = 2, width: int = 256, hidden: int = 512) -> list[float]:
    """Fits a fixed random map; the loss of each step."""
    torch.manual_seed(0)
    layer = Experts(experts, top_k, width, hidden)
    x = torch.randn(tokens, width, device="cuda", dtype=torch.bfloat16)
    target = torch.randn(tokens, width, device="cuda")
    optimizer = torch.optim.Adam(layer.parameters(), lr=2e-3)
    losses = []
    for _ in range(steps):
        loss = (layer(x).float() - target).square().mean()
        optimizer.zero_grad()
        loss.backward()
        optimizer.step()
        losses.append(loss.item())
    return losses


if __name__ == "__main__":
    for step, loss in enumerate(train(int(sys.argv[1]) if len(sys.argv) > 1 else 20)):
        print(f"step {step}: loss {loss:.4f}")
