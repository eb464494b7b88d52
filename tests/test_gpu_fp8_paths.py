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
