"""The 8-bit linear layer's operators at the ends of their ranges, on the GPU, against plain
implementations in 64 bits on the CPU: magnitudes where fp32 ends, many rows and tokens, what
autograd and tensors' views may hand them.

Tolerances count roundings as in test_gpu_operators.py: u = 2^-24 for each of fp32 arithmetic,
half a step for the one to the output's type.  With S roundings of a row's sums, r of the norm
has S / 2 + 4.  In dx = r (g - n mean(g n)) the last term has r three times, the sum of g h once
(S + 3) and five more: 2.5 S + 20 u of r (|g| + |n| mean|g n|) + |gh|.
"""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import paper_2608_20818_amd as prm  # noqa: E402
from paper_2608_20818_amd import operators  # noqa: E402
from test_gpu_operators import TYPES, NAMES, U, check, check_product, check_scale, eight, half, low, norm64, rand, sums  # noqa: E402

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]


@pytest.fixture(params=["native", "python"])
def path(request, monkeypatch):
    """Both ways a call can take: native code, and Python where that is not built."""
    if request.param == "python":
        monkeypatch.setattr(operators, "_native", type("none", (), {n: staticmethod(lambda *a: None) for n in (
            "quantize_rows", "quantize_cols", "int8_matmul", "int8_linear", "rms_norm")}))
    return request.param


# ---------------------------------------------------------------- magnitudes
def tall_rows(t):
    # largest values 254 2^n, a multiple of 127, up to the end of the range: every odd multiple of
    # 2^n is a border of two whole numbers there
    v = torch.tensor([254, -254, 150, 250, 253, -251, 127, 1, -3, 0, 129, 75], dtype=torch.float64)
    return torch.stack([v * s * 2.0 ** n for n in range(108, 121) for s in (1, -1)]).to(t)


@pytest.mark.parametrize("t", [torch.bfloat16, torch.float32], ids=NAMES.get)
def test_quantize_rows_near_the_ranges_end(t):
    x = tall_rows(t)
    assert torch.isfinite(x).all()
    qe, se = eight(x.double())
    for q, s in (prm.quantize_rows(x.cuda()), prm.quantize_rows(x.t().contiguous().cuda(), transpose=True)):
        assert torch.equal(q.cpu().double(), qe)
        check_scale(s, se)
    # the layer's own quantiser of rows; one-hot weights give back the values that q stands for, of
    # which a scale has 2 u and the product 4
    w = torch.eye(12, dtype=t)
    y = prm.int8_linear(x.cuda(), w.cuda()).double().cpu()
    want = qe * se[:, None]
    ok = (want * 127).abs() < 3.4e38  # the sum times the first scale, before the weight's 1 / 127, in fp32's range
    assert ok.any() and ((y - want).abs() <= 8 * U * want.abs() + half(t) * want.abs() * (1 + 1e-3))[ok].all()


def test_norm_eight_bits_of_large_products():
    # h w past 2^120 in fp32, on borders of two whole numbers; the squares of h stay in its range
    v = torch.tensor([254, 253, -251, 127, 1, -3, 0, 129, 75, -254, 249, 5], dtype=torch.float64)
    x, w = (torch.stack([v * 2.0 ** 52, v.flip(0) * 2.0 ** 50])).to(torch.bfloat16), torch.full((12,), 2.0 ** 63, dtype=torch.bfloat16)
    q, s = prm.rms_norm(x.cuda(), w.cuda(), quantize=True)
    _, r, _ = norm64(x, None, w, 1e-6, torch.bfloat16)
    qe, se = eight(x.double() * w.double())
    assert torch.equal(q.cpu().double(), qe)
    check_scale(s, se * r[:, 0], (sums(12) / 2 + 6) * U)
