"""Calls of the language model operators at the ends of their ranges: magnitudes next to binary32's, sums of many terms, logits far from zero,
layouts that only the C ABI makes, reports of waits that ran out."""
import numpy as np
import pytest
import torch

from paper_1805_10032_b200 import zeno

import operators_ref as R

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module", autouse=True)
def _library():
    from paper_1805_10032_b200 import build as zbuild
    zbuild.build()
    assert torch.cuda.is_available(), "these tests need a CUDA device"
    zeno.load_library()


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


@pytest.mark.parametrize("cols", [8, 132, 136, 520, 1032, 2056, 4104, 5000])
@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("saved", [False, True])
def test_layer_norm_gradient_of_large_constant_rows(cols, act, saved):
    """Finite statistics whose product is beyond binary32 (a constant row of 2^112: mean rstd is 2^120 and more; eps 2^-16 to 2^-96): columns that no
    entry of the row has must not reach its averages.  h is zero in such a row, so dx = rstd (g - avg(g)) and dweight is zero."""
    g = _gen(cols)
    m, n = 2, 19
    x = torch.full((m, n, cols), 2.0 ** 112, device="cuda").to(act)
    mean = torch.full((m, n), 2.0 ** 112, device="cuda")
    rstd = (2.0 ** torch.linspace(8, 48, n, device="cuda").round()).expand(m, n).contiguous()
    dy = torch.randn(m, n, cols, generator=g, device="cuda").to(act)
    w = 1 + 0.2 * torch.randn(cols, generator=g, device="cuda")
    source = zeno.pack_activations(x) if saved else x
    dw, db = torch.full((m, cols), NAN, device="cuda"), torch.full((m, cols), NAN, device="cuda")
    dx = zeno.layer_norm_gradient(dy, source, w, mean, rstd, dw, db)
    want = R.norm_gradient(dy, x, w, mean, rstd)
    # the slacks without what stands for the rounding of x - mean, which is exact here
    g64 = dy.double() * w.double()
    size = rstd.double().unsqueeze(-1) * (g64.abs() + g64.abs().mean(-1, keepdim=True))
    R.assert_near(dx, want[0], (cols / 32 + 40) * R.U * size, "dx")
    assert torch.equal(dw, torch.zeros_like(dw))
    R.assert_near(db, want[2], want[5], "db")
