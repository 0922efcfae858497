"""Long sums of sbw_token_logprobs: rows of one term that is no sum of few powers of two, repeated through the whole
row, where the roundings of a running sum all go the same way.

Such a row has a closed form: k columns of value m, V - k of value m - D, so with t = exp(-D / tau)
Z = k + (V - k) t, H = ln Z + (V - k) t (D / tau) / Z and log p = -ln Z or -D / tau - ln Z.  Tolerances are those that the
header states: log p within 8e-6 + 2^-21 (H + |log p|), H within 16e-6 (1 + H); Z is within that of ln Z, 8e-6 + 2^-21 H,
relative."""
import math

import numpy as np
import pytest
import torch

import paper_2609_03844_b200 as sbw
from gpu_util import KEY, require_gpu

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def check(dev, dtype, V, top, step, tau, n=0, marked=False, column=None, every=None):
    """Rows of `top` in one column, or in one of `every` columns, and `top - step` in the others."""
    column = V // 3 if column is None else column
    x = torch.full((2, V), top - step, dtype=dtype, device=dev)
    x[:, column::every or V] = top
    k, other = len(range(column, V, every or V)), column - 1 if column else 1
    assert float(x[0, other]) == top - step and float(x[0, column]) == top      # both are values of the type
    tokens = torch.tensor([column, other], dtype=torch.int32, device=dev)
    lp, ent, z = (torch.zeros(2, device=dev) for _ in range(3))
    alt = dict(out_top_ids=torch.zeros((2, n), dtype=torch.int32, device=dev),
               out_top_logprobs=torch.zeros((2, n), device=dev)) if n else {}
    # a delta that is lost in the logits' precision: the columns are hashed and stay what they are
    mark = dict(ctx_tokens=torch.tensor([[5], [6]], dtype=torch.int32, device=dev), key=KEY, gamma=0.5, delta=1e-30) if marked else {}
    sbw.sbw_token_logprobs(x, tokens, tau, out_logprob=lp, out_entropy=ent, out_sumexp=z, **alt, **mark)
    tau = float(np.float32(tau))
    d = step / tau
    Z = k + (V - k) * math.exp(-d)
    H = math.log(Z) + (V - k) * math.exp(-d) * d / Z
    off = {"Z": (abs(float(z[0]) / Z - 1), 8e-6 + 2.0 ** -21 * H), "H": (abs(float(ent[0]) - H), 16e-6 * (1 + H))}
    for i, want in enumerate((-math.log(Z), -d - math.log(Z))):
        off[f"log p {i}"] = (abs(float(lp[i]) - want), 8e-6 + 2.0 ** -21 * (H + abs(want)))
    if n:
        assert int(alt["out_top_ids"][0, 0]) == column
        off["alternative"] = (abs(float(alt["out_top_logprobs"][0, 0]) + math.log(Z)), 8e-6 + 2.0 ** -21 * (H + math.log(Z)))
    assert all(err <= tol for err, tol in off.values()), off


@pytest.mark.parametrize("marked", [False, True])
@pytest.mark.parametrize("V", [1 << 17, 1 << 18, 1 << 20])
def test_rows_beyond_ordinary_values(V, marked):
    """Largest values beyond 2^25 tau ln 2, which are summed as differences from it."""
    dev = require_gpu()
    for tau in (0.4, 0.48, 0.59, 0.74, 0.9):
        check(dev, F32, V, -24000000.0, 2.0, tau, marked=marked)
        check(dev, F32, V, 24000002.0, 2.0, tau, n=3, marked=marked)


@pytest.mark.parametrize("dtype,V,marked", [(F32, 1 << 25, True), (F32, 1 << 27, False), (BF16, 1 << 26, True),
                                            (BF16, 1 << 28, False)])
def test_rows_of_thousands_of_trips(dtype, V, marked):
    """Every thread meets its part of the row in 4096 trips (eight CTAs to a row with alternatives).  One column of a
    warp's vectors holds the largest value, so that the terms of all others are relative to it."""
    dev = require_gpu()
    for step in (2.5, 1.375, 2.1875, 0.71875):
        check(dev, dtype, V, 1.0, step, 1.0, n=1, marked=marked, column=0, every=128 if dtype == F32 else 256)


@pytest.mark.parametrize("column", [0, 1, 70000, 262143])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_the_largest_value_in_any_trip(dtype, column):
    """Trips before the largest value are kept with another reference than those after it."""
    dev = require_gpu()
    for marked in (False, True):
        for n in (0, 2):
            check(dev, dtype, 1 << 18, 1.0, 2.5, 1.0, n=n, marked=marked, column=column)
            check(dev, dtype, 1 << 18, 1.0, 2.5, 0.25, n=n, marked=marked, column=column)
