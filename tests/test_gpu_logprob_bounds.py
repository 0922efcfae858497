"""The bounds-flag build checks single columns of the log-probability kernels as it checks vectors: rows too short to hold a
vector, whose logits and gradients are all single columns, and the passes of one column at a time."""
import pytest
import torch

from paper_2609_03844_b200 import binding, inputs
from gpu_util import KEY, require_gpu
from test_gpu_logprob_owed import _flags, dbg  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,most", [(torch.float32, 3), (torch.bfloat16, 7)])
@pytest.mark.parametrize("delta", [0.0, 2.0])
def test_every_single_column_is_checked(dbg, dtype, most, delta):  # noqa: F811
    dev = require_gpu()
    code = 0 if dtype == torch.float32 else 1
    for B in (1, 5):
        for V in range(1, most + 1):
            x = inputs.logits_normal(B, V, 3.0, dtype, seed=V, device=dev)
            t = inputs.uniform_tokens((B,), V, 5, dev)
            ctx = inputs.uniform_tokens((B, 1), 1000, 6, dev)
            lp, m, z = (torch.zeros(B, device=dev) for _ in range(3))
            g, grad = torch.ones(B, device=dev), torch.full_like(x, 9.0)
            head = (x.data_ptr(), code, B, V, V, 0, ctx.data_ptr(), 1, KEY, 0.25, delta, 0, 1.0, t.data_ptr())
            _flags(dbg)
            assert dbg.sbw_token_logprobs(*head, 0, lp.data_ptr(), None, None, m.data_ptr(), z.data_ptr(), None, None, None) == 0
            torch.cuda.synchronize()
            mask, failures, passed, _ = _flags(dbg)
            assert mask == 0 and failures == 0 and passed >= B * (V + 2)       # columns, the token's own value by
            assert dbg.sbw_token_logprobs_backward(*head, m.data_ptr(), z.data_ptr(), None, g.data_ptr(), None,  # every thread, output
                                                   grad.data_ptr(), V, None) == 0
            torch.cuda.synchronize()
            mask, failures, passed, _ = _flags(dbg)
            assert mask == 0 and failures == 0 and passed == 2 * B * V         # each read and written once
            assert float((grad - 9.0).abs().min()) > 1.0


def test_the_passes_of_single_columns(dbg):  # noqa: F811
    """Rows of very large values, of many equal values and with a token of -inf: read again column by column."""
    dev = require_gpu()
    B, V = 9, 5003
    x = torch.full((B, V), -1e9, device=dev)
    x[1::3] = 1.25
    x[2::3] = float("-inf")
    t = inputs.uniform_tokens((B,), V, 5, dev)
    f = lambda *s: torch.zeros(*s, device=dev)           # noqa: E731
    lp, ent, z, rank = f(B), f(B), f(B), torch.zeros(B, dtype=torch.int32, device=dev)
    ids, tops = torch.zeros((B, 5), dtype=torch.int32, device=dev), f(B, 5)
    _flags(dbg)
    assert dbg.sbw_token_logprobs(x.data_ptr(), 0, B, V, V, 0, None, 1, KEY, 0.25, 0.0, 0, 1.0, t.data_ptr(), 5, lp.data_ptr(),
                                  ent.data_ptr(), rank.data_ptr(), None, z.data_ptr(), ids.data_ptr(), tops.data_ptr(), None) == 0
    torch.cuda.synchronize()
    mask, failures, passed, _ = _flags(dbg)
    assert mask == 0 and failures == 0 and passed > B * V                      # the row's own pass is a quarter of that
    assert torch.equal(ids.cpu(), torch.arange(5, dtype=torch.int32).expand(B, 5)) and torch.equal(rank, t + 1)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,V,delta", [(600, 36007, 2.0), (230, 140009, 0.0), (1, 600011, 2.0)])
def test_rows_of_more_than_sixteen_trips(dbg, B, V, delta, dtype):  # noqa: F811
    """No access outside, and the bits of the release build."""
    dev = require_gpu()
    x = inputs.logits_normal(B, V, 3.0, dtype, seed=V, device=dev)
    t = inputs.uniform_tokens((B,), V, 5, dev)
    t[::4] = -1 if B > 1 else 7
    ctx = inputs.uniform_tokens((B, 2), V, 6, dev)
    results = []
    for L in (dbg, binding.lib()):
        for scheme in (0, 1):
            for n in (0, 7):
                f = [torch.zeros(B, device=dev) for _ in range(4)]
                rank, ids = torch.zeros(B, dtype=torch.int32, device=dev), torch.zeros((B, 7), dtype=torch.int32, device=dev)
                _flags(dbg)
                lp, ent, m, z = (v.data_ptr() for v in f)
                assert L.sbw_token_logprobs(x.data_ptr(), int(dtype == torch.bfloat16), B, V, V, 0, ctx.data_ptr(), 2, KEY, 0.25,
                                            delta, scheme, 1.0, t.data_ptr(), n, lp, ent, rank.data_ptr(), m, z,
                                            ids.data_ptr() if n else None, None, None) == 0
                torch.cuda.synchronize()
                results.append([*f, rank, ids])
                if L is dbg:
                    mask, failures, passed, _ = _flags(dbg)
                    assert mask == 0 and failures == 0 and passed > 0
    assert all(torch.equal(a, b) for p, q in zip(results[:4], results[4:]) for a, b in zip(p, q))
