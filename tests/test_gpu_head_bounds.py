"""The 8-bit projection and the sampler from given random numbers in the bounds-flag build: awkward sizes pass every check
and give the bits of the release build."""
import pytest
import torch

import paper_2609_03844_b200 as sbw
from paper_2609_03844_b200 import inputs
from gpu_util import KEY, require_gpu
from test_gpu_head import blocks, codes, scales
from test_gpu_logprob_owed import _flags, dbg  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("delta", [0.0, 2.0])
@pytest.mark.parametrize("B,V,K,ld", [(1, 1, 1, 1), (3, 130, 100, 133), (127, 257, 300, 257), (130, 300, 256, 304), (260, 515, 64, 515)])
def test_head(dbg, B, V, K, ld, delta, dtype):  # noqa: F811
    require_gpu()
    x, w, xs, ws = codes(B, K, 1), codes(V, K, 2), scales(B, K, 3), scales(blocks(V), K, 4)
    ctx = inputs.uniform_tokens((B, 2), V + 5, seed=5).cuda()
    want = torch.empty(B, ld, dtype=dtype, device="cuda").fill_(7)
    got = want.clone()
    mark = dict(ctx_tokens=ctx, key=KEY, gamma=0.25, delta=delta) if delta else {}
    sbw.sbw_head_logits(x, xs, w, ws, want[:, :V], **mark)
    _flags(dbg)
    dbg.sbw_head_logits.argtypes = sbw.lib().sbw_head_logits.argtypes
    rc = dbg.sbw_head_logits(x.data_ptr(), x.stride(0), xs.data_ptr(), xs.stride(0), w.data_ptr(), w.stride(0), ws.data_ptr(),
                             ws.stride(0), B, V, K, got.data_ptr(), 0 if dtype == torch.float32 else 1, ld, 0, ctx.data_ptr(), 2, KEY,
                             0.25, delta, 0, None)
    assert rc == 0
    torch.cuda.synchronize()
    mask, failures, passed, _ = _flags(dbg)
    assert mask == 0 and failures == 0 and passed >= B
    assert torch.equal(got, want)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("delta", [0.0, 2.0])
@pytest.mark.parametrize("B,V,skew", [(1, 1, 0), (2, 9, 1), (5, 4099, 3), (200, 1003, 2), (3, 30001, 0)])
def test_sampler(dbg, B, V, skew, delta, dtype):  # noqa: F811
    require_gpu()
    full = inputs.logits_normal(B, V + skew, 3.0, dtype, seed=V).cuda()
    x = full[:, skew:]
    ctx = inputs.uniform_tokens((B, 1), V + 1, seed=6).cuda()
    u, t, p = torch.rand(B, device="cuda"), torch.ones(B, device="cuda"), torch.full((B,), 0.9, device="cuda")
    want, got = (torch.empty(B, dtype=torch.int32, device="cuda") for _ in range(2))
    mark = dict(ctx_tokens=ctx, key=KEY, gamma=0.25, delta=delta) if delta else {}
    sbw.sbw_sample_given(x, u, want, temperature=t, top_p=p, **mark)
    _flags(dbg)
    dbg.sbw_sample_given.argtypes = sbw.lib().sbw_sample_given.argtypes
    rc = dbg.sbw_sample_given(x.data_ptr(), 0 if dtype == torch.float32 else 1, B, V, full.stride(0), 0, ctx.data_ptr(), 1, KEY, 0.25,
                              delta, 0, u.data_ptr(), t.data_ptr(), None, p.data_ptr(), None, got.data_ptr(), None, None, None)
    assert rc == 0
    torch.cuda.synchronize()
    mask, failures, _, _ = _flags(dbg)
    assert mask == 0 and failures == 0
    assert torch.equal(got, want)
