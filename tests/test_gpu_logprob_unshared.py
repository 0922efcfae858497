"""sbw_token_logprobs where every CTA takes whole rows, several in turn and several trips each, against the oracle: with
the hash that is from four rows per SM on, without it from two.  Odd row lengths, so that the alignment changes from
row to row; some rows padded.  Tolerances as in test_gpu_logprob."""
import pytest
import torch

import paper_2609_03844_b200 as sbw
from paper_2609_03844_b200 import inputs
from gpu_util import KEY, require_gpu
from test_gpu_logprob import check, tokens_of

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def batch(B, V, dtype, dev):
    x = inputs.logits_normal(B, V, 4.0, dtype, seed=B + V, device=dev)
    x[:, V // 2] = 25.0                                  # half of the rows' tokens rank behind it ...
    t = tokens_of(B, V, B, dev)
    t[::2] = x[::2].float().argmax(1).to(torch.int32)    # ... the others are it
    x[1::5, V // 3:V // 3 + 3000] = float("-inf")
    t[3::7] = -1
    t[B - 1] = V
    return x, t


@pytest.mark.parametrize("scheme", [sbw.SCHEME_CONTEXT, sbw.SCHEME_SELFSALT])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,V,n", [(700, 9001, 0), (1300, 9001, 20), (600, 36007, 3)])
def test_watermarked(oracle, B, V, n, dtype, scheme):
    dev = require_gpu()
    x, t = batch(B, V, dtype, dev)
    ctx = inputs.uniform_tokens((B, 2), V, 4, dev)
    check(oracle, x, t, 0.7, n, ctx=ctx, key=KEY, gamma=0.25, delta=2.0, scheme=scheme, vocab_offset=11)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,V,n", [(500, 20011, 0), (500, 20011, 20), (250, 73013, 5), (230, 140009, 0)])
def test_plain(oracle, B, V, n, dtype):
    dev = require_gpu()
    x, t = batch(B, V, dtype, dev)
    check(oracle, x, t, 1.0, n)
