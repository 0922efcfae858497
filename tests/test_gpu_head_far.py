"""The 8-bit projection, its quantiser and the sampler from given random numbers on rows whose offsets pass 32 bits: the bits that rows
next to each other give."""
import pytest
import torch

import paper_2609_03844_b200 as sbw
from paper_2609_03844_b200 import inputs
from gpu_util import KEY, require_gpu
from test_gpu_head import E4M3, blocks, codes, scales

pytestmark = pytest.mark.gpu


def apart(t, stride):
    """The same rows, `stride` elements apart."""
    R, n = t.shape
    far = torch.empty((R - 1) * stride + n, dtype=t.dtype, device="cuda").as_strided((R, n), (stride, 1))
    far.copy_(t)
    return far


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("ahead", [0, 1])                     # the paths for aligned rows and the others
def test_rows_of_logits(dtype, ahead):
    require_gpu()
    B, V, K, stride = 3, 1500, 300, 2 ** 31 + 8 + ahead
    x, w, xs, ws = codes(B, K, 1), codes(V, K, 2), scales(B, K, 3), scales(blocks(V), K, 4)
    ctx = inputs.uniform_tokens((B, 2), V, seed=5).cuda()
    mark = dict(ctx_tokens=ctx, key=KEY, gamma=0.25, delta=2.0)
    want = sbw.sbw_head_logits(x, xs, w, ws, torch.empty(B, V, dtype=dtype, device="cuda"), **mark)
    far = apart(torch.zeros_like(want), stride)
    assert torch.equal(sbw.sbw_head_logits(x, xs, w, ws, far, **mark), want)
    u, t = torch.full((B,), 0.7, device="cuda"), torch.full((B,), 3000.0, device="cuda")
    for extra in ({}, mark):
        ids = [sbw.sbw_sample_given(l, u, torch.empty(B, dtype=torch.int32, device="cuda"), temperature=t, **extra) for l in (want, far)]
        assert torch.equal(*ids)


def test_rows_of_operands_and_scales():
    require_gpu()
    B, V, K = 3, 3, 300
    x, w, xs, ws = codes(B, K, 1), codes(V, K, 2), scales(B, K, 3), scales(blocks(V), K, 4)
    new = lambda: torch.empty(B, V, device="cuda")  # noqa: E731
    want = sbw.sbw_head_logits(x, xs, w, ws, new())
    byte = lambda t: apart(t.view(torch.uint8), 2 ** 32 + 16).view(E4M3)  # noqa: E731
    assert torch.equal(sbw.sbw_head_logits(byte(x), xs, w, ws, new()), want)
    assert torch.equal(sbw.sbw_head_logits(x, apart(xs, 2 ** 31 + 1), w, ws, new()), want)
    assert torch.equal(sbw.sbw_head_logits(x, xs, byte(w), ws, new()), want)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("ahead", [0, 1])
def test_rows_of_the_quantizer(ahead, block_rows, dtype):
    require_gpu()
    R, K = 3, 600
    x = inputs.logits_normal(R, K, 3.0, dtype, seed=1).cuda()
    S = -(-R // block_rows)
    out = lambda: (torch.empty(R, K, dtype=E4M3, device="cuda"), torch.empty(S, blocks(K), device="cuda"))  # noqa: E731
    q, s = sbw.sbw_quantize_fp8(x, *out(), block_rows=block_rows)
    far_q = apart(torch.zeros(R, K, dtype=torch.uint8, device="cuda"), 2 ** 32 + 16 + ahead).view(E4M3)
    far_s = apart(torch.zeros(S, blocks(K), device="cuda"), 2 ** 30 + 1)
    sbw.sbw_quantize_fp8(apart(x, 2 ** 31 + 8 + ahead), far_q, far_s, block_rows=block_rows)
    assert torch.equal(far_q.contiguous().view(torch.uint8), q.view(torch.uint8)) and torch.equal(far_s, s)


def test_more_elements_than_31_bits_count():
    """Rows next to each other, 2^31 elements and some: the last rows against a call on them alone."""
    require_gpu()
    R, K = 2 ** 31 // 4096 + 129, 4096
    x = torch.zeros(R, K, dtype=torch.bfloat16, device="cuda")
    x[-200:] = inputs.logits_normal(200, K, 3.0, torch.bfloat16, seed=1).cuda()
    q, s = torch.empty(R, K, dtype=E4M3, device="cuda"), torch.empty(R, K // 128, device="cuda")
    sbw.sbw_quantize_fp8(x, q, s)
    q1, s1 = torch.empty(200, K, dtype=E4M3, device="cuda"), torch.empty(200, K // 128, device="cuda")
    sbw.sbw_quantize_fp8(x[-200:], q1, s1)
    assert torch.equal(q[-200:].view(torch.uint8), q1.view(torch.uint8)) and torch.equal(s[-200:], s1)
    first = (R - 1) // 128 * 128                              # the last tile, whose rows begin there
    t = torch.empty(-(-R // 128), K // 128, device="cuda")
    sbw.sbw_quantize_fp8(x, q, t, block_rows=128)
    q2, t2 = torch.empty(R - first, K, dtype=E4M3, device="cuda"), torch.empty(1, K // 128, device="cuda")
    sbw.sbw_quantize_fp8(x[first:], q2, t2, block_rows=128)
    assert torch.equal(q[first:].view(torch.uint8), q2.view(torch.uint8)) and torch.equal(t[-1:], t2)
