"""The 8-bit projection to the vocabulary and its quantiser on the GPU, against the definition in 64 bits.

Tolerances.  A product of two e4m3 codes is exact in fp32 (8 significant bits).  A block's sum of 128 products and the
blocks' sum are fp32: with S = sum_kb |xs ws| sum_k |x w| the largest sum of magnitudes of a logit, a block's sum is off by at
most 128 units of 2^-23 (chopped additions allowed for), the product of the two scales by 2^-24, and every step over the
blocks by 2^-24 of the running sum: at most (128 * 2 + 1 + blocks) 2^-24 S.  A bf16 logit is rounded once more: 2^-8.
"""
import numpy as np
import pytest
import torch

from gpu_util import KEY, assert_same_bits, host_bits, require_gpu

pytestmark = pytest.mark.gpu

E4M3 = torch.float8_e4m3fn


def blocks(n):
    return -(-n // 128)


def codes(rows, K, seed, pad=16):
    """Random finite e4m3 codes, rows on 16-byte boundaries, the padding behind a row NaN codes."""
    g = torch.Generator().manual_seed(seed)
    ld = -(-K // 16) * 16 + pad
    c = torch.full((rows, ld), 0x7F, dtype=torch.uint8)
    v = torch.randint(0, 0x7F, (rows, K), generator=g, dtype=torch.uint8) | torch.randint(0, 2, (rows, K), generator=g, dtype=torch.uint8) << 7
    c[:, :K] = v
    return c.cuda().view(E4M3)[:, :K]


def scales(rows, K, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.exp(2 * torch.randn(rows, blocks(K), generator=g)).cuda()


def by_definition(x, xs, w, ws):
    """Logits in 64 bits and the sums of magnitudes that the tolerance is in."""
    K, V = x.shape[1], w.shape[0]
    at = torch.arange(K, device="cuda") // 128
    X = x.double() * xs.double()[:, at]
    W = w.double() * ws.double()[torch.arange(V, device="cuda") // 128][:, at]
    return X @ W.T, X.abs() @ W.abs().T


def check(got, want, size, K):
    tol = (257 + blocks(K)) * 2.0 ** -24 * size
    if got.dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * (want.abs() + tol)
    off = (got.double() - want).abs() - tol
    assert bool((off <= 0).all()), f"off by {float(off.max())} more than allowed at {divmod(int(off.argmax()), want.shape[1])}"


SIZES = [(1, 1, 1), (1, 128, 128), (3, 129, 127), (8, 1000, 130), (17, 127, 512), (64, 500, 1000), (127, 257, 300),
         (128, 640, 256), (129, 300, 129), (200, 1025, 640), (256, 256, 2048), (1, 20000, 1024), (513, 700, 1300), (1, 130, 9000)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,V,K", SIZES)
def test_head_is_the_product(B, V, K, dtype):
    require_gpu()
    import paper_2609_03844_b200 as sbw

    x, w, xs, ws = codes(B, K, 1), codes(V, K, 2), scales(B, K, 3), scales(blocks(V), K, 4)
    want, size = by_definition(x, xs, w, ws)
    for ld in (V, V + 3, V + 8):
        full = torch.full((B, ld), 7.0, dtype=dtype, device="cuda")
        out = sbw.sbw_head_logits(x, xs, w, ws, full[:, :V] if ld > V else full)
        check(out, want, size, K)
        assert bool((full[:, V:] == 7).all())
    at_odd = torch.empty(B * V + 1, dtype=dtype, device="cuda")[1:].view(B, V)      # starts on an element, no more
    assert torch.equal(sbw.sbw_head_logits(x, xs, w, ws, at_odd), out)
