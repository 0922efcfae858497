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


def test_the_check_of_an_address(dbg):  # noqa: F811
    """The check itself, on the host: 5 rows of 7 elements, 9 apart, at 4096."""
    import ctypes

    require_gpu()
    dbg.sbw_debug_lies_in_rows.argtypes = [ctypes.c_int64] * 3 + [ctypes.c_int] + [ctypes.c_int64] * 3
    for size in (1, 2, 4):
        for n in (1, 4, 7, 8):
            for row in (-1, 0, 1, 4, 5):
                for col in range(9):
                    at = 4096 + (row * 9 + col) * size
                    assert dbg.sbw_debug_lies_in_rows(at, n, 4096, size, 5, 7, 9) == int(0 <= row < 5 and col + n <= 7)
                    assert size == 1 or dbg.sbw_debug_lies_in_rows(at + 1, n, 4096, size, 5, 7, 9) == 0
    far = 3 * (1 << 33)
    assert dbg.sbw_debug_lies_in_rows(4096 + 4 * far, 7, 4096, 4, 4, 7, 1 << 33) == 1
    assert dbg.sbw_debug_lies_in_rows(4096 + 4 * far, 7, 4096, 4, 3, 7, 1 << 33) == 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("delta,scheme", [(0.0, 0), (2.0, 0), (2.0, 1)])
@pytest.mark.parametrize("B,V,K,ld", [(1, 1, 1, 1), (3, 130, 100, 133), (64, 515, 64, 516), (130, 300, 256, 304), (260, 515, 400, 515)])
def test_every_access_of_the_head_is_checked(dbg, B, V, K, ld, delta, scheme, dtype):  # noqa: F811
    """Stores of at most 2 (fp32) or 4 (bf16) logits; at least a hidden-state scale per row and block, and a weight scale per 128
    columns and block."""
    require_gpu()
    x, w, xs, ws = codes(B, K, 1), codes(V, K, 2), scales(B, K, 3), scales(blocks(V), K, 4)
    ctx = inputs.uniform_tokens((B, 2), V + 5, seed=5).cuda()
    results = []
    for L in (sbw.lib(), dbg):
        out = torch.full((B, ld), 7.0, dtype=dtype, device="cuda")
        L.sbw_head_logits.argtypes = sbw.lib().sbw_head_logits.argtypes
        _flags(dbg)
        assert L.sbw_head_logits(x.data_ptr(), x.stride(0), xs.data_ptr(), xs.stride(0), w.data_ptr(), w.stride(0), ws.data_ptr(),
                                 ws.stride(0), B, V, K, out.data_ptr(), 0 if dtype == torch.float32 else 1, ld, 0, ctx.data_ptr(), 2,
                                 KEY, 0.25, delta, scheme, None) == 0
        torch.cuda.synchronize()
        results.append(out)
    mask, failures, passed, _ = _flags(dbg)
    stores = B * -(-V // (2 if dtype == torch.float32 else 4))
    assert mask == 0 and failures == 0 and passed >= stores + (B + blocks(V)) * blocks(K)
    assert torch.equal(*results)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("delta,scheme", [(0.0, 0), (2.0, 0), (2.0, 1)])
@pytest.mark.parametrize("B,V,skew", [(1, 1, 0), (2, 9, 1), (5, 4099, 3), (200, 1003, 2), (3, 30001, 0), (2, 151937, 1)])
@pytest.mark.parametrize("kind", ["spread", "equal", "narrow", "large", "zeros"])
def test_every_access_of_the_sampler_is_checked(dbg, B, V, skew, kind, delta, scheme, dtype):  # noqa: F811
    """A vector of 16 bytes is one checked access, and so is an element of a row's ragged ends; then the token, the probability
    and the settings.  Rows that go through lists, splits of bins, candidates of one value and, in bf16, each of the two ways."""
    require_gpu()
    full = inputs.logits_normal(B, V + skew, 3.0, torch.float32, seed=V)
    full = {"spread": full, "equal": full * 0 + 1.5, "narrow": 1e-5 * full + 3, "large": 200 * full, "zeros": -full.abs().floor()}[kind].to(dtype).cuda()
    x = full[:, skew:]
    ctx = inputs.uniform_tokens((B, 1), V + 1, seed=6).cuda()
    u, t, p = torch.rand(B, device="cuda"), torch.ones(B, device="cuda"), torch.full((B,), 0.9, device="cuda")
    k = torch.full((B,), max(1, V // 2), dtype=torch.int32, device="cuda")
    results = []
    for L in (sbw.lib(), dbg):
        ids, prob, kept = torch.empty(B, dtype=torch.int32, device="cuda"), torch.empty(B, device="cuda"), torch.empty(B, dtype=torch.int32, device="cuda")
        L.sbw_sample_given.argtypes = sbw.lib().sbw_sample_given.argtypes
        _flags(dbg)
        assert L.sbw_sample_given(x.data_ptr(), 0 if dtype == torch.float32 else 1, B, V, full.stride(0), 0, ctx.data_ptr(), 1, KEY, 0.25,
                                  delta, scheme, u.data_ptr(), t.data_ptr(), k.data_ptr(), p.data_ptr(), None, ids.data_ptr(),
                                  prob.data_ptr(), kept.data_ptr(), None) == 0
        torch.cuda.synchronize()
        results.append((ids, prob, kept))
    mask, failures, passed, _ = _flags(dbg)
    assert mask == 0 and failures == 0 and passed >= B * (-(-V // (16 // dtype.itemsize)) + 3)
    assert all(torch.equal(a, b) for a, b in zip(*results))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("R,K,ld", [(1, 1, 1), (3, 130, 131), (129, 257, 272), (200, 1000, 1000), (2, 5000, 5008), (300, 384, 385)])
def test_every_access_of_the_quantizer_is_checked(dbg, R, K, ld, block_rows, dtype):  # noqa: F811
    """Loads and stores of at most 16 bytes of values, and a store per scale."""
    require_gpu()
    x = inputs.logits_normal(R, ld, 3.0, dtype, seed=R).cuda()
    results = []
    for L in (sbw.lib(), dbg):
        q = torch.full((R, ld), 0x55, dtype=torch.uint8, device="cuda")
        s = torch.full((-(-R // block_rows), blocks(K)), 7.0, device="cuda")
        L.sbw_quantize_fp8.argtypes = sbw.lib().sbw_quantize_fp8.argtypes
        _flags(dbg)
        assert L.sbw_quantize_fp8(x.data_ptr(), 0 if dtype == torch.float32 else 1, R, K, ld, block_rows, q.data_ptr(), ld, s.data_ptr(),
                                  s.stride(0), None) == 0
        torch.cuda.synchronize()
        results.append((q, s))
    mask, failures, passed, _ = _flags(dbg)
    assert mask == 0 and failures == 0 and passed >= 2 * R * -(-K // (16 // dtype.itemsize)) + s.numel()
    assert all(torch.equal(a, b) for a, b in zip(*results))
