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


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("scheme", [0, 1])
@pytest.mark.parametrize("B,V,K,W,off", [(1, 129, 100, 1, 0), (2, 1000, 256, 4, 7), (64, 515, 128, 1, 0), (100, 257, 640, 8, 2 ** 32 - 257),
                                         (128, 384, 64, 2, 128), (130, 700, 300, 1, 0), (300, 513, 2048, 4, 1)])
def test_watermark_on_the_way_out(B, V, K, W, off, scheme, dtype):
    """The bits of the plain product followed by sbw_bias_logits."""
    require_gpu()
    import paper_2609_03844_b200 as sbw
    from paper_2609_03844_b200 import inputs

    x, w, xs, ws = codes(B, K, 1), codes(V, K, 2), scales(B, K, 3), scales(blocks(V), K, 4)
    ctx = inputs.uniform_tokens((B, W), V, seed=5).cuda()
    for ld in (V, V + 1, V + 8):
        plain, marked = (torch.full((B, ld), 7.0, dtype=dtype, device="cuda") for _ in range(2))
        sbw.sbw_head_logits(x, xs, w, ws, plain)
        sbw.sbw_bias_logits(plain, ctx, KEY, 0.25, 2.0, scheme, V=V, vocab_offset=off)
        sbw.sbw_head_logits(x, xs, w, ws, marked, ctx_tokens=ctx, key=KEY, gamma=0.25, delta=2.0, scheme=scheme, vocab_offset=off)
        assert_same_bits(host_bits(marked), host_bits(plain))
    tiny = torch.empty(B, V, dtype=dtype, device="cuda")      # a bias that is 0 in the logits' precision needs no context
    sbw.sbw_head_logits(x, xs, w, ws, tiny, ctx_tokens=ctx, delta=0.0)
    assert_same_bits(host_bits(tiny), host_bits(sbw.sbw_head_logits(x, xs, w, ws, torch.empty_like(tiny))))


def test_rows_shards_streams_and_captures():
    """Rows do not depend on each other nor on the batch's size, shards of the vocabulary are slices; calls on several streams
    and replays of a capture give the same bits."""
    require_gpu()
    import paper_2609_03844_b200 as sbw

    B, V, K = 200, 1280, 512
    x, w, xs, ws = codes(B, K, 1), codes(V, K, 2), scales(B, K, 3), scales(blocks(V), K, 4)
    all_rows = sbw.sbw_head_logits(x, xs, w, ws, torch.empty(B, V, device="cuda"))
    for lo, hi in ((0, 1), (5, 70), (100, 200)):
        part = sbw.sbw_head_logits(x[lo:hi], xs[lo:hi], w, ws, torch.empty(hi - lo, V, device="cuda"))
        assert torch.equal(part, all_rows[lo:hi])
    halves = torch.empty(B, V, device="cuda")
    sbw.sbw_head_logits(x, xs, w[:512], ws[:4], halves[:, :512])
    sbw.sbw_head_logits(x, xs, w[512:], ws[4:], halves[:, 512:])
    assert torch.equal(halves, all_rows)
    streams = [torch.cuda.Stream() for _ in range(4)]
    outs = [torch.empty(B, V, device="cuda") for _ in streams]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, o in zip(streams, outs):
            sbw.sbw_head_logits(x, xs, w, ws, o, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(o, all_rows) for o in outs)
    graph, out, out2 = torch.cuda.CUDAGraph(), torch.empty(B, V, device="cuda"), torch.empty(3, V, dtype=torch.bfloat16, device="cuda")
    with torch.cuda.graph(graph):
        sbw.sbw_head_logits(x, xs, w, ws, out)
        sbw.sbw_head_logits(x[:3], xs[:3], w, ws, out2)
    for seed in (7, 8):
        x.copy_(codes(B, K, seed))
        graph.replay()
        torch.cuda.synchronize()
        want, size = by_definition(x, xs, w, ws)
        check(out, want, size, K)
        check(out2, want[:3], size[:3], K)


def test_values_that_are_no_numbers():
    require_gpu()
    import paper_2609_03844_b200 as sbw

    B, V, K = 40, 300, 400
    x, w, xs, ws = codes(B, K, 1), codes(V, K, 2), scales(B, K, 3), scales(blocks(V), K, 4)
    want = sbw.sbw_head_logits(x, xs, w, ws, torch.empty(B, V, device="cuda"))
    x.view(torch.uint8)[3, 399] = 0x7F                        # NaN codes
    w.view(torch.uint8)[200, 0] = 0xFF
    xs[5, 1] = float("nan")
    xs[6, 0] = float("inf")
    got = sbw.sbw_head_logits(x, xs, w, ws, torch.empty(B, V, device="cuda"))
    bad = torch.zeros(B, V, dtype=torch.bool, device="cuda")
    bad[3], bad[5], bad[6], bad[:, 200] = True, True, True, True
    assert torch.equal(got[~bad], want[~bad])
    assert bool(got[3].isnan().all() and got[5].isnan().all() and got[:, 200].isnan().all()) and not bool(got[6].isfinite().any())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("R,K", [(1, 1), (1, 128), (3, 130), (128, 128), (129, 257), (200, 1000), (1000, 64), (2, 5000), (300, 384)])
def test_quantizer(R, K, block_rows, dtype):
    """Scales and codes bit for bit: both divisions are IEEE fp32, which numpy's are, and torch rounds to e4m3 to nearest even."""
    require_gpu()
    import paper_2609_03844_b200 as sbw

    g = torch.Generator().manual_seed(R + K)
    x = (torch.randn(R, K, generator=g) * torch.exp(3 * torch.randn(R, 1, generator=g))).to(dtype)
    x[0, : K // 2] = 0.0
    if R > 1:
        x[1] = 0.0
        x[R - 1, K - 1] = 2.0 ** -140 if dtype == torch.float32 else 2.0 ** -130
    pad = lambda n, b: -(-n // b) * b  # noqa: E731
    full = np.zeros((pad(R, block_rows), pad(K, 128)), np.float32)
    full[:R, :K] = x.float().numpy()
    b = full.reshape(-1, block_rows, pad(K, 128) // 128, 128)
    scale = np.maximum(np.abs(b).max((1, 3)) / np.float32(448), np.float32(2.0 ** -126))
    q = (b / scale[:, None, :, None]).reshape(full.shape)[:R, :K]
    want = torch.from_numpy(np.ascontiguousarray(np.clip(q, -448, 448))).to(torch.float8_e4m3fn).view(torch.uint8)
    for extra in (0, 1, 16):
        src = torch.full((R, K + extra), float("nan"), dtype=dtype, device="cuda")
        src[:, :K] = x.cuda()
        out = torch.full((R, K + extra), 0x55, dtype=torch.uint8, device="cuda")
        s = torch.full((-(-R // block_rows), blocks(K) + extra), 7.0, device="cuda")
        sbw.sbw_quantize_fp8(src[:, :K], out.view(E4M3)[:, :K], s[:, :blocks(K)], block_rows=block_rows)
        assert np.array_equal(s[:, :blocks(K)].cpu().numpy(), scale) and bool((s[:, blocks(K):] == 7).all())
        assert torch.equal(out[:, :K].cpu(), want) and bool((out[:, K:] == 0x55).all())


@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantizer_of_values_that_are_no_numbers(block_rows):
    require_gpu()
    import paper_2609_03844_b200 as sbw

    for bad in (float("nan"), float("inf"), -float("inf")):
        x = torch.ones(130, 300, device="cuda")
        x[2, 140] = bad
        q, s = torch.empty(130, 300, dtype=E4M3, device="cuda"), torch.empty(-(-130 // block_rows), 3, device="cuda")
        sbw.sbw_quantize_fp8(x, q, s, block_rows=block_rows)
        there = torch.zeros(130, 300, dtype=torch.bool, device="cuda")
        there[2 if block_rows == 1 else slice(0, 128), 128:256] = True
        back = q.float() * s.repeat_interleave(block_rows, 0)[:130].repeat_interleave(128, 1)[:, :300]
        assert bool(back[there].isnan().all()) and bool((back[~there] == 1).all())


def test_gradient_of_the_hidden_states():
    """d_x = d_l w is the same product with the transposed weights: against the formula, and against differences of the
    forward product in 64 bits (which is linear in x)."""
    require_gpu()
    import paper_2609_03844_b200 as sbw

    B, V, K = 24, 640, 384
    g = torch.Generator().manual_seed(4)
    w = torch.randn(V, K, generator=g).cuda() * 0.02
    wq, ws = torch.empty(V, K, dtype=E4M3, device="cuda"), torch.empty(blocks(V), blocks(K), device="cuda")
    sbw.sbw_quantize_fp8(w, wq, ws, block_rows=128)
    dl = torch.randn(B, V, generator=g).cuda()
    dq, ds = torch.empty(B, V, dtype=E4M3, device="cuda"), torch.empty(B, blocks(V), device="cuda")
    sbw.sbw_quantize_fp8(dl, dq, ds)
    dx = sbw.sbw_head_logits(dq, ds, wq.view(torch.uint8).T.contiguous().view(E4M3), ws.T.contiguous(), torch.empty(B, K, device="cuda"))
    at = torch.arange(V, device="cuda") // 128
    W = wq.double() * ws.double()[at][:, torch.arange(K, device="cuda") // 128]
    D = dq.double() * ds.double()[:, at]
    check(dx, D @ W, D.abs() @ W.abs(), V)
    x, step = torch.randn(B, K, generator=g).double().cuda(), torch.randn(B, K, generator=g).double().cuda()
    loss = lambda v: (D * (v @ W.T)).sum()  # noqa: E731
    slope = (loss(x + step) - loss(x - step)) / 2
    size = (step.abs() * (D.abs() @ W.abs())).sum()
    assert abs(float(slope - (dx.double() * step).sum())) <= (257 + blocks(V)) * 2.0 ** -24 * float(size)
    # and the quantizing itself: half an e4m3 step of every d_l (2^-4 of it, or 2^-10 of its block's scale)
    exact = dl.double() @ W
    off = 2.0 ** -4 * dl.double().abs() + 2.0 ** -10 * ds.double()[:, at]
    assert bool(((dx.double() - exact).abs() <= off @ W.abs() + (257 + blocks(V)) * 2.0 ** -24 * (D.abs() @ W.abs())).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantizer_keeps_the_sign_of_zero(block_rows, dtype):
    """-0 / scale is -0, code 0x80, whatever the scale: ordinary ones, those of blocks whose quotients are divisions (scales from
    2^90 on and below 2^-90), blocks of zeros alone; so is a negative quotient too small for a code."""
    require_gpu()
    import paper_2609_03844_b200 as sbw

    R, K = 130, 1300                                          # the last row and the last block are ragged
    x = torch.zeros(R, K)
    x[:, 1::2] = -0.0
    for kb, top in enumerate((1.0, 3.0e4, 2.0 ** 100, 2.0 ** -100, 2.0 ** -80, 0.0, 448.0, 0.7, 2.0 ** 98, 2.0 ** -82, 5.0)):
        x[:, kb * 128 + 3] = top
        x[:, kb * 128 + 5] = -top * 2.0 ** -30
        x[:, kb * 128 + 6] = top * 2.0 ** -30
    x = x.to(dtype)
    want = torch.where(torch.signbit(x), 0x80, 0).to(torch.uint8)
    want[:, 3::128] = torch.where(x[:, 3::128] > 0, 0x7E, 0).to(torch.uint8)
    for extra in (0, 1, 16):
        src = torch.zeros((R, K + extra), dtype=dtype, device="cuda")
        src[:, :K] = x.cuda()
        out = torch.full((R, K + extra), 0x55, dtype=torch.uint8, device="cuda")
        s = torch.empty(-(-R // block_rows), blocks(K), device="cuda")
        sbw.sbw_quantize_fp8(src[:, :K], out.view(E4M3)[:, :K], s, block_rows=block_rows)
        assert torch.equal(out[:, :K].cpu(), want)


@pytest.mark.parametrize("block_rows", [1, 128])
def test_quotients_next_to_the_borders_of_codes(block_rows):
    """x within two steps of what lies half-way between two codes, times the scale: where a quotient that is not the rounded one
    gives another code.  Scales over their whole range, the ends of the one in which quotients are three operations among them."""
    require_gpu()
    import paper_2609_03844_b200 as sbw

    g = torch.Generator().manual_seed(12)
    R, K = 512, 1024
    values = torch.arange(0x7F, dtype=torch.uint8).view(E4M3).float()              # 0 .. 448
    middles = ((values[1:] + values[:-1]) / 2).numpy()
    exponent = torch.randint(-118, 110, (R, K // 128), generator=g).float()
    exponent[:8] = torch.tensor([-91.0, -90, -89, -88, 88, 89, 90, 91])[:, None]
    if block_rows == 128:
        exponent = exponent[:, :].view(4, 128, -1)[:, :1].expand(4, 128, -1).reshape(R, -1)
    top = (torch.rand(R, K // 128, generator=g) + 1) * 448 * torch.exp2(exponent)
    if block_rows == 128:
        top = top.view(4, 128, -1)[:, :1].expand(4, 128, -1).reshape(R, -1)
    top = top.numpy().astype(np.float32)
    scale = top / np.float32(448)
    pick = torch.randint(0, len(middles), (R, K), generator=g).numpy()
    x = (middles[pick].astype(np.float64) * np.repeat(scale, 128, 1)).astype(np.float32)
    x = (x.view(np.int32) + torch.randint(-2, 3, (R, K), generator=g).numpy().astype(np.int32)).view(np.float32)
    x *= np.where(torch.rand(R, K, generator=g).numpy() < 0.5, np.float32(-1), np.float32(1))
    x[:, ::128] = top                                                               # the largest magnitude of its block
    assert np.all(np.abs(x) <= np.repeat(top, 128, 1))
    want = torch.from_numpy(np.clip(x / np.repeat(scale, 128, 1), -448, 448)).to(E4M3).view(torch.uint8)
    q, s = torch.empty(R, K, dtype=E4M3, device="cuda"), torch.empty(R // block_rows, K // 128, device="cuda")
    sbw.sbw_quantize_fp8(torch.from_numpy(x).cuda(), q, s, block_rows=block_rows)
    assert np.array_equal(s.cpu().numpy(), scale[::block_rows])
    assert torch.equal(q.view(torch.uint8).cpu(), want)
