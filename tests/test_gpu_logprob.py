"""sbw_token_logprobs against the fp64 oracle: sizes from one column on, every alignment, masks that leave little or
nothing, ties, special values, both schemes; and what a call owes beside its numbers (streams, graphs, untouched
memory, equal bits on equal calls).

Tolerances.  With u = 2^-24, the sums behind Z are chains of at most 48 additions (48 u), every term carries the
exponential's 2^-22 = 4 u and 3 u |d| / tau from its argument (difference, product and the rounded 1/tau), and
moving the reference up to 16 times another 5 u each.  Weighted with p, |d| / tau averages to at most the entropy H, so
ln Z is within (48 + 4 + 80) u + 3 u H < 8e-6 + 2^-21 H / 2; log p adds u |log p| for its own rounding.  The entropy
sums |d| / tau once more: (1 + H) times that, doubled for the two sums: 16e-6 (1 + H)."""
import numpy as np
import pytest
import torch

import paper_2609_03844_b200 as sbw
from paper_2609_03844_b200 import inputs
from gpu_util import KEY, host_bits, require_gpu

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def outputs(B, n, dev, fill=-7):
    f = lambda *s: torch.full(s, float(fill), dtype=F32, device=dev)       # noqa: E731
    i = lambda *s: torch.full(s, fill, dtype=torch.int32, device=dev)      # noqa: E731
    o = dict(out_logprob=f(B), out_entropy=f(B), out_rank=i(B), out_max=f(B), out_sumexp=f(B))
    if n:
        o |= dict(out_top_ids=i(B, n), out_top_logprobs=f(B, n))
    return o


def close(got, want, tol, what):
    got = got.astype(np.float64)
    # fp32 rounds what lies beyond its largest number by half a step, FLT_MAX (1 + u), to an infinity: the lowest value
    # minus the highest is -2 FLT_MAX, beyond it whatever the error
    far = np.abs(want) > np.finfo(np.float32).max * (1 + 2.0 ** -24)
    want = np.where(far, np.copysign(np.inf, want), want)
    assert np.array_equal(np.isnan(got), np.isnan(want)), (what, got, want)
    inf = np.isinf(want)
    assert np.array_equal(got[inf], want[inf]) and not np.isinf(got[~inf]).any(), (what, got, want)
    ok = np.isfinite(want)
    off = np.abs(got[ok] - want[ok]) - np.broadcast_to(tol, want.shape)[ok]
    assert off.size == 0 or off.max() <= 0, (what, off.max())


def compare(o, want, n):
    h = {k: v.cpu().numpy() for k, v in o.items()}
    H = np.nan_to_num(want["entropy"])
    lp_tol = lambda lp: 8e-6 + 2.0 ** -21 * (H.reshape(-1, *[1] * (lp.ndim - 1)) + np.abs(np.nan_to_num(lp, posinf=0, neginf=0)))  # noqa: E731
    if "out_rank" in h:
        assert np.array_equal(h["out_rank"], want["rank"])
    if "out_logprob" in h:
        close(h["out_logprob"], want["logprob"], lp_tol(want["logprob"]), "logprob")
    if "out_entropy" in h:
        close(h["out_entropy"], want["entropy"], 16e-6 * (1 + H), "entropy")
    if "out_max" in h:
        close(h["out_max"], want["max"], 0.0, "max")
    if "out_sumexp" in h:
        close(h["out_sumexp"], want["sumexp"], np.nan_to_num(want["sumexp"]) * (8e-6 + 2.0 ** -21 * H), "sumexp")
    if n:
        if "out_top_ids" in h:
            assert np.array_equal(h["out_top_ids"], want["top_ids"])
        if "out_top_logprobs" in h:
            close(h["out_top_logprobs"], want["top_logprobs"], lp_tol(want["top_logprobs"]), "top")


def check(oracle, x, tokens, tau, n=0, V=None, **mark):
    """One call on a CUDA [B, ld] tensor against the oracle; returns the outputs."""
    B, V = x.shape[0], V or x.shape[1]
    o = outputs(B, n, x.device)
    ctx = mark.pop("ctx", None)
    before = x.clone()
    sbw.sbw_token_logprobs(x, tokens, tau, V=V, ctx_tokens=ctx, **o, **mark)
    torch.cuda.synchronize()
    assert torch.equal(x.view(torch.uint8) if x.is_contiguous() else x.contiguous().view(torch.uint8),
                       before.contiguous().view(torch.uint8))               # read only
    want = oracle.token_logprobs(host_bits(x), V, tokens.cpu().numpy(), tau, n,
                                 None if ctx is None else ctx.cpu().numpy(), **mark)
    compare(o, want, n)
    return o


def tokens_of(B, V, seed, dev):
    return inputs.uniform_tokens((B,), V, seed, dev)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", [1, 2, 3, 4, 7, 8, 9, 15, 17, 31, 33, 64, 127, 255, 1000, 2047, 4099])
def test_short_rows_of_every_alignment(oracle, V, dtype):
    dev = require_gpu()
    for B, ld, n in ((1, V, 1), (3, V + 1, min(V, 5)), (9, V + 3, 20), (2, V + 8, 64), (5, V, 0)):
        full = inputs.logits_normal(B, ld, 3.0, dtype, seed=V * 31 + B, device=dev)
        check(oracle, full, tokens_of(B, V, V + B, dev), 1.0, n, V=V)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_that_start_anywhere(oracle, dtype):
    dev = require_gpu()
    for first in range(1, 9):                            # a view whose first row starts `first` columns into memory
        x = inputs.logits_normal(4, 700, 3.0, dtype, seed=first, device=dev)[:, first:]
        check(oracle, x, tokens_of(4, x.shape[1], first, dev), 0.75, 6)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,V", [(1, 32000), (2, 151936), (5, 32003), (19, 50001), (40, 32003), (75, 20011), (149, 9001),
                                 (299, 5003), (700, 2500)])
def test_batches_from_one_row_to_many(oracle, B, V, dtype):
    dev = require_gpu()
    x = inputs.logits_normal(B, V, 4.0, dtype, seed=B, device=dev)
    for n, tau in ((20, 1.0), (0, 0.7)):
        check(oracle, x, tokens_of(B, V, B + 1, dev), tau, n)


@pytest.mark.parametrize("scheme", [sbw.SCHEME_CONTEXT, sbw.SCHEME_SELFSALT])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,V,W,off", [(1, 1, 1, 0), (3, 37, 2, 5), (2, 5003, 4, 100000), (33, 4100, 8, (1 << 32) - 4100),
                                       (150, 3001, 1, 7)])
def test_watermarked(oracle, B, V, W, off, dtype, scheme):
    dev = require_gpu()
    x = inputs.logits_normal(B, V, 3.0, dtype, seed=V, device=dev)
    ctx = inputs.uniform_tokens((B, W), 1 << 30, V + 1, dev)
    for delta, n in ((2.0, min(V, 10)), (-1.5, 0), (1e-30, 3)):
        check(oracle, x, tokens_of(B, V, 3, dev), 0.7, n, ctx=ctx, key=KEY, gamma=0.25, delta=delta, scheme=scheme,
              vocab_offset=off)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B", [1, 40, 200])
def test_masks_and_special_values(oracle, dtype, B):
    dev = require_gpu()
    V = 6007
    low = torch.finfo(dtype).min
    g = torch.Generator(device=dev)
    g.manual_seed(5)
    rnd = lambda: inputs.logits_normal(B, V, 3.0, dtype, seed=int(torch.randint(1 << 20, (1,), generator=g, device=dev)),  # noqa: E731
                                       device=dev)
    rows = {}
    rows["all -inf"] = torch.full((B, V), -np.inf, dtype=dtype, device=dev)
    rows["all lowest"] = torch.full((B, V), low, dtype=dtype, device=dev)
    rows["all highest"] = torch.full((B, V), -low, dtype=dtype, device=dev)
    rows["all equal"] = torch.full((B, V), 1.25, dtype=dtype, device=dev)
    rows["zeros of both signs"] = rnd().sign() * 0.0
    rows["one finite"] = rows["all -inf"].clone()
    rows["one finite"][:, 4321] = 3.0
    for name, fill in (("ten kept, -inf", -np.inf), ("ten kept, lowest", low)):
        rows[name] = torch.full((B, V), fill, dtype=dtype, device=dev)
        rows[name][:, 100:5100:500] = rnd()[:, :10]
    rows["half masked"] = torch.where(torch.rand(B, V, generator=g, device=dev) < 0.5, rnd(), -np.inf)
    rows["lowest and highest"] = torch.where(rnd() > 0, low, -low).to(dtype)
    rows["huge"] = (rnd().float() * 1e37).to(dtype)
    rows["ascending"] = rnd().sort(1).values
    rows["descending"] = rnd().sort(1, descending=True).values
    rows["few values"] = rnd().round()
    rows["nan"] = rnd()
    rows["nan"][:, 17] = float("nan")
    rows["nan and masked"] = rows["ten kept, -inf"].clone()
    rows["nan and masked"][:, ::3] = float("nan")
    rows["all nan"] = torch.full((B, V), float("nan"), dtype=dtype, device=dev)
    rows["+inf"] = rnd()
    rows["+inf"][:, 5000] = float("inf")
    rows["subnormal"] = (torch.randint(0, 50, (B, V), generator=g, device=dev).float() * 1e-40).to(dtype)
    tok = tokens_of(B, V, 9, dev)
    for name, x in rows.items():
        for t in (tok, torch.full_like(tok, 4321)):
            try:
                check(oracle, x, t, 1.0, 20)
            except AssertionError as e:
                raise AssertionError(f"{name}: {e}") from e
    ctx = inputs.uniform_tokens((B, 1), V, 3, dev)
    for name in ("all -inf", "all equal", "ten kept, -inf", "ascending", "nan", "few values"):
        try:
            check(oracle, rows[name], tok, 1.0, 20, ctx=ctx, key=KEY, gamma=0.5, delta=2.0, scheme=1)
        except AssertionError as e:
            raise AssertionError(f"watermarked, {name}: {e}") from e


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("tau", [1e-3, 0.3, 1.0, 5.0])
def test_rows_and_masks_of_any_magnitude(oracle, dtype, tau):
    """2^(l c - round(m c)) leaves the exponent range when m c is large, whether the row's own largest value is that
    large or only the largest one that some warp meets (a run of masked columns)."""
    dev = require_gpu()
    tau = float(np.float32(tau))
    for V, B in ((300, 3), (9001, 12), (5003, 700)):
        base = inputs.logits_normal(B, V, 3.0, F32, seed=V, device=dev)
        t = tokens_of(B, V, 3, dev)
        power = torch.arange(B, device=dev)[:, None] % 29 + 3.0          # a magnitude from 1e3 to 1e31 a row
        for sign in (1.0, -1.0):
            check(oracle, (sign * base.abs() * 10.0 ** power).to(dtype), t, tau, 9)
            level = torch.full_like(base, sign) * 10.0 ** power          # equal values: entropy ln V
            check(oracle, level.to(dtype), t, tau)
            check(oracle, (level * (1 + base.abs() / 2048)).to(dtype), t, tau)
        masked = base.clone()
        masked[:, V // 2:] = (-(10.0 ** power)).expand(B, V - V // 2)
        check(oracle, masked.to(dtype), t, tau, 9)
        masked[:, :V // 2] -= 2.0 ** 25 * tau * 0.6931472                # near where ordinary values end
        check(oracle, masked.to(dtype), t, tau, 9)


def test_padded_rows(oracle):
    dev = require_gpu()
    for B, V in ((1, 5000), (30, 5000), (400, 1001)):
        x = inputs.logits_normal(B, V, 3.0, F32, seed=B, device=dev)
        t = tokens_of(B, V, 2, dev)
        t[::3] = -100
        t[1::5] = V
        t[2::7] = -2 ** 31
        x[t < 0] = float("nan")                          # nothing of a padded row counts
        check(oracle, x, t, 1.0, 5)


def test_temperatures(oracle):
    dev = require_gpu()
    x = inputs.logits_normal(12, 3001, 3.0, F32, seed=1, device=dev)
    t = tokens_of(12, 3001, 2, dev)
    for tau in (0.01, 0.3, 8.0, 1e4):
        check(oracle, x, t, float(np.float32(tau)), 3)


def test_any_set_of_outputs(oracle):
    dev = require_gpu()
    B, V = 37, 4001
    x = inputs.logits_normal(B, V, 3.0, BF16, seed=4, device=dev)
    t = tokens_of(B, V, 5, dev)
    want = oracle.token_logprobs(host_bits(x), V, t.cpu().numpy(), 1.0, 7)
    every = outputs(B, 7, dev)
    for keep in (["out_logprob"], ["out_rank"], ["out_entropy"], ["out_max", "out_sumexp"], ["out_top_ids"],
                 ["out_top_logprobs"], ["out_logprob", "out_top_ids", "out_top_logprobs"]):
        o = {k: torch.full_like(every[k], -7) for k in keep}
        sbw.sbw_token_logprobs(x, t, **o)
        compare(o, want, 7)
    o = {k: v for k, v in outputs(B, 7, dev).items() if k not in ("out_logprob", "out_rank")}
    sbw.sbw_token_logprobs(x, None, **o)                 # no tokens: every row counts
    compare(o, want, 7)


def test_no_rows_and_refusals():
    dev = require_gpu()
    x = torch.zeros((0, 100), dtype=BF16, device=dev)
    t = torch.zeros(0, dtype=torch.int32, device=dev)
    f = torch.zeros(0, dtype=F32, device=dev)
    assert sbw.sbw_token_logprobs(x, t, out_logprob=f) is f
    x = torch.zeros((2, 100), dtype=BF16, device=dev)
    t = torch.zeros(2, dtype=torch.int32, device=dev)
    f = torch.zeros(2, dtype=F32, device=dev)
    with pytest.raises(TypeError):
        sbw.sbw_token_logprobs(x, t.long(), out_logprob=f)
    with pytest.raises(TypeError):
        sbw.sbw_token_logprobs(x, t.cpu(), out_logprob=f)
    with pytest.raises(TypeError):
        sbw.sbw_token_logprobs(x.half(), t, out_logprob=f)
    with pytest.raises(ValueError):
        sbw.sbw_token_logprobs(x, t, out_logprob=torch.zeros(3, dtype=F32, device=dev))
    with pytest.raises(TypeError):
        sbw.sbw_token_logprobs(x, t, out_logprob=torch.zeros(4, dtype=F32, device=dev)[::2])
    with pytest.raises(ValueError):
        sbw.sbw_token_logprobs(x, t, out_logprob=f, V=101)
    with pytest.raises(ValueError):
        sbw.sbw_token_logprobs(x, t, out_logprob=f, delta=1.0)
    with pytest.raises(ValueError):
        sbw.sbw_token_logprobs(x, t, out_top_ids=torch.zeros((3, 2), dtype=torch.int32, device=dev))
    with pytest.raises(ValueError):
        sbw.sbw_token_logprobs(x.t(), t, out_logprob=f)
    with pytest.raises(sbw.SbwError):
        sbw.sbw_token_logprobs(x, t, 0.0, out_logprob=f)
    with pytest.raises(sbw.SbwError):
        sbw.sbw_token_logprobs(x, t)                     # nothing asked for
    with pytest.raises(sbw.SbwError):
        sbw.sbw_token_logprobs(x, t, out_top_ids=torch.zeros((2, 65), dtype=torch.int32, device=dev))


@pytest.mark.parametrize("B,V", [(1, 128256), (60, 32003), (700, 5000)])
def test_equal_calls_give_equal_bits_on_streams_and_in_graphs(B, V):
    dev = require_gpu()
    x = inputs.logits_normal(B, V, 3.0, BF16, seed=6, device=dev)
    t = tokens_of(B, V, 7, dev)
    ctx = inputs.uniform_tokens((B, 1), V, 8, dev)
    for mark in ({}, dict(ctx_tokens=ctx, key=KEY, gamma=0.5, delta=2.0)):
        first = outputs(B, 9, dev)
        sbw.sbw_token_logprobs(x, t, 0.7, **first, **mark)
        torch.cuda.synchronize()
        same = lambda o: all(torch.equal(o[k], first[k]) for k in first)   # noqa: E731
        streams, many = [torch.cuda.Stream() for _ in range(3)], [outputs(B, 9, dev) for _ in range(3)]
        torch.cuda.synchronize()
        for s, o in zip(streams, many):                  # at the same time on three streams
            sbw.sbw_token_logprobs(x, t, 0.7, stream=s, **o, **mark)
        torch.cuda.synchronize()
        assert all(same(o) for o in many)
        a, b = outputs(B, 9, dev), outputs(B, 9, dev)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            sbw.sbw_token_logprobs(x, t, 0.7, **a, **mark)
            sbw.sbw_token_logprobs(x, t, 0.7, **b, **mark)
        for _ in range(3):
            for v in (*a.values(), *b.values()):
                v.zero_()
            g.replay()
            torch.cuda.synchronize()
            assert same(a) and same(b)


def test_statistics_are_those_of_the_sampler():
    dev = require_gpu()
    B, V = 24, 32003
    for dtype in (F32, BF16):
        x = inputs.logits_normal(B, V, 3.0, dtype, seed=8, device=dev)
        ctx = inputs.uniform_tokens((B, 1), V, 9, dev)
        ids = torch.empty(B, dtype=torch.int32, device=dev)
        m, z, p = (torch.empty(B, dtype=F32, device=dev) for _ in range(3))
        ws = torch.empty(sbw.sbw_sample_workspace_bytes(B, V), dtype=torch.uint8, device=dev)
        sbw.sbw_bias_sample(x, ctx, KEY, 0.5, 2.0, 0, 0.7, 1, 2, ids, ws, out_max=m, out_sumexp=z, out_prob=p)
        o = outputs(B, 0, dev)
        sbw.sbw_token_logprobs(x, ids, 0.7, ctx_tokens=ctx, key=KEY, gamma=0.5, delta=2.0, **o)
        assert torch.equal(o["out_max"], m)
        # both within their bounds of the exact value: 1e-6 the sampler's, 8e-6 + 2^-21 H ours, H < ln V = 10.4
        assert torch.all((o["out_sumexp"] / z - 1).abs() < 1e-6 + 8e-6 + 2.0 ** -21 * 10.4)
        assert torch.all((o["out_logprob"].exp() / p - 1).abs() < 1e-6 + 8e-6 + 2.0 ** -21 * 32)


def test_rows_far_into_a_large_batch(oracle):
    dev = require_gpu()
    V, B = 131072, 17000                                 # 2.2e9 elements: offsets pass 32 bits
    x = torch.zeros((B, V), dtype=BF16, device=dev)
    last = inputs.logits_normal(40, V, 3.0, BF16, seed=2, device=dev)
    x[-40:] = last
    t = tokens_of(B, V, 3, dev)
    o = outputs(B, 4, dev)
    sbw.sbw_token_logprobs(x, t, **o)
    want = oracle.token_logprobs(host_bits(last), V, t[-40:].cpu().numpy(), 1.0, 4)
    compare({k: v[-40:] for k, v in o.items()}, want, 4)
    assert torch.all((o["out_logprob"][:-40] + np.log(V)).abs() < 2e-5) and torch.all(o["out_rank"][:-40] == t[:-40] + 1)
    assert torch.equal(o["out_top_ids"][0].cpu(), torch.arange(4, dtype=torch.int32))
