"""Sampling from given random numbers on the GPU: tokens and numbers kept equal the definition's, probabilities are its
ratio of whole numbers rounded to fp32 (two divisors rounded to 53 bits, then 2^-24: within 2^-23)."""
import math

import numpy as np
import pytest
import torch

from gpu_util import KEY, require_gpu
from oracle import given
from paper_2609_03844_b200 import inputs

pytestmark = pytest.mark.gpu


def call(logits, u, tau, k=None, p=None, low=None, **mark):
    import paper_2609_03844_b200 as sbw

    B = logits.shape[0]
    dev = lambda v, dt: None if v is None else torch.as_tensor(np.asarray(v), dtype=dt).cuda()  # noqa: E731
    out = (torch.full((B,), -7, dtype=torch.int32, device="cuda"), torch.full((B,), -7.0, device="cuda"),
           torch.full((B,), -7, dtype=torch.int32, device="cuda"))
    sbw.sbw_sample_given(logits, dev(u, torch.float32), out[0], temperature=dev(tau, torch.float32),
                         top_k=dev(k, torch.int32), top_p=dev(p, torch.float32), min_p=dev(low, torch.float32),
                         out_prob=out[1], out_kept=out[2], **mark)
    torch.cuda.synchronize()
    return tuple(o.cpu().numpy() for o in out)


def compare(logits, u, tau, k=None, p=None, low=None, biased=None, **mark):
    got = call(logits, u, tau, k, p, low, **mark)
    x = (logits if biased is None else biased).float().cpu().numpy()
    want = given.sample(x, u, tau, k, p, low)
    assert np.array_equal(got[2], want[2]), (got[2], want[2])
    assert np.array_equal(got[0], want[0]), (got[0], want[0])
    assert np.all(np.abs(got[1] - want[1]) <= 2.0 ** -23 * want[1])
    return got


def settings(B, seed):
    r = np.random.default_rng(seed)
    return (r.random(B, dtype=np.float32), r.choice([0.0, 0.5, 0.7, 1.0, 1.3, 5.0], B).astype(np.float32),
            r.choice([0, 1, 2, 20, 50, 1000, 3000, 100000], B).astype(np.int32),
            r.choice([1.0, 0.95, 0.8, 0.3, 1e-9], B).astype(np.float32),
            r.choice([0.0, 0.0, 0.02, 0.1, 1.0], B).astype(np.float32))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,V,std", [(1, 1, 1.0), (3, 2, 1.0), (5, 7, 3.0), (40, 33, 1.0), (33, 1000, 1.0), (9, 4099, 3.0),
                                     (40, 32003, 3.0), (7, 32000, 1.0), (1, 128256, 4.0), (6, 151936, 1.0), (5, 151937, 4.0),
                                     (2, 262144, 3.0), (2, 327680, 1.0), (150, 5000, 4.0)])
def test_rows_with_settings_of_their_own(B, V, std, dtype):
    require_gpu()
    x = inputs.logits_normal(B, V, std, dtype, seed=V + B).cuda()
    u, tau, k, p, low = settings(B, V)
    compare(x, u, tau, k, p, low)
    one = np.ones(B, np.float32)
    compare(x, u, one)                                  # no filter
    compare(x, u, one, p=p)
    compare(x, u, one, k=k)
    compare(x, u, 0.7 * one, low=low)


@pytest.mark.parametrize("u", [0.0, 1.0 - 2.0 ** -24, 0.999, 0.5, 1.0, 2.0, -1.0, math.nan])
def test_ends_of_the_unit_interval(u):
    require_gpu()
    x = inputs.logits_normal(3, 20011, 2.0, torch.float32, seed=5).cuda()
    us = np.full(3, u, np.float32)
    got = compare(x, us, np.ones(3, np.float32))
    if not u > 0:
        assert np.array_equal(got[0], x.argmax(1).cpu().numpy())
    compare(x, us, np.ones(3, np.float32), k=np.array([5, 1, 20000]), p=np.array([0.9, 0.9, 0.99999]))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_many_equal_values(dtype):
    """Bins too full for a list: constant rows, two values, a few hundred values, narrow and wide ranges."""
    require_gpu()
    V = 100003
    g = torch.Generator().manual_seed(1)
    rows = [torch.zeros(V), torch.full((V,), -3.25), (torch.rand(V, generator=g) < 0.5).float() * 0.001,
            torch.randint(0, 200, (V,), generator=g) / 64.0, torch.randn(V, generator=g) * 1e-4,
            torch.randn(V, generator=g) * 1e-7 - 20.0 * (torch.rand(V, generator=g) < 0.9), -torch.rand(V, generator=g) * 30 - 5]
    rows[-1][17] = 10.0                                 # all others far below, in the tail
    x = torch.stack(rows).to(dtype).cuda()
    for seed in range(4):
        r = np.random.default_rng(seed)
        u = r.random(len(rows), dtype=np.float32)
        one = np.ones(len(rows), np.float32)
        compare(x, u, one)
        compare(x, u, one, p=r.random(len(rows), dtype=np.float32))
        compare(x, u, 0.8 * one, k=r.integers(1, V, len(rows)), p=r.random(len(rows), dtype=np.float32))
    compare(x, np.full(len(rows), 1 - 2.0 ** -24, np.float32), 1.5 * one)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_masked_rows_and_values_that_are_no_numbers(dtype):
    require_gpu()
    V = 3001
    x = inputs.logits_normal(10, V, 3.0, dtype, seed=2)
    x[0] = -math.inf
    x[1, 1:] = -math.inf
    x[2] = torch.finfo(dtype).min
    x[3, ::2] = torch.finfo(dtype).min
    x[4, 5] = math.inf
    x[5, ::7] = math.inf
    x[6, ::3] = math.nan
    x[7] = math.nan
    x[8] = -0.0
    x[8, 5] = 0.0
    x[9] = torch.finfo(dtype).max
    x = x.cuda()
    for seed in range(3):
        u = np.random.default_rng(seed).random(10, dtype=np.float32)
        one = np.ones(10, np.float32)
        got = compare(x, u, one)
        assert got[0][0] == 0 and got[2][0] == 0 and got[2][7] == 0 and got[0][1] == 0 and got[0][4] == 5
        assert not np.isnan(x.float().cpu().numpy()[6, got[0][6]])
        compare(x, u, one, k=np.full(10, 3), p=0.9 * one, low=0.01 * one)
        compare(x, u, 0 * one)
    compare(x, u, np.array([math.nan, math.inf, 1e-7, 1e-6, 1e30, 1e6, -1, math.inf, 1, 1], np.float32))
    compare(x, u, one, k=np.full(10, -5), p=np.array([math.nan, 0, -1, 2, 1, 0.5, 0.5, 0.5, 1e-12, 0.1]),
            low=np.array([math.nan, 2.0, -1, 1e-30, 1, 0.5, 0.5, 0.5, 0.5, 1e-13]))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("scheme", [0, 1])
@pytest.mark.parametrize("B,V,W", [(3, 1003, 1), (2, 32000, 4), (20, 5001, 8)])
def test_watermarked_rows(oracle, B, V, W, scheme, dtype):
    require_gpu()
    import paper_2609_03844_b200 as sbw

    off = 4096
    x = inputs.logits_normal(B, V, 3.0, dtype, seed=9)
    ctx = inputs.uniform_tokens((B, W), V, seed=10).cuda()
    mark = dict(ctx_tokens=ctx, key=KEY, gamma=0.25, delta=2.0, scheme=scheme, vocab_offset=off)
    biased = x.cuda().clone()
    sbw.sbw_bias_logits(biased, ctx, KEY, 0.25, 2.0, scheme, vocab_offset=off)
    u, tau, k, p, low = settings(B, 3)
    got = compare(x.cuda(), u, tau, k, p, low, biased=biased, **mark)
    for a, b in zip(got, call(biased, u, tau, k, p, low)):
        assert np.array_equal(a, b)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_of_any_alignment(dtype):
    require_gpu()
    for V in (5, 1000, 8195):
        for ld in (V, V + 1, V + 3, V + 8):
            for start in range(0, 9, 2):
                buf = torch.full((start + 6 * ld,), math.inf, dtype=dtype, device="cuda")     # what lies between must not count
                x = buf[start:start + 6 * ld].view(6, ld)[:, :V]
                x.copy_(inputs.logits_normal(6, V, 2.0, dtype, seed=start))
                u, tau, k, p, low = settings(6, V + start)
                compare(x, u, tau, k, p, low)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_values_of_every_size(dtype):
    """Values from 256 on and from -256 down, magnitudes around 2^-24 and below, zeros of both signs, powers of two."""
    require_gpu()
    V = 9000
    g = torch.Generator().manual_seed(3)
    n = torch.randn(V, generator=g)
    rows = [n * 300, n * 0.01 - 300, n * 2.0 ** -24, n * 2.0 ** -30, n * 1e-38, torch.where(n < 0, n, -0.0 * n), n.clone(), n.clone(),
            n.clone(), n * 100, torch.exp2((n * 8).round()) * torch.sign(n), n * 0 + 255.0, n * 0 - 255.0]
    rows[6][100], rows[7][5], rows[8][2000:] = 256.0, 2.0 ** -24, -1000.0
    x = torch.stack(rows).to(dtype).cuda()
    B = len(rows)
    for seed in range(3):
        r = np.random.default_rng(seed)
        u = r.random(B, dtype=np.float32)
        for tau in (1.0, 30.0, 1000.0, 0.01):
            t = np.full(B, tau, np.float32)
            compare(x, u, t)
            compare(x, u, t, k=r.integers(1, V, B), p=r.random(B, dtype=np.float32), low=np.full(B, 1e-4))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_any_number_of_rows(dtype):
    """The numbers of CTAs per row: few rows, as many as SMs, more."""
    require_gpu()
    for B in (1, 2, 17, 36, 37, 74, 75, 148, 149, 400):
        x = inputs.logits_normal(B, 9001, 2.0, dtype, seed=B).cuda()
        u, tau, k, p, low = settings(B, B)
        compare(x, u, tau, k, p, low)
        compare(x, u, np.ones(B, np.float32))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_values_around_zero(dtype):
    """Draws and cuts among zeros of both signs and magnitudes too small for a counter of their own."""
    require_gpu()
    V = 6000
    g = torch.Generator().manual_seed(8)
    sign = torch.randint(0, 2, (V,), generator=g) * 2.0 - 1.0
    low = torch.where(torch.rand(V, generator=g) < 0.3, -5.0 - torch.rand(V, generator=g), 0.0)
    tiny = torch.exp2(-50.0 - torch.randint(0, 60, (V,), generator=g).float())
    rows = [low + 0.0 * sign, torch.where(low == 0, 0.0 * sign, low), torch.where(low == 0, tiny * sign, low),
            torch.where(torch.rand(V, generator=g) < 0.01, tiny * sign, torch.where(low == 0, 0.0 * sign, low))]
    rows += [r.clone() for r in rows]
    for i, r in enumerate(rows):
        r[7] = 0.5 if i < 4 else 2.0 ** -21             # the maximum
    x = torch.stack(rows).to(dtype).repeat(1, 3).cuda()
    for seed in range(5):
        r = np.random.default_rng(seed)
        u = r.random(len(rows), dtype=np.float32)
        one = np.ones(len(rows), np.float32)
        compare(x, u, one)
        compare(x, u, one, k=r.integers(1, V, len(rows)), p=r.random(len(rows), dtype=np.float32))
    wide = x[:4].repeat(60, 1)                          # a CTA per row
    u = np.random.default_rng(9).random(240, dtype=np.float32)
    compare(wide, u, np.ones(240, np.float32))


def test_bins_keep_the_order():
    """The sampler's bins are the weights' fp32 bits from the 17th up.  The polynomial of the weights, fused as they are, over every
    fp32 argument from 0 down to -40: a smaller argument never lies in a higher bin."""
    require_gpu()

    def fma(a, b, c):
        """a b + c of fp32 values, rounded once: the sum in fp64 rounded to odd, then to fp32."""
        p, c = a.double() * b.double(), torch.full_like(b, c, dtype=torch.float64)
        s = p + c
        part = s - p
        rest = (p - (s - part)) + (c - part)
        bits = s.view(torch.int64)
        toward = torch.where((rest > 0) == (s > 0), 1, -1)
        even = (bits & 1) == 0
        return torch.where((rest != 0) & even, bits + toward, bits).view(torch.float64).float()

    step, last = 1 << 25, None
    end = int(np.float32(40).view(np.int32)) + 1
    for at in range(0, end, step):
        y = -torch.arange(at, min(at + step, end), dtype=torch.int32, device="cuda").view(torch.float32)
        n = y.round()
        f = y - n
        p = torch.full_like(f, float(given._EXP2[0]))
        for a in given._EXP2[1:]:
            p = fma(p, f, float(a))
        bins = ((p.view(torch.int32).long() + (n.long() << 23)) >> 17)
        assert bool((bins[1:] <= bins[:-1]).all()) and (last is None or int(bins[0]) <= last)
        last = int(bins[-1])
