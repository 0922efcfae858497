"""sbw_token_logprobs_backward against the fp64 oracle on the same saved statistics.

Tolerance per element, u = 2^-24, d = (l - m)/tau, p = e^d / Z: the exponential is off by 4 u + 3 u |d| relative (its own
2^-22, and the roundings of difference, 1/tau and product in its argument); base, slope, their fused sum and
the product add 4 u of the largest magnitude that enters, |g| + |h| (|H - ln Z| + |d|); the token's own share g/tau and
the sum with it 2 u |g|/tau.  The result is rounded once to the logits' type: eps/2 of it.  e^d below 2^-126 is 0."""
import numpy as np
import pytest
import torch

import paper_2609_03844_b200 as sbw
from paper_2609_03844_b200 import inputs
from gpu_util import KEY, host_bits, require_gpu

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24


def saved(oracle, x, V, t, tau, mark):
    """m, Z, H of the forward pass as the fp32 values a caller keeps."""
    s = oracle.token_logprobs(host_bits(x), V, t.cpu().numpy(), tau, **mark)
    return [torch.tensor(s[k], dtype=F32, device=x.device) for k in ("max", "sumexp", "entropy")]


def check(oracle, x, t, tau, V=None, out=None, use=("g", "h"), ctx=None, **mark):
    B, V, dev = x.shape[0], V or x.shape[1], x.device
    host = dict(mark, ctx_tokens=None if ctx is None else ctx.cpu().numpy())
    m, Z, H = saved(oracle, x, V, t, tau, host)
    gen = torch.Generator(device=dev)
    gen.manual_seed(V)
    g = torch.randn(B, generator=gen, device=dev) if "g" in use else None
    h = torch.randn(B, generator=gen, device=dev) if "h" in use else None
    bits = host_bits(x)
    grad = torch.full_like(x, 9.0) if out is None else out
    edge = None if grad.data_ptr() == x.data_ptr() else grad.clone()
    sbw.sbw_token_logprobs_backward(x, t if g is not None or h is None else None, tau, m, Z, grad, grad_logprob=g,
                                    entropy=H if h is not None else None, grad_entropy=h, V=V, ctx_tokens=ctx, **mark)
    torch.cuda.synchronize()
    n = lambda a: None if a is None else a.cpu().numpy().astype(np.float64)   # noqa: E731
    tok = t.cpu().numpy() if g is not None else None
    want = oracle.token_logprobs_backward(bits, V, tok, tau, n(m), n(Z), n(H), n(g), n(h), **host)
    got = grad[:, :V].cpu().double().numpy()
    if edge is not None:                                 # columns beyond V stay as they were
        assert torch.equal(grad[:, V:], edge[:, V:])
    biased = bits if ctx is None else oracle.bias_logits(bits, V, host["ctx_tokens"], **mark)
    l = torch.tensor(biased.view(np.int16)).view(BF16).double().numpy() if biased.dtype == np.uint16 else biased.astype(np.float64)
    with np.errstate(all="ignore"):
        d = (l[:, :V] - n(m)[:, None]) / tau
        p = np.nan_to_num(np.exp(d) / n(Z)[:, None])
        size = np.zeros((B, V))
        if g is not None:
            size += np.abs(n(g))[:, None]
        if h is not None:
            size += np.abs(n(h))[:, None] * (np.abs(n(H) - np.log(n(Z)))[:, None] + np.maximum(np.abs(d), 0))
        tol = np.where(p > 0, p / tau * size * (8 * U + 3 * U * np.abs(np.where(p > 0, d, 0))), 0.0)
    if g is not None:
        rows = np.flatnonzero((tok >= 0) & (tok < V))
        tol[rows, tok[rows]] += 2 * U * np.abs(n(g))[rows] / tau
    tol = np.nan_to_num(tol) + 1e-36
    tol += (torch.finfo(x.dtype).eps / 2) * (np.abs(np.nan_to_num(want)) + tol) + (1e-38 if x.dtype == F32 else 1e-37)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    off = np.abs(np.nan_to_num(got) - np.nan_to_num(want)) - tol
    assert off.max() <= 0, (np.unravel_index(off.argmax(), off.shape), off.max())
    return grad


def tokens_of(B, V, seed, dev):
    return inputs.uniform_tokens((B,), V, seed, dev)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", [1, 2, 3, 7, 8, 9, 17, 33, 127, 1000, 4099, 32003])
def test_sizes_and_alignments(oracle, V, dtype):
    dev = require_gpu()
    for B, ld in ((1, V), (3, V + 1), (9, V + 5), (4, V + 8)):
        x = inputs.logits_normal(B, ld, 3.0, dtype, seed=V + B, device=dev)
        check(oracle, x, tokens_of(B, V, 3, dev), 0.75, V=V)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_gradient_of_another_alignment_than_the_logits(oracle, dtype):
    dev = require_gpu()
    for first in range(0, 9):
        x = inputs.logits_normal(4, 900, 3.0, dtype, seed=first, device=dev)[:, 4:804]
        out = torch.full((4, 830), 9.0, dtype=dtype, device=dev)[:, first:first + 800]
        check(oracle, x, tokens_of(4, 800, first, dev), 1.0, out=out)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_in_place(oracle, dtype):
    dev = require_gpu()
    for V, ld in ((5003, 5003), (4096, 4100), (32003, 32003)):
        x = inputs.logits_normal(7, ld, 3.0, dtype, seed=V, device=dev)
        t = tokens_of(7, V, 1, dev)
        apart = check(oracle, x, t, 1.0, V=V)
        keep = x[:, V:].clone()
        assert check(oracle, x, t, 1.0, V=V, out=x) is x
        assert torch.equal(x[:, :V], apart[:, :V]) and torch.equal(x[:, V:], keep)


@pytest.mark.parametrize("use", [("g",), ("h",), ("g", "h")])
def test_one_gradient_or_both(oracle, use):
    dev = require_gpu()
    x = inputs.logits_normal(20, 3001, 3.0, F32, seed=2, device=dev)
    check(oracle, x, tokens_of(20, 3001, 3, dev), 0.7, use=use)


@pytest.mark.parametrize("scheme", [sbw.SCHEME_CONTEXT, sbw.SCHEME_SELFSALT])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,V,W,off", [(3, 37, 2, 5), (2, 5003, 4, 100000), (33, 4100, 8, (1 << 32) - 4100)])
def test_watermarked(oracle, B, V, W, off, dtype, scheme):
    dev = require_gpu()
    x = inputs.logits_normal(B, V, 3.0, dtype, seed=V, device=dev)
    ctx = inputs.uniform_tokens((B, W), 1 << 30, V + 1, dev)
    check(oracle, x, tokens_of(B, V, 3, dev), 0.7, ctx=ctx, key=KEY, gamma=0.25, delta=2.0, scheme=scheme, vocab_offset=off)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_masks_padding_and_special_values(oracle, dtype):
    dev = require_gpu()
    B, V, low = 6, 3001, torch.finfo(dtype).min
    t = tokens_of(B, V, 3, dev)
    t[1], t[4] = -100, V
    rnd = lambda s: inputs.logits_normal(B, V, 3.0, dtype, seed=s, device=dev)   # noqa: E731
    hide = torch.rand(B, V, device=dev, generator=torch.Generator(device=dev).manual_seed(1)) < 0.6
    nan, inf, one = rnd(1), rnd(2), torch.full((B, V), -np.inf, dtype=dtype, device=dev)
    nan[:, 9] = float("nan")
    inf[:, 2000] = float("inf")
    one[:, 77] = 2.0
    for x in (rnd(3).masked_fill(hide, -np.inf), rnd(4).masked_fill(hide, low), torch.full_like(nan, -np.inf),
              torch.full_like(nan, low), torch.full_like(nan, -low), torch.zeros_like(nan), nan, inf, one,
              (rnd(5).float() * 1e37).to(dtype), torch.where(rnd(6) > 0, low, -low).to(dtype)):
        check(oracle, x, t, 1.0)


def test_gradient_against_differences():
    """The loss g logprob + h entropy of the forward call itself, fp32: central differences with step s carry the forward
    call's own error 2 (8e-6 + ...) / (2 s) and s^2 / 6 of a third derivative below |g| + 12 |h|."""
    dev = require_gpu()
    V, B = 50, 50
    row = inputs.logits_normal(1, V, 1.0, F32, seed=3, device=dev)
    g, h, t, s = 0.8, 0.6, 11, 0.0625
    o = lambda n: [torch.empty(n, dtype=F32, device=dev) for _ in range(4)]   # noqa: E731

    def value(x):
        lp, ent, m, z = o(x.shape[0])
        tok = torch.full((x.shape[0],), t, dtype=torch.int32, device=dev)
        sbw.sbw_token_logprobs(x, tok, 1.0, out_logprob=lp, out_entropy=ent, out_max=m, out_sumexp=z)
        return lp.double() * g + ent.double() * h, m, z, ent

    step = s * torch.eye(B, V, device=dev)
    diff = (value(row + step)[0] - value(row - step)[0]) / (2 * s)
    _, m, z, ent = value(row)
    grad = torch.empty_like(row)
    sbw.sbw_token_logprobs_backward(row, torch.tensor([t], dtype=torch.int32, device=dev), 1.0, m, z, grad,
                                    grad_logprob=torch.tensor([g], device=dev), entropy=ent,
                                    grad_entropy=torch.tensor([h], device=dev))
    bound = (g * (8e-6 + 2.0 ** -21 * 12) + h * 16e-6 * 5) / s + s * s / 6 * (g + 12 * h)
    assert (diff - grad[0].double()).abs().max() < bound


def test_refusals():
    dev = require_gpu()
    x = torch.zeros((3, 64), device=dev)
    t = torch.zeros(3, dtype=torch.int32, device=dev)
    f = torch.ones(3, device=dev)
    go = lambda **kw: sbw.sbw_token_logprobs_backward(**{**dict(logits=x, tokens=t, temperature=1.0, max=f, sumexp=f,  # noqa: E731
                                                                grad_logits=torch.empty_like(x), grad_logprob=f), **kw})
    go()
    for bad in (dict(grad_logits=torch.empty((2, 64), device=dev)), dict(grad_logits=torch.empty_like(x).bfloat16()),
                dict(V=65), dict(delta=2.0)):
        with pytest.raises(ValueError):
            go(**bad)
    for bad in (dict(max=None), dict(sumexp=None), dict(grad_logprob=f.double()), dict(tokens=t.long()),
                dict(grad_logprob=torch.ones(1, device=dev).expand(3))):
        with pytest.raises(TypeError):
            go(**bad)
    buf = torch.zeros(1024, device=dev)
    for bad in (dict(grad_logprob=None), dict(tokens=None), dict(grad_entropy=f), dict(temperature=0.0),
                dict(logits=buf[:192].view(3, 64), grad_logits=buf[4:196].view(3, 64))):
        with pytest.raises(sbw.SbwError):
            go(**bad)
    wide = torch.randn(3, 128, device=dev)               # rows side by side in one buffer are apart
    go(logits=wide[:, :64], grad_logits=wide[:, 64:])
    empty = torch.zeros((0, 64), device=dev)
    z = torch.zeros(0, device=dev)
    go(logits=empty, tokens=t[:0], max=z, sumexp=z, grad_logits=empty.clone(), grad_logprob=z)


def test_graph_streams_and_equal_bits():
    dev = require_gpu()
    B, V = 30, 32003
    x = inputs.logits_normal(B, V, 3.0, BF16, seed=6, device=dev)
    t = tokens_of(B, V, 7, dev)
    lp, ent, m, z = (torch.empty(B, dtype=F32, device=dev) for _ in range(4))
    g = torch.randn(B, device=dev)
    outs = [torch.zeros_like(x) for _ in range(3)]

    def step(out, **kw):
        sbw.sbw_token_logprobs(x, t, 0.7, out_logprob=lp, out_entropy=ent, out_max=m, out_sumexp=z, **kw)
        sbw.sbw_token_logprobs_backward(x, t, 0.7, m, z, out, grad_logprob=g, entropy=ent, grad_entropy=g, **kw)

    step(outs[0])
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    step(outs[1], stream=s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(outs[2])
    outs[2].zero_()
    x2 = x.clone()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2]) and torch.equal(x, x2)
