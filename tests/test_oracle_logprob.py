"""Pins of the oracle's log probabilities, their gradient and weighted detection: scipy's log-softmax and
entropy, brute-force order, torch autograd and central differences in fp64, closed forms, and the plain
detector for weights of one."""
import math

import numpy as np
import pytest
import torch
from scipy.special import entr, log_softmax

KEY = 0x5EED


def _rows(B, V, seed, std=3.0):
    return np.random.default_rng(seed).normal(0.0, std, (B, V)).astype(np.float32)


@pytest.mark.parametrize("V", [1, 2, 5, 64, 1000])
@pytest.mark.parametrize("tau", [0.5, 1.0, 1.75])       # exact in fp32
def test_values_against_scipy(oracle, V, tau):
    x = _rows(6, V, V)
    t = np.random.default_rng(1).integers(0, V, 6)
    n = min(V, 4)
    got = oracle.token_logprobs(x, V, t, tau, top_n=n)
    lp = log_softmax(x.astype(np.float64) / tau, axis=1)
    assert np.allclose(got["logprob"], lp[np.arange(6), t], rtol=0, atol=1e-12)
    assert np.allclose(got["entropy"], entr(np.exp(lp)).sum(1), rtol=0, atol=1e-12)
    assert np.array_equal(got["max"], x.max(1).astype(np.float64))
    assert np.allclose(got["sumexp"], np.exp((x - x.max(1, keepdims=True)).astype(np.float64) / tau).sum(1), rtol=1e-6)
    order = np.argsort(-x, axis=1, kind="stable")
    assert np.array_equal(got["top_ids"], order[:, :n])
    assert np.allclose(got["top_logprobs"], np.take_along_axis(lp, order[:, :n], 1), rtol=0, atol=1e-12)
    assert np.array_equal(got["rank"], 1 + np.argmax(order == t[:, None], axis=1))


def test_ties_zeros_and_nan_in_the_order(oracle):
    x = np.array([[0.0, -0.0, 1.0, 1.0, -0.0]], dtype=np.float32)
    for t, rank in ((2, 1), (3, 2), (0, 3), (1, 4), (4, 5)):
        got = oracle.token_logprobs(x, 5, [t], 1.0, top_n=5)
        assert got["rank"][0] == rank
        assert got["top_ids"][0].tolist() == [2, 3, 0, 1, 4]
    x[0, 2] = np.nan                                     # counts as -inf in the order; the statistics are NaN
    got = oracle.token_logprobs(x, 5, [3], 1.0, top_n=5)
    assert got["top_ids"][0].tolist() == [3, 0, 1, 4, 2] and got["rank"][0] == 1
    assert math.isnan(got["logprob"][0]) and math.isnan(got["entropy"][0]) and math.isnan(got["sumexp"][0])


def test_empty_padded_and_short_rows(oracle):
    x = np.full((3, 4), -np.inf, dtype=np.float32)
    x[1] = 2.5
    x[2] = np.finfo(np.float32).min
    got = oracle.token_logprobs(x, 4, [1, 7, 3], 1.0, top_n=6)
    assert got["logprob"].tolist() == [-math.inf, 0.0, -math.log(4)]
    assert got["entropy"][0] == 0.0 and got["entropy"][1] == 0.0 and abs(got["entropy"][2] - math.log(4)) < 1e-15
    assert got["rank"].tolist() == [2, 0, 4]
    assert got["max"][0] == -math.inf and got["sumexp"].tolist() == [0.0, 0.0, 4.0]
    assert got["top_ids"].tolist() == [[0, 1, 2, 3, -1, -1], [-1] * 6, [0, 1, 2, 3, -1, -1]]
    assert np.all(got["top_logprobs"][0] == -np.inf) and np.all(got["top_logprobs"][1] == -np.inf)


def test_watermarked_values_are_those_of_the_biased_logits(oracle):
    x, ctx = _rows(4, 300, 9), np.array([[3, 4], [5, 6], [7, 8], [1, 2]], dtype=np.int32)
    for scheme in (0, 1):
        biased = oracle.bias_logits(x, 300, ctx, KEY, 0.25, 2.0, scheme, vocab_offset=11)
        a = oracle.token_logprobs(x, 300, [0, 9, 299, 4], 0.75, 3, ctx, KEY, 0.25, 2.0, scheme, vocab_offset=11)
        b = oracle.token_logprobs(biased, 300, [0, 9, 299, 4], 0.75, 3)
        assert all(np.array_equal(a[k], b[k]) for k in a)


@pytest.mark.parametrize("tau", [0.5, 1.0, 1.75])
def test_gradient_against_autograd_and_differences(oracle, tau):
    B, V = 5, 40
    x = _rows(B, V, 3)
    x[1, ::3] = -np.inf                                  # masked columns
    t = np.array([0, 4, 39, -100, 17])                   # one padded row
    rng = np.random.default_rng(4)
    g, h = rng.normal(size=B), rng.normal(size=B)
    s = oracle.token_logprobs(x, V, t, tau)
    got = oracle.token_logprobs_backward(x, V, t, tau, s["max"], s["sumexp"], s["entropy"], g, h)
    assert np.all(got[3] == 0)
    w = torch.tensor(x, dtype=torch.float64, requires_grad=True)
    lp = torch.log_softmax(w / tau, 1)
    keep = torch.tensor(t >= 0)
    plain = torch.where(torch.isinf(lp), torch.zeros_like(lp), lp)
    ent = -(lp.exp() * plain).sum(1)
    loss = (torch.tensor(g) * lp[torch.arange(B), torch.tensor(t).clamp(0)] + torch.tensor(h) * ent)[keep].sum()
    want, = torch.autograd.grad(loss, w)
    assert np.allclose(got, want.numpy(), rtol=0, atol=1e-11)

    def value(row, y):
        lp = log_softmax(y / tau)
        return g[row] * lp[t[row]] + h[row] * entr(np.exp(lp)).sum()

    for row in (0, 2, 4):
        for v in (0, 7, int(t[row])):
            d = np.zeros(V)
            d[v] = 1e-5
            y = x[row].astype(np.float64)
            diff = (value(row, y + d) - value(row, y - d)) / 2e-5
            assert abs(diff - got[row, v]) < 1e-8        # third derivatives times 1e-10, and rounding 1e-16 / 1e-5


def test_gradient_of_empty_rows_is_zero(oracle):
    x = np.full((1, 6), -np.inf, dtype=np.float32)
    s = oracle.token_logprobs(x, 6, [2], 1.0)
    assert np.all(oracle.token_logprobs_backward(x, 6, [2], 1.0, s["max"], s["sumexp"], s["entropy"], [1.0], [1.0]) == 0)


def test_weighted_detection(oracle):
    rng = np.random.default_rng(8)
    lengths = np.array([0, 1, 2, 9, 200, 57], dtype=np.int32)
    tok = rng.integers(0, 1000, lengths.sum()).astype(np.int32)
    for scheme in (0, 1):
        for W in (1, 4):
            ones = oracle.detect_weighted(tok, np.ones(tok.size), lengths, KEY, 0.25, scheme, W)
            counts, T, z = oracle.detect(tok, lengths, KEY, 0.25, scheme, W)
            assert np.array_equal(ones[0], counts) and np.array_equal(ones[1], T) and np.allclose(ones[3], z, atol=1e-12)
            w = rng.exponential(size=tok.size).astype(np.float32)
            G, S1, S2, z = oracle.detect_weighted(tok, w, lengths, KEY, 0.25, scheme, W)
            green = oracle.detect_bits(tok, lengths, KEY, 0.25, scheme, W).astype(bool)
            start = 0
            for s, L in enumerate(lengths):
                part = slice(start + W, start + L) if L > W else slice(start, start)
                y, v = green[part], w[part].astype(np.float64)
                assert math.isclose(G[s], v[y].sum(), abs_tol=1e-12) and math.isclose(S1[s], v.sum(), abs_tol=1e-12)
                assert math.isclose(S2[s], (v * v).sum(), abs_tol=1e-12)
                want = (v[y].sum() - 0.25 * v.sum()) / math.sqrt(0.1875 * (v * v).sum()) if v.size else 0.0
                assert math.isclose(z[s], want, abs_tol=1e-12)
                start += L
    zero = oracle.detect_weighted(tok, np.zeros(tok.size), lengths, KEY, 0.25, 0, 1)
    assert all(np.all(a == 0) for a in zero)
