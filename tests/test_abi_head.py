"""Refusals of the 8-bit projection, its quantiser and the sampler from given random numbers: all on the host, no device
needed.  And the oracle of that sampler against the C oracle's weights and filtered sampler's rules."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2609_03844_b200 as sbw
from oracle import given
from paper_2609_03844_b200 import binding

OK, INV, UNS, BIG = binding.SBW_OK, binding.SBW_ERR_INVALID_ARG, binding.SBW_ERR_UNSUPPORTED, binding.SBW_ERR_TOO_LARGE
at = ctypes.c_void_p
fake = at(0x1000)                                        # never dereferenced on the host
NAN, INF = float("nan"), float("inf")


def quantize(**kw):
    a = dict(x=fake, dtype=0, R=2, K=200, ld=200, rows=1, out=fake, ldo=200, s=fake, lds=2)
    a.update(kw)
    return sbw.lib().sbw_quantize_fp8(a["x"], a["dtype"], a["R"], a["K"], a["ld"], a["rows"], a["out"], a["ldo"], a["s"], a["lds"], None)


def head(**kw):
    a = dict(x=fake, ldx=208, xs=fake, ldxs=2, w=fake, ldw=208, ws=fake, ldws=2, B=2, V=8, K=200, out=fake, dtype=0, ld=8,
             off=0, ctx=fake, W=1, gamma=0.25, delta=2.0, scheme=0)
    a.update(kw)
    return sbw.lib().sbw_head_logits(a["x"], a["ldx"], a["xs"], a["ldxs"], a["w"], a["ldw"], a["ws"], a["ldws"], a["B"], a["V"],
                                     a["K"], a["out"], a["dtype"], a["ld"], a["off"], a["ctx"], a["W"], 1, a["gamma"],
                                     a["delta"], a["scheme"], None)


def sample(**kw):
    a = dict(x=fake, dtype=0, B=2, V=8, ld=8, off=0, ctx=fake, W=1, gamma=0.25, delta=2.0, scheme=0, u=fake, t=fake, k=None,
             p=None, low=None, out=fake, prob=None, kept=None)
    a.update(kw)
    return sbw.lib().sbw_sample_given(a["x"], a["dtype"], a["B"], a["V"], a["ld"], a["off"], a["ctx"], a["W"], 1, a["gamma"],
                                      a["delta"], a["scheme"], a["u"], a["t"], a["k"], a["p"], a["low"], a["out"], a["prob"],
                                      a["kept"], None)


MARK = [dict(W=0), dict(W=9), dict(gamma=0.0), dict(gamma=1.0), dict(gamma=NAN), dict(delta=NAN), dict(delta=INF),
        dict(scheme=2), dict(scheme=-1), dict(ctx=None), dict(dtype=2), dict(dtype=-1), dict(off=-1)]


def test_quantizer_refusals():
    assert quantize(R=0) == OK and quantize(R=0, x=None, out=None, s=None) == OK
    for bad in (dict(dtype=2), dict(R=-1), dict(K=0), dict(ld=199), dict(ldo=199), dict(lds=1), dict(rows=0), dict(rows=64),
                dict(x=None), dict(out=None), dict(s=None), dict(x=at(0x1002)), dict(dtype=1, x=at(0x1001)), dict(s=at(0x1002))):
        assert quantize(**bad) == INV, bad
    big = 1 << 31
    assert quantize(K=big, ld=big, ldo=big, lds=1 << 25) == UNS and quantize(rows=128, R=1 << 39) == UNS


def test_head_refusals():
    assert head(B=0) == OK and head(B=0, x=None, w=None, out=None, ctx=None) == OK
    for bad in MARK + [dict(B=-1), dict(V=0), dict(K=0), dict(ld=7), dict(ldx=199), dict(ldw=192), dict(ldx=201), dict(ldw=209),
                       dict(ldxs=1), dict(ldws=1), dict(x=None), dict(xs=None), dict(w=None), dict(ws=None), dict(out=None),
                       dict(x=at(0x1008)), dict(w=at(0x1001)), dict(xs=at(0x1002)), dict(ws=at(0x1001)), dict(out=at(0x1002)),
                       dict(dtype=1, out=at(0x1001))]:
        assert head(**bad) == INV, bad
    big = 1 << 31
    assert head(off=(1 << 32) - 4) == UNS and head(V=big, ld=big) == UNS and head(B=big) == UNS
    assert head(K=big, ldx=big, ldw=big, ldxs=1 << 25, ldws=1 << 25) == UNS


def test_sampler_refusals():
    assert sample(B=0) == OK and sample(B=0, x=None, ctx=None, u=None, t=None, out=None) == OK
    for bad in MARK + [dict(B=-1), dict(V=0), dict(ld=7), dict(x=None), dict(u=None), dict(t=None), dict(out=None),
                       dict(x=at(0x1002)), dict(dtype=1, x=at(0x1001))]:
        assert sample(**bad) == INV, bad
    assert sample(off=(1 << 32) - 4) == UNS
    assert sample(V=327681, ld=327681) == BIG and sample(V=327681, ld=327681, B=0) == BIG
    assert sbw.lib().sbw_last_cuda_error() == 0


def test_binding_refuses_what_is_not_there():
    e4m3 = torch.float8_e4m3fn
    x, t = torch.zeros(2, 128), torch.zeros(2)
    with pytest.raises(ValueError):
        sbw.sbw_quantize_fp8(x, torch.zeros(2, 128, dtype=e4m3), torch.zeros(2, 1))
    with pytest.raises(ValueError):
        sbw.sbw_head_logits(x.to(e4m3), torch.zeros(2, 1), x.to(e4m3), torch.zeros(1, 1), torch.zeros(2, 2))
    with pytest.raises(ValueError):
        sbw.sbw_sample_given(x, t, torch.zeros(2, dtype=torch.int32), temperature=t)
    for name in ("sbw_quantize_fp8", "sbw_head_logits", "sbw_sample_given"):
        assert callable(getattr(sbw, name)) and name in binding.EXPORTS and name in sbw.__all__


def test_the_samplers_weights_are_the_filtered_samplers(oracle):
    L, r = oracle.lib(), np.random.default_rng(0)
    for m, tau in ((3.0, 1.0), (17.2, 0.7), (0.0, 5.0), (-4.5, 0.05)):
        m, c = np.float32(m), np.float32(1.4426950408889634 / tau)
        x = (m - np.abs(r.normal(0, 8 * tau, 3000))).astype(np.float32)
        x[0] = m
        want = [L.sbw_oracle_nucleus_weight(float(v), float(m), int(v == m), float(c)) for v in x]
        assert np.array_equal(given.weights(x, m, c), np.array(want, np.int64))


def test_the_samplers_oracle_draws_the_softmax():
    """Equally spaced random numbers give each candidate its share of them, to one number; closed forms of the filters."""
    r = np.random.default_rng(1)
    x = (2 * r.standard_normal(12)).astype(np.float32)
    n = 4096
    drawn = [given.sample_row(x, (i + 0.5) / n, 0.7)[0] for i in range(n)]
    p = np.exp((x.astype(np.float64) - x.max()) / 0.7)
    assert np.all(np.abs(np.bincount(drawn, minlength=12) / n - p / p.sum()) <= 1.5 / n)
    assert given.sample_row(x, 0.99, 0.0)[0] == x.argmax() and given.sample_row(x, 0.0, 1.0)[0] == x.argmax()
    flat = np.zeros(10, np.float32)
    assert [given.sample_row(flat, 0.999, 1.0, top_p=p)[3] for p in (0.05, 0.31, 0.999)] == [1, 4, 10]
    assert given.sample_row(flat, 0.999, 1.0, top_k=3)[0] == 2 and given.sample_row(flat, 0.999, 1.0, min_p=1.0)[3] == 10
    two = np.array([0.0, -1.0, -5.0], np.float32)
    assert given.sample_row(two, 0.999, 1.0, min_p=0.3)[3] == 2 and given.sample_row(two, 0.999, 1.0, min_p=0.4)[3] == 1


@pytest.mark.parametrize("K,top_p,tau", [(0, 0.8, 0.7), (20, 1.5, 1.0), (50, 0.9, 1.3), (0, 0.3, 0.5)])
def test_the_samplers_filters_keep_what_the_filtered_sampler_keeps(oracle, K, top_p, tau):
    V, B = 700, 6
    x = (3 * np.random.default_rng(2).standard_normal((B, V))).astype(np.float32)
    ref = oracle.bias_sample_filtered(x, V, np.zeros((B, 1), np.int32), 1, 0.25, 0.0, 0, tau, K, top_p, 3, 4)
    kept = ref["kept"] if isinstance(ref, dict) else ref[1]
    p = np.full(B, np.float64(np.float32(top_p)) if top_p < 1 else 1.0)
    assert np.array_equal(given.sample(x, np.full(B, 0.5), np.full(B, tau), np.full(B, K), p)[2], kept)


def test_a_place_for_the_number_of_waits_is_needed():
    assert sbw.lib().sbw_head_gave_up(None, None) == INV
    assert callable(sbw.sbw_head_gave_up) and "sbw_head_gave_up" in binding.EXPORTS and "sbw_head_gave_up" in sbw.__all__
