"""Refusals of the log-probability calls and of weighted detection: all on the host, no device needed."""
import ctypes

import pytest
import torch

import paper_2609_03844_b200 as sbw
from paper_2609_03844_b200 import binding

OK, INV, UNS, WSP, BIG = (binding.SBW_OK, binding.SBW_ERR_INVALID_ARG, binding.SBW_ERR_UNSUPPORTED,
                          binding.SBW_ERR_WORKSPACE, binding.SBW_ERR_TOO_LARGE)
fake = ctypes.c_void_p(0x1000)                           # never dereferenced on the host
base = dict(logits=fake, dtype=0, B=2, V=8, ld=8, off=0, ctx=fake, W=1, gamma=0.25, delta=2.0, scheme=0, tau=1.0,
            tokens=fake)
bad_common = [dict(dtype=2), dict(B=-1), dict(V=0), dict(V=-1), dict(ld=7), dict(off=-1), dict(ctx=None), dict(W=0),
              dict(W=9), dict(gamma=0.0), dict(gamma=1.0), dict(gamma=float("nan")), dict(delta=float("nan")),
              dict(delta=float("inf")), dict(scheme=2), dict(scheme=-1), dict(tau=0.0), dict(tau=-1.0),
              dict(tau=float("nan")), dict(tau=float("inf")), dict(tau=1e-30), dict(tau=1e38), dict(logits=None),
              dict(logits=ctypes.c_void_p(0x1001)), dict(logits=ctypes.c_void_p(0x1002))]


def forward(**kw):
    a = {**base, "n": 0, "lp": fake, "ent": None, "rank": None, "m": None, "Z": None, "ids": None, "tops": None, **kw}
    return sbw.lib().sbw_token_logprobs(a["logits"], a["dtype"], a["B"], a["V"], a["ld"], a["off"], a["ctx"], a["W"], 1,
                                        a["gamma"], a["delta"], a["scheme"], a["tau"], a["tokens"], a["n"], a["lp"],
                                        a["ent"], a["rank"], a["m"], a["Z"], a["ids"], a["tops"], None)


def backward(**kw):
    a = {**base, "m": fake, "Z": fake, "H": fake, "g": fake, "h": fake, "out": ctypes.c_void_p(0x200000), "gld": 8, **kw}
    return sbw.lib().sbw_token_logprobs_backward(a["logits"], a["dtype"], a["B"], a["V"], a["ld"], a["off"], a["ctx"],
                                                 a["W"], 1, a["gamma"], a["delta"], a["scheme"], a["tau"], a["tokens"],
                                                 a["m"], a["Z"], a["H"], a["g"], a["h"], a["out"], a["gld"], None)


def weighted(**kw):
    a = dict(tokens=fake, weights=fake, lengths=fake, offsets=None, N=4, total=40, W=1, gamma=0.25, scheme=0, z=fake,
             ws=fake, bytes=1 << 20)
    a.update(kw)
    return sbw.lib().sbw_detect_weighted(a["tokens"], a["weights"], a["lengths"], a["offsets"], a["N"], a["total"],
                                         a["W"], 1, a["gamma"], a["scheme"], None, None, None, a["z"], a["ws"],
                                         a["bytes"], None)


@pytest.mark.parametrize("bad", bad_common)
def test_common_arguments(bad):
    assert forward(**bad) == INV
    assert backward(**bad) == INV


def test_forward_refusals():
    assert forward(B=0) == OK and forward(B=0, logits=None, ctx=None, tokens=None, lp=None) == OK
    for bad in (dict(lp=None), dict(tokens=None), dict(tokens=None, lp=None, rank=fake), dict(n=-1), dict(n=3),
                dict(n=0, ids=fake), dict(n=0, tops=fake)):
        assert forward(**bad) == INV, bad
    assert forward(n=sbw.MAX_TOP_LOGPROBS + 1, ids=fake) == BIG
    assert forward(n=sbw.MAX_TOP_LOGPROBS + 1, ids=fake, gamma=2.0) == INV      # the other fault is reported first
    assert forward(V=1 << 31, ld=1 << 31) == UNS and forward(off=(1 << 32) - 4) == UNS
    assert forward(delta=0.0, ctx=None, lp=None) == INV                          # nothing asked for


def test_backward_refusals():
    assert backward(B=0) == OK and backward(B=0, m=None, out=None, logits=None) == OK
    for bad in (dict(m=None), dict(Z=None), dict(out=None), dict(g=None, h=None), dict(H=None), dict(tokens=None),
                dict(gld=7), dict(out=ctypes.c_void_p(0x200001))):
        assert backward(**bad) == INV, bad
    assert backward(V=1 << 31, ld=1 << 31, gld=1 << 31) == UNS and backward(off=(1 << 32) - 4) == UNS
    assert backward(B=1 << 40, out=ctypes.c_void_p(0x1000)) == UNS               # in place, too many rows for a launch


def test_backward_refuses_a_gradient_that_half_overlaps_the_logits():
    at = lambda k: ctypes.c_void_p(0x1000 + 4 * k)       # noqa: E731
    for k in (1, 4, 8, 9, 15):                           # shifted by k elements, two rows of eight
        assert backward(out=at(k)) == INV, k
    assert backward(out=at(0), gld=16) == INV            # same start, other stride
    # two rows of eight columns with stride 16, the gradient in the gaps: apart; moved by less: not
    for k in (1, 7, 9, 15):
        assert backward(ld=16, gld=16, out=at(k)) == INV, k


def test_weighted_refusals():
    assert weighted(N=0) == OK
    for bad in (dict(gamma=0.0), dict(N=-1), dict(total=-5), dict(W=0), dict(W=9), dict(scheme=2), dict(lengths=None),
                dict(weights=None), dict(tokens=None), dict(z=None)):
        assert weighted(**bad) == INV, bad
    assert weighted(ws=None) == WSP and weighted(bytes=8) == WSP and weighted(ws=ctypes.c_void_p(0x1008)) == WSP
    assert sbw.lib().sbw_last_cuda_error() == 0


def test_binding_refuses_host_tensors():
    x, t = torch.zeros(2, 8), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError):
        sbw.sbw_token_logprobs(x, t, out_logprob=torch.zeros(2))
    with pytest.raises(ValueError):
        sbw.sbw_token_logprobs_backward(x, t, 1.0, torch.zeros(2), torch.zeros(2), torch.zeros(2, 8),
                                        grad_logprob=torch.zeros(2))
    with pytest.raises(ValueError):
        sbw.sbw_detect_weighted(t, torch.zeros(2), torch.ones(1, dtype=torch.int32), 1, 0.25, 0, torch.zeros(1))


def test_the_names_are_exported():
    for name in ("sbw_token_logprobs", "sbw_token_logprobs_backward", "sbw_detect_weighted"):
        assert callable(getattr(sbw, name)) and name in binding.EXPORTS and name in sbw.__all__
    assert sbw.MAX_TOP_LOGPROBS == 64
