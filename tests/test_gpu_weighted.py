"""sbw_detect_weighted against the oracle (long-double sums): fp64 sums of n terms are within n 2^-53 of the sum of their
magnitudes, below 1e-10 of it for the lengths here; z within the library's 1e-9."""
import numpy as np
import pytest
import torch

import paper_2609_03844_b200 as sbw
from paper_2609_03844_b200 import inputs
from gpu_util import KEY, require_gpu

pytestmark = pytest.mark.gpu
SCHEMES = [sbw.SCHEME_CONTEXT, sbw.SCHEME_SELFSALT]


def call(tok, w, lens, gamma, scheme, W, offsets=None, scratch=True, stream=None):
    N, dev = lens.numel(), lens.device
    G, S1, S2, z = (torch.full((N,), -5.0, dtype=torch.float64, device=dev) for _ in range(4))
    ws = torch.empty(sbw.sbw_detect_workspace_bytes(N), dtype=torch.uint8, device=dev) if scratch and offsets is None else None
    sbw.sbw_detect_weighted(tok, w, lens, KEY, gamma, scheme, z, out_green=G, out_weight=S1, out_weight2=S2,
                            offsets=offsets, workspace=ws, ctx_width=W, stream=stream)
    return G, S1, S2, z


def check(oracle, tok, w, lens, gamma, scheme, W, offsets=None):
    got = [v.cpu().numpy() for v in call(tok, w, lens, gamma, scheme, W, offsets)]
    want = oracle.detect_weighted(tok.cpu().numpy(), w.cpu().numpy(), lens.cpu().numpy(), KEY, gamma, scheme, W)
    size = oracle.detect_weighted(tok.cpu().numpy(), w.abs().cpu().numpy(), lens.cpu().numpy(), KEY, gamma, scheme, W)
    for k in range(3):
        assert np.all(np.abs(got[k] - want[k]) <= 1e-10 * size[1 if k < 2 else 2])
    assert np.all(np.abs(got[3] - want[3]) <= 1e-9)
    return got


@pytest.mark.parametrize("scheme", SCHEMES)
@pytest.mark.parametrize("W", [1, 2, 4, 8])
def test_lengths_from_nothing_to_long(oracle, scheme, W):
    dev = require_gpu()
    for lens in ([0], [1], [W], [W + 1], [200], [31 + W, 32 + W, 33 + W, 63, 64, 65, 127 + W, 128 + W, 129 + W, 0, 1, -5, 7],
                 [9000], [100003], [5000, 0, 40000], [300] * 40 + [0] * 3 + [5] * 40):
        lens = torch.tensor(lens, dtype=torch.int32, device=dev)
        total = int(lens.clamp(0).sum())
        tok = inputs.uniform_tokens((total,), 128256, 5, dev)
        w = torch.empty(total, device=dev).exponential_(1.0, generator=torch.Generator(device=dev).manual_seed(3))
        check(oracle, tok, w, lens, 0.25, scheme, W)


@pytest.mark.parametrize("scheme", SCHEMES)
@pytest.mark.parametrize("N", [1, 40, 296, 592, 1184, 1185, 3000])
def test_every_number_of_texts(oracle, scheme, N):
    dev = require_gpu()
    tok, lens = inputs.null_token_streams(N, 0, 400, 50000, 7, dev)
    w = torch.randn(tok.numel(), device=dev, generator=torch.Generator(device=dev).manual_seed(N))
    offsets = torch.zeros(N + 1, dtype=torch.int64, device=dev)
    offsets[1:] = lens.long().cumsum(0)
    a = check(oracle, tok, w, lens, 0.5, scheme, 1)
    b = check(oracle, tok, w, lens, 0.5, scheme, 1, offsets)
    assert all(np.array_equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("scheme", SCHEMES)
@pytest.mark.parametrize("N,W", [(5, 1), (100, 4), (2000, 2)])
def test_weights_of_one_give_the_plain_detector(scheme, N, W):
    dev = require_gpu()
    tok, lens = inputs.null_token_streams(N, 0, 700, 1000, 9, dev)
    G, S1, S2, z = call(tok, torch.ones(tok.numel(), device=dev), lens, 0.25, scheme, W)
    c, T = (torch.empty(N, dtype=torch.int32, device=dev) for _ in range(2))
    pz = torch.empty(N, dtype=torch.float64, device=dev)
    ws = torch.empty(sbw.sbw_detect_workspace_bytes(N), dtype=torch.uint8, device=dev)
    sbw.sbw_detect(tok, lens, KEY, 0.25, scheme, c, pz, out_T=T, workspace=ws, ctx_width=W)
    assert torch.equal(G, c.double()) and torch.equal(S1, T.double()) and torch.equal(S2, S1) and torch.equal(z, pz)


def test_weights_that_say_nothing_or_are_not_numbers(oracle):
    dev = require_gpu()
    lens = torch.tensor([50, 50, 50, 50, 50], dtype=torch.int32, device=dev)
    tok = inputs.uniform_tokens((250,), 1000, 3, dev)
    w = torch.ones(250, device=dev)
    w[0:50] = 0.0
    w[50] = float("nan")                                 # seeds only: not read into any sum
    w[100 + 10] = float("nan")
    w[150 + 20] = float("inf")
    w[200:250] = 1e30
    G, S1, S2, z = call(tok, w, lens, 0.25, 0, 1)
    assert z[0] == 0 and S2[0] == 0 and G[0] == 0
    assert not torch.isnan(z[1]) and S1[1] == 49
    assert torch.isnan(z[2]) and torch.isnan(z[3])
    plain = call(tok[200:], torch.ones(50, device=dev), lens[4:], 0.25, 0, 1)[3]
    assert abs(float(z[4] - plain[0])) < 1e-9


def test_texts_that_end_after_the_tokens_and_offsets_of_the_callers(oracle):
    dev = require_gpu()
    tok = inputs.uniform_tokens((1000,), 1000, 3, dev)
    w = torch.rand(1000, device=dev)
    lens = torch.tensor([100, 500, 100, 10], dtype=torch.int32, device=dev)
    offsets = torch.tensor([900, 700, 2000, -3, 0], dtype=torch.int64, device=dev)   # ends there; cut; beyond; before
    G, S1, S2, z = call(tok, w, lens, 0.25, 0, 1, offsets)
    for s, (lo, hi) in enumerate(((900, 1000), (700, 1000), (0, 0), (0, 0))):
        want = oracle.detect_weighted(tok[lo:hi].cpu().numpy(), w[lo:hi].cpu().numpy(), [hi - lo], KEY, 0.25, 0, 1)
        assert abs(float(G[s]) - want[0][0]) < 1e-9 and abs(float(z[s]) - want[3][0]) < 1e-9


def test_refusals_no_texts_streams_and_graphs():
    dev = require_gpu()
    tok, lens = inputs.null_token_streams(300, 0, 300, 1000, 2, dev)
    w = torch.rand(tok.numel(), device=dev)
    with pytest.raises(sbw.SbwError):
        call(tok, w, lens, 0.25, 0, 1, scratch=False)
    with pytest.raises(ValueError):
        call(tok, w[1:], lens, 0.25, 0, 1)
    with pytest.raises(TypeError):
        call(tok, w.double(), lens, 0.25, 0, 1)
    with pytest.raises(TypeError):
        call(tok.cpu(), w, lens, 0.25, 0, 1)
    none = torch.zeros(0, dtype=torch.int32, device=dev)
    call(none, w[:0], none, 0.25, 0, 1)
    offsets = torch.zeros(301, dtype=torch.int64, device=dev)
    offsets[1:] = lens.long().cumsum(0)
    first = call(tok, w, lens, 0.25, 1, 4, offsets)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    second = call(tok, w, lens, 0.25, 1, 4, offsets, stream=s)
    torch.cuda.synchronize()
    out = [torch.zeros_like(v) for v in first]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        sbw.sbw_detect_weighted(tok, w, lens, KEY, 0.25, 1, out[3], out_green=out[0], out_weight=out[1],
                                out_weight2=out[2], offsets=offsets, ctx_width=4)
    g.replay()
    torch.cuda.synchronize()
    for a, b, c in zip(first, second, out):
        assert torch.equal(a, b) and torch.equal(a, c)
