"""What the log-probability calls and weighted detection owe beside their numbers: no device allocation, a first call
inside a stream capture, gradients of rows whose offsets pass 32 bits, and clean runs of the bounds-flag build."""
import ctypes
import subprocess
import sys
from pathlib import Path

import numpy as np
import pytest
import torch

import paper_2609_03844_b200 as sbw
from paper_2609_03844_b200 import binding, build as sbw_build, inputs
from gpu_util import KEY, host_bits, require_gpu

pytestmark = pytest.mark.gpu
ROOT = Path(__file__).resolve().parent.parent


def _calls(dev, B=70, V=5003):
    """One call of each entry point on tensors made here, as functions of a stream."""
    x = inputs.logits_normal(B, V, 3.0, torch.bfloat16, seed=1, device=dev)
    t = inputs.uniform_tokens((B,), V, 2, dev)
    ctx = inputs.uniform_tokens((B, 4), V, 3, dev)
    lp, ent, m, z, g = (torch.ones(B, device=dev) for _ in range(5))
    ids = torch.zeros((B, 7), dtype=torch.int32, device=dev)
    tops = torch.zeros((B, 7), device=dev)
    grad = torch.zeros_like(x)
    tok, lens = inputs.null_token_streams(50, 0, 300, V, 4, dev)
    w = torch.rand(tok.numel(), device=dev)
    wz = torch.zeros(50, dtype=torch.float64, device=dev)
    ws = torch.zeros(sbw.sbw_detect_workspace_bytes(50), dtype=torch.uint8, device=dev)

    def every():
        for mark in ({}, dict(ctx_tokens=ctx, key=KEY, gamma=0.25, delta=2.0, scheme=1)):
            sbw.sbw_token_logprobs(x, t, 0.7, out_logprob=lp, out_entropy=ent, out_max=m, out_sumexp=z, out_top_ids=ids,
                                   out_top_logprobs=tops, **mark)
            sbw.sbw_token_logprobs(x, t, 0.7, out_logprob=lp, **mark)
            sbw.sbw_token_logprobs_backward(x, t, 0.7, m, z, grad, grad_logprob=g, entropy=ent, grad_entropy=g, **mark)
        sbw.sbw_detect_weighted(tok, w, lens, KEY, 0.25, 1, wz, workspace=ws, ctx_width=4)
        return lp, ent, ids, tops, grad, wz

    return every


def test_no_device_memory_is_allocated():
    dev = require_gpu()
    every = _calls(dev)
    every()                                              # the kernels are loaded
    torch.cuda.synchronize()
    free, held = torch.cuda.mem_get_info()[0], torch.cuda.memory_allocated()
    for _ in range(50):
        every()
    torch.cuda.synchronize()
    assert torch.cuda.mem_get_info()[0] == free and torch.cuda.memory_allocated() == held


FIRST = """
import sys; sys.path[:0] = [{root!r}, {tests!r}]
import torch
from test_gpu_logprob_owed import _calls
every = _calls(torch.device("cuda:0"))
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    out = every()
for v in out: v.zero_()
g.replay()
torch.cuda.synchronize()
a = [v.clone() for v in out]
for v in out: v.zero_()
every()
torch.cuda.synchronize()
assert all(torch.equal(u, v) for u, v in zip(a, out)) and any(float(v.float().abs().sum()) for v in out)
print("captured first")
"""


def test_the_first_call_of_a_process_can_be_captured():
    require_gpu()
    code = FIRST.format(root=str(ROOT), tests=str(ROOT / "tests"))
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "captured first" in r.stdout, r.stderr[-2000:]


def test_gradient_far_into_a_large_batch(oracle):
    dev = require_gpu()
    V, B = 131072, 17000                                 # 2.2e9 elements: offsets pass 32 bits
    x = torch.zeros((B, V), dtype=torch.bfloat16, device=dev)
    x[-3:] = inputs.logits_normal(3, V, 3.0, torch.bfloat16, seed=2, device=dev)
    t = inputs.uniform_tokens((B,), V, 3, dev)
    s = oracle.token_logprobs(host_bits(x[-3:]), V, t[-3:].cpu().numpy(), 1.0)
    m, z = torch.zeros(B, device=dev), torch.full((B,), float(V), device=dev)
    m[-3:], z[-3:] = torch.tensor(s["max"], device=dev), torch.tensor(s["sumexp"], device=dev)
    g = torch.ones(B, device=dev)
    last = x[-3:].clone()
    assert sbw.sbw_token_logprobs_backward(x, t, 1.0, m, z, x, grad_logprob=g) is x          # in place
    want = oracle.token_logprobs_backward(host_bits(last), V, t[-3:].cpu().numpy(), 1.0, m[-3:].double().cpu().numpy(),
                                          z[-3:].double().cpu().numpy(), None, np.ones(3))
    got = x[-3:].double().cpu().numpy()
    # half a bf16 step, and p's fp32 error (4 + 8 + 3 |d|) 2^-24 p, |d| < 60
    assert np.all(np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 200 * 2.0 ** -24 * np.abs(want) + 2.0 ** -23 * (np.abs(want) > 0.01))
    row = x[5].float()
    hit = int(t[5])
    assert float(row[hit]) == 1.0 and torch.all((row[row != row[hit]] + 1.0 / V).abs() <= 2.0 ** -8 / V)


@pytest.fixture(scope="module")
def dbg():
    require_gpu()
    binding.lib()
    L = ctypes.CDLL(str(sbw_build.build(debug=True)))    # compiled here if missing or older than the sources
    for name in ("sbw_token_logprobs", "sbw_token_logprobs_backward", "sbw_detect_weighted"):
        getattr(L, name).restype = ctypes.c_int
        getattr(L, name).argtypes = getattr(binding.lib(), name).argtypes
    L.sbw_debug_flags.argtypes = [ctypes.c_void_p, ctypes.c_int]
    return L


def _flags(L):
    out = (ctypes.c_uint * 4)()
    assert L.sbw_debug_flags(out, 1) == 0
    return list(out)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,V,ld,first", [(1, 1, 1, 0), (2, 3, 4, 1), (3, 7, 9, 0), (5, 8, 8, 3), (4, 33, 37, 5), (2, 40001, 40001, 0),
                                          (40, 9001, 9003, 1), (400, 2500, 2500, 0), (600, 1025, 1030, 7)])
@pytest.mark.parametrize("delta", [0.0, 2.0])
def test_bounds_flag_build_sees_no_access_outside(dbg, B, V, ld, first, dtype, delta):
    dev = require_gpu()
    es = 4 if dtype == torch.float32 else 2
    buf = inputs.logits_normal(1, B * ld + 16, 3.0, dtype, seed=B + V, device=dev)[0]
    t = inputs.uniform_tokens((B,), V, 5, dev)
    t[::4] = -1
    ctx = inputs.uniform_tokens((B, 2), V, 6, dev)
    n = min(V, 9)
    f = lambda *s: torch.zeros(*s, device=dev)           # noqa: E731
    i = lambda *s: torch.zeros(*s, dtype=torch.int32, device=dev)   # noqa: E731
    p = lambda v: v.data_ptr()                           # noqa: E731
    code = 0 if dtype == torch.float32 else 1
    results = []
    for L in (dbg, binding.lib()):
        lp, ent, rank, m, z, ids, tops = f(B), f(B), i(B), f(B), f(B), i(B, n), f(B, n)
        grad = torch.zeros(B * V + 8, dtype=dtype, device=dev)
        _flags(dbg)
        for scheme in (0, 1):
            head = (p(buf) + first * es, code, B, V, ld, 0, p(ctx), 2, KEY, 0.25, delta, scheme, 1.0, p(t))
            assert L.sbw_token_logprobs(*head, n, p(lp), p(ent), p(rank), p(m), p(z), p(ids), p(tops), None) == 0
            assert L.sbw_token_logprobs(*head, 0, p(lp), p(ent), p(rank), p(m), p(z), None, None, None) == 0
            assert L.sbw_token_logprobs_backward(*head, p(m), p(z), p(ent), p(lp), p(ent), p(grad) + es, V, None) == 0
        torch.cuda.synchronize()
        results.append([v.clone() for v in (lp, ent, rank, m, z, ids, tops, grad)])
        if L is dbg:
            mask, failures, passed, _ = _flags(dbg)
            assert mask == 0 and failures == 0 and (passed > 0 or B == 1)   # row 0 is a padded one
    assert all(torch.equal(a, b) for a, b in zip(*results))


@pytest.mark.parametrize("N,lmax", [(1, 0), (1, 3), (7, 40), (300, 300), (3000, 130), (2, 20000)])
def test_bounds_flag_build_of_weighted_detection(dbg, N, lmax):
    dev = require_gpu()
    tok, lens = inputs.null_token_streams(N, 0, lmax, 5000, N, dev)
    w = torch.rand(tok.numel(), device=dev)
    ws = torch.zeros(sbw.sbw_detect_workspace_bytes(N), dtype=torch.uint8, device=dev)
    results = []
    for L in (dbg, binding.lib()):
        _flags(dbg)
        z = torch.zeros(N, dtype=torch.float64, device=dev)
        for scheme in (0, 1):
            assert L.sbw_detect_weighted(tok.data_ptr(), w.data_ptr(), lens.data_ptr(), None, N, tok.numel(), 4, KEY, 0.25,
                                         scheme, None, None, None, z.data_ptr(), ws.data_ptr(), ws.numel(), None) == 0
        torch.cuda.synchronize()
        results.append(z.clone())
        if L is dbg:
            mask, failures, _, _ = _flags(dbg)
            assert mask == 0 and failures == 0
    assert torch.equal(*results)
