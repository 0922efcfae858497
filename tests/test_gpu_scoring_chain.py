"""The calls together, as a scoring run uses them: sample watermarked texts from a small random language model, take log
probabilities and entropies of their tokens, weigh the detector with the entropies, compare with null texts by ROC-AUC;
and one training step on the log probabilities."""
import numpy as np
import pytest
import torch

import paper_2609_03844_b200 as sbw
from paper_2609_03844_b200 import inputs
from gpu_util import KEY, host_bits, require_gpu

pytestmark = pytest.mark.gpu
GAMMA, DELTA, TAU, V, N, L = 0.25, 3.0, 1.0, 2003, 60, 80


def texts(dev):
    """N texts of L tokens by watermarked sampling, with the logits each token was sampled from."""
    base = inputs.logits_normal(64, V, 1.0, torch.float32, seed=5, device=dev)
    sharp = torch.rand(64, 1, generator=torch.Generator(device=dev).manual_seed(6), device=dev) * 6
    tok = torch.empty((N, L), dtype=torch.int32, device=dev)
    tok[:, 0] = inputs.uniform_tokens((N,), V, 7, dev)
    ws = torch.empty(sbw.sbw_sample_workspace_bytes(N, V), dtype=torch.uint8, device=dev)
    logits = []
    for i in range(1, L):
        prev = tok[:, i - 1].contiguous()
        x = (base * (1 + sharp))[(prev % 64).long()].contiguous()       # some states know what comes next, others do not
        out = torch.empty(N, dtype=torch.int32, device=dev)
        sbw.sbw_bias_sample(x, prev[:, None].contiguous(), KEY, GAMMA, DELTA, 0, TAU, 3, i, out, ws)
        tok[:, i] = out
        logits.append(x)
    return tok, torch.stack(logits, 1)


def test_scoring_and_weighted_detection(oracle):
    dev = require_gpu()
    tok, logits = texts(dev)
    rows = logits.reshape(N * (L - 1), V)
    ids = tok[:, 1:].reshape(-1).contiguous()
    lp, ent = (torch.empty(rows.shape[0], device=dev) for _ in range(2))
    sbw.sbw_token_logprobs(rows, ids, TAU, out_logprob=lp, out_entropy=ent)
    want = oracle.token_logprobs(host_bits(rows), V, ids.cpu().numpy(), TAU)
    assert np.abs(lp.cpu().numpy() - want["logprob"]).max() < 8e-6 + 2.0 ** -21 * 60
    ppl = torch.exp(-lp.view(N, L - 1).mean(1))
    assert torch.isfinite(ppl).all()

    weights = torch.zeros((N, L), device=dev)
    weights[:, 1:] = ent.view(N, L - 1)
    null = inputs.uniform_tokens((N, L), V, 11, dev)
    every = torch.cat([tok, null]).reshape(-1).contiguous()
    w = torch.cat([weights, weights]).reshape(-1).contiguous()
    lens = torch.full((2 * N,), L, dtype=torch.int32, device=dev)
    z = torch.empty(2 * N, dtype=torch.float64, device=dev)
    ws = torch.empty(sbw.sbw_detect_workspace_bytes(2 * N), dtype=torch.uint8, device=dev)
    sbw.sbw_detect_weighted(every, w, lens, KEY, GAMMA, 0, z, workspace=ws)
    ref = oracle.detect_weighted(every.cpu().numpy(), w.cpu().numpy(), lens.cpu().numpy(), KEY, GAMMA, 0)[3]
    assert np.abs(z.cpu().numpy() - ref).max() < 1e-9
    labels = torch.cat([torch.ones(N), torch.zeros(N)]).to(torch.uint8).to(dev)
    auc = torch.empty(1, dtype=torch.float64, device=dev)
    rws = torch.empty(sbw.binding.lib().sbw_roc_auc_workspace_bytes(2 * N), dtype=torch.uint8, device=dev)
    sbw.sbw_roc_auc(z, labels, auc, rws)
    want_auc, _ = oracle.roc_auc(ref, labels.cpu().numpy())
    assert abs(float(auc) - want_auc) < 1e-12


def test_forward_and_backward_as_a_training_step():
    """The gradient of mean log probability plus entropy bonus through the two calls against autograd in fp64."""
    dev = require_gpu()
    B = 90
    x = inputs.logits_normal(B, V, 2.0, torch.float32, seed=9, device=dev)
    t = inputs.uniform_tokens((B,), V, 10, dev)
    t[::4] = -100                                        # prompt tokens
    real = t >= 0
    lp, ent, m, z = (torch.empty(B, device=dev) for _ in range(4))
    sbw.sbw_token_logprobs(x, t, 0.75, out_logprob=lp, out_entropy=ent, out_max=m, out_sumexp=z)
    count = int(real.sum())
    g, h = torch.full((B,), -1.0 / count, device=dev), torch.full((B,), -0.1 / count, device=dev)
    grad = torch.empty_like(x)
    sbw.sbw_token_logprobs_backward(x, t, 0.75, m, z, grad, grad_logprob=g, entropy=ent, grad_entropy=h)
    y = x.double().requires_grad_(True)
    logp = torch.log_softmax(y / 0.75, 1)
    loss = -(logp[torch.arange(B), t.clamp(0).long()] - 0.1 * (logp.exp() * logp).sum(1))[real].sum() / count
    loss.backward()
    ours = float((g * lp + h * ent).double().sum())
    # the mean of the rows' errors 8e-6 + 2^-21 (H + |log p|) and 0.1 * 16e-6 (1 + H), H < 7.7, |log p| < 30
    assert abs(ours - float(loss.detach())) < 8e-6 + 2.0 ** -21 * 38 + 1.6e-6 * 8.7
    # saved Z and H are off by up to 8e-6 + 2^-21 H relative and 16e-6 (1 + H): p and its factor follow them
    p = logp.exp().detach()
    tol = (p * (1 + 0.1 * (logp.detach().abs() + 8)) * 5e-5 + 1e-7) / 0.75 / count + 1e-9
    assert torch.all((grad.double() - y.grad).abs() <= tol)
    assert torch.all(grad[~real] == 0)
