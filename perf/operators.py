"""The log-probability operators and the weighted detector as workloads: inputs, calls, and what they compute.

``run`` makes one call of an operator.  With ``own`` it is the library's call; without, the same result from
elementary torch operations.  ``exact`` computes it once more in 64 bits from the definition.

Operators (``op`` of a case):

* ``logprobs``  log probability, entropy and rank of one given token per row of logits, the row's softmax
  statistics, and its ``top`` most probable columns; optionally of the watermarked logits (Eq. 1 and Eq. 2 of the
  paper applied on the way, the logits themselves stay as they are);
* ``backward``  the gradient of those log probabilities and entropies with respect to the logits;
* ``weighted``  batch detection with a weight per token, as an entropy-weighted detector uses it.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

KEY = 0x5EED
CONTEXT, SELFSALT = 0, 1
MASK32 = 0xFFFFFFFF


def listed():
    return [
        # One user's decode step: the served answer carries its log probability and 20 alternatives.
        dict(name="logprobs, one decode row", op="logprobs", B=1, V=128256, dtype="bf16", std=4.0, tau=1.0, top=20,
             delta=0.0, gamma=0.5, scheme=CONTEXT, width=1, mask="none", pad=0.0, entropy=True),
        # A watermarked decode batch: log probabilities under the distribution that was sampled from.
        dict(name="logprobs, watermarked batch", op="logprobs", B=64, V=128256, dtype="bf16", std=4.0, tau=0.7, top=5,
             delta=2.0, gamma=0.5, scheme=CONTEXT, width=1, mask="none", pad=0.0, entropy=True),
        # The self-salt scheme over the paper's vocabulary size, fp32 logits, a large decode batch.
        dict(name="logprobs, self-salt fp32", op="logprobs", B=256, V=151936, dtype="f32", std=4.0, tau=0.7, top=20,
             delta=4.0, gamma=0.25, scheme=SELFSALT, width=1, mask="none", pad=0.0, entropy=True),
        # Padded prompts of odd vocabulary size with part of the vocabulary masked out.
        dict(name="logprobs, odd and masked", op="logprobs", B=301, V=32003, dtype="f32", std=3.0, tau=1.0, top=3,
             delta=0.0, gamma=0.5, scheme=CONTEXT, width=1, mask="inf", pad=0.2, entropy=True),
        # Scoring whole texts (perplexity, entropies): every position of a few long prompts.
        dict(name="logprobs, scoring texts", op="logprobs", B=4096, V=128256, dtype="bf16", std=4.0, tau=1.0, top=0,
             delta=0.0, gamma=0.5, scheme=CONTEXT, width=1, mask="none", pad=0.0, entropy=True),
        # A short training batch.
        dict(name="backward, small", op="backward", B=8, V=32000, dtype="f32", std=3.0, tau=1.0,
             delta=0.0, gamma=0.5, scheme=CONTEXT, width=1, mask="none", pad=0.0, entropy=False),
        # Fine-tuning batch, odd vocabulary, padded.
        dict(name="backward, odd and padded", op="backward", B=301, V=32003, dtype="f32", std=3.0, tau=1.0,
             delta=0.0, gamma=0.5, scheme=CONTEXT, width=1, mask="inf", pad=0.2, entropy=True),
        # Policy gradient on watermarked samples: gradient through the distribution that was sampled from.
        dict(name="backward, watermarked", op="backward", B=128, V=128256, dtype="bf16", std=4.0, tau=0.7,
             delta=2.0, gamma=0.25, scheme=CONTEXT, width=1, mask="none", pad=0.0, entropy=True),
        # A full training micro-batch of 2048 positions with an entropy bonus.
        dict(name="backward, training batch", op="backward", B=2048, V=128256, dtype="bf16", std=4.0, tau=1.0,
             delta=0.0, gamma=0.5, scheme=CONTEXT, width=1, mask="none", pad=0.0, entropy=True),
        # One suspected text of the paper's completion length.
        dict(name="weighted, one text", op="weighted", N=1, lmin=200, lmax=200, V=32000, scheme=CONTEXT, width=1,
             gamma=0.25),
        # An evaluation set of a thousand texts under the self-salt scheme with four context tokens.
        dict(name="weighted, evaluation set", op="weighted", N=1000, lmin=64, lmax=1024, V=128256, scheme=SELFSALT,
             width=4, gamma=0.25),
        # Corpus-scale screening.
        dict(name="weighted, corpus", op="weighted", N=100000, lmin=64, lmax=1024, V=128256, scheme=CONTEXT, width=1,
             gamma=0.25),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["logprobs", "logprobs", "backward", "backward", "weighted"])
    scheme = rng.choice([CONTEXT, SELFSALT])
    gamma = rng.choice([0.25, 0.5])
    width = rng.choice([1, 2, 4, 8])
    if op == "weighted":
        lmax = _log_uniform(rng, 10, 20000)
        return dict(op=op, N=max(1, min(_log_uniform(rng, 1, 100000), 50_000_000 // lmax)), lmin=rng.randint(0, lmax),
                    lmax=lmax, V=_log_uniform(rng, 1000, 200000), scheme=scheme, width=width, gamma=gamma)
    delta = rng.choice([0.0, 0.0, 1.0, 2.0, 5.0])
    V = _log_uniform(rng, 1000, 160000)
    top = rng.choice([0, rng.randint(1, 20)]) if op == "logprobs" else 0
    most = 30_000_000 if delta else 100_000_000 if top else 250_000_000
    case = dict(op=op, B=max(1, min(_log_uniform(rng, 1, 4096), most // V)), V=V, dtype=rng.choice(["bf16", "f32"]),
                std=rng.choice([1.0, 3.0, 4.0]), tau=rng.choice([0.7, 1.0, 1.3]), delta=delta, gamma=gamma,
                scheme=scheme, width=width, mask=rng.choice(["none", "none", "inf", "lowest"]),
                pad=rng.choice([0.0, 0.0, 0.1, 0.5]), entropy=rng.random() < 0.6 or op == "logprobs")
    if op == "logprobs":
        case["top"] = top
    return case


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 7919 + 17)
    if case["op"] == "weighted":
        N, V = case["N"], case["V"]
        lengths = torch.randint(case["lmin"], case["lmax"] + 1, (N,), generator=g, device="cuda", dtype=torch.int32)
        offsets = torch.zeros(N + 1, dtype=torch.int64, device="cuda")
        offsets[1:] = lengths.to(torch.int64).cumsum(0)
        total = int(offsets[-1])
        tokens = torch.randint(0, V, (total,), generator=g, device="cuda", dtype=torch.int32)
        # entropies of text: mostly small, a few large; a fifth below a threshold and not scored
        weights = torch.empty(total, device="cuda").exponential_(1.0, generator=g)
        weights = torch.where(torch.rand(total, generator=g, device="cuda") < 0.2, torch.zeros_like(weights), weights)
        new = lambda: torch.empty(N, dtype=torch.float64, device="cuda")  # noqa: E731
        return dict(case=case, tokens=tokens, weights=weights, lengths=lengths, offsets=offsets,
                    out=dict(green=new(), weight=new(), weight2=new(), z=new()))
    B, V, dt = case["B"], case["V"], _dtype(case)
    logits = torch.randn(B, V, generator=g, device="cuda").mul_(case["std"]).to(dt)
    ids = torch.randint(0, V, (B,), generator=g, device="cuda")
    # half of the tokens are ones the model finds likely, as in text; the others are any
    likely = torch.argmax(logits.float() + 4 * torch.rand(B, V, generator=g, device="cuda"), 1)
    ids = torch.where(torch.rand(B, generator=g, device="cuda") < 0.5, likely, ids)
    if case["mask"] != "none":
        low = -math.inf if case["mask"] == "inf" else torch.finfo(dt).min
        hidden = torch.rand(B, V, generator=g, device="cuda") < 0.3
        hidden.scatter_(1, ids[:, None], False)
        logits.masked_fill_(hidden, low)
    tokens = ids.to(torch.int32)
    if case["pad"]:
        tokens = torch.where(torch.rand(B, generator=g, device="cuda") < case["pad"], torch.full_like(tokens, -100), tokens)
    ctx = torch.randint(0, V, (B, case["width"]), generator=g, device="cuda", dtype=torch.int32)
    s = dict(case=case, logits=logits, tokens=tokens, ctx=ctx)
    f = lambda *shape: torch.empty(*shape, dtype=torch.float32, device="cuda")  # noqa: E731
    i = lambda *shape: torch.empty(*shape, dtype=torch.int32, device="cuda")  # noqa: E731
    if case["op"] == "logprobs":
        s["out"] = dict(logprob=f(B), entropy=f(B), rank=i(B), max=f(B), sumexp=f(B))
        if case["top"]:
            s["out"] |= dict(top_ids=i(B, case["top"]), top_logprobs=f(B, case["top"]))
        return s
    # what the forward call saved, and the gradients that come from the loss
    x = _biased(s)
    m = x.max(1).values.float()
    s["max"], s["sumexp"], s["entropy"] = f(B), f(B), f(B)
    step = max(1, 64_000_000 // V)
    for r in range(0, B, step):
        d = (x[r:r + step].double() - m[r:r + step, None].double()) / case["tau"]
        e = d.exp()
        z = e.sum(1)
        s["max"][r:r + step], s["sumexp"][r:r + step] = m[r:r + step], z
        s["entropy"][r:r + step] = z.log() - torch.where(e > 0, e * d, 0.0).sum(1) / z
    s["grad_logprob"] = torch.randn(B, generator=g, device="cuda")
    s["grad_entropy"] = 0.01 * torch.randn(B, generator=g, device="cuda") if case["entropy"] else None
    s["grad"] = torch.empty_like(logits)
    return s


# ---- the plain form -------------------------------------------------------------------------


def _mulhilo(a, b):
    p = a * b                                     # the low 64 bits of the product
    return (p >> 32) & MASK32, p & MASK32


def _philox0(v, r):
    """Word 0 of Philox4x32-10 with counter (v, 0, 0, 0) and key r, for int64 tensors of 32- and 64-bit values."""
    c0, c1, c2, c3 = v, torch.zeros_like(v), torch.zeros_like(v), torch.zeros_like(v)
    k0, k1 = r & MASK32, (r >> 32) & MASK32
    for _ in range(10):
        h0, l0 = _mulhilo(c0, 0xD2511F53)
        h1, l1 = _mulhilo(c2, 0xCD9E8D57)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & MASK32, (k1 + 0xBB67AE85) & MASK32
    return c0


def _jenkins(a):
    a = (a + 0x7ED55D16 + (a << 12)) & MASK32
    a = a ^ 0xC761C23C ^ (a >> 19)
    a = (a + 0x165667B1 + (a << 5)) & MASK32
    a = ((a + 0xD3A2646C) ^ (a << 9)) & MASK32
    a = (a + 0xFD7046C5 + (a << 3)) & MASK32
    return a ^ 0xB55A4F09 ^ (a >> 16)


def _green(v, ctx, case):
    """The green test of ids `v` after contexts `ctx` (ids along the last axis, which `v` lacks)."""
    if case["scheme"] == CONTEXT:
        r = ctx.sum(-1) * KEY
    else:
        j = _jenkins(v)
        r = j * torch.minimum(j, _jenkins(ctx).amin(-1)) * KEY
    return _philox0(v, r.expand_as(v)) < math.ceil(case["gamma"] * 2.0 ** 32)


def _biased(s):
    """The watermarked logits, in the logits' own precision."""
    case, x = s["case"], s["logits"]
    if not case["delta"]:
        return x
    v = torch.arange(case["V"], device="cuda").expand(case["B"], -1)
    green = _green(v, s["ctx"].to(torch.int64)[:, None, :], case)
    return torch.where(green, x + torch.tensor(case["delta"], dtype=x.dtype, device="cuda"), x)


def _plain_logprobs(s):
    case, V = s["case"], s["case"]["V"]
    x, t = _biased(s).float(), s["tokens"].to(torch.int64)
    real = (t >= 0) & (t < V)
    t = torch.where(real, t, 0)[:, None]
    m = x.max(1, keepdim=True).values
    d = torch.where(x > -math.inf, (x - m) / case["tau"], -math.inf)   # a row of -inf alone has no probability
    e = d.exp()
    z = e.sum(1, keepdim=True)
    logp = d - z.clamp_min(1e-30).log()
    entropy = -torch.where(e > 0, e * logp, 0.0).sum(1) / z[:, 0].clamp_min(1e-30)
    xt = x.gather(1, t)
    before = torch.arange(V, device="cuda") < t
    rank = 1 + ((x > xt) | ((x == xt) & before)).sum(1)
    zero = torch.zeros_like(entropy)
    out = dict(logprob=torch.where(real, logp.gather(1, t)[:, 0], zero), entropy=torch.where(real, entropy, zero),
               rank=torch.where(real, rank, 0).to(torch.int32), max=torch.where(real, m[:, 0], zero),
               sumexp=torch.where(real, z[:, 0], zero))
    if case["top"]:
        # values in order, as whole numbers, and lower columns first among equals
        bits = (x + 0.0).view(torch.int32).to(torch.int64) & MASK32
        code = torch.where(bits >= 0x80000000, MASK32 - bits, bits + 0x80000000)
        order = (code - 0x80000000) * 2 ** 32 + (MASK32 - torch.arange(V, device="cuda"))
        ids = order.topk(case["top"], 1).indices
        out["top_ids"] = torch.where(real[:, None], ids, -1).to(torch.int32)
        out["top_logprobs"] = torch.where(real[:, None], logp.gather(1, ids), -math.inf)
    return out


def _plain_backward(s):
    case, V = s["case"], s["case"]["V"]
    x, t = _biased(s).float(), s["tokens"].to(torch.int64)
    real = ((t >= 0) & (t < V))[:, None]
    d = ((x - s["max"][:, None]) / case["tau"]).clamp_min(-1e30)
    z = s["sumexp"][:, None]
    p = d.exp() / z
    g = s["grad_logprob"][:, None]
    hit = torch.arange(V, device="cuda") == t[:, None]
    grad = torch.where(hit, g * (1 - p), -g * p)
    if s["grad_entropy"] is not None:
        grad = grad - s["grad_entropy"][:, None] * p * (d - z.log() + s["entropy"][:, None])
    grad = torch.where(real, grad / case["tau"], 0.0)
    return grad.to(s["logits"].dtype)


def _plain_weighted(s):
    case, W = s["case"], s["case"]["width"]
    N, tok = case["N"], s["tokens"].to(torch.int64)
    total = tok.numel()
    text = torch.repeat_interleave(torch.arange(N, device="cuda"), s["lengths"].to(torch.int64), output_size=total)
    place = torch.arange(total, device="cuda")
    scored = place - s["offsets"][text] >= W
    back = (place[:, None] - torch.arange(1, W + 1, device="cuda")).clamp_min(0)
    green = _green(tok, tok[back], case)
    w = torch.where(scored, s["weights"].double(), 0.0)
    new = torch.zeros(N, dtype=torch.float64, device="cuda")
    G, S1, S2 = (new.index_add(0, text, v) for v in (torch.where(green, w, 0.0), w, w * w))
    gamma = case["gamma"]
    z = torch.where(S2 > 0, (G - gamma * S1) / (S2 * gamma * (1 - gamma)).clamp_min(1e-300).sqrt(), 0.0)
    return dict(green=G, weight=S1, weight2=S2, z=z)


# ---- one pass -------------------------------------------------------------------------------


def run(s):
    case = s["case"]
    if not own:
        return {"logprobs": _plain_logprobs, "backward": _plain_backward, "weighted": _plain_weighted}[case["op"]](s)
    import paper_2609_03844_b200 as sbw

    if case["op"] == "weighted":
        o = s["out"]
        sbw.sbw_detect_weighted(s["tokens"], s["weights"], s["lengths"], KEY, case["gamma"], case["scheme"], o["z"],
                                out_green=o["green"], out_weight=o["weight"], out_weight2=o["weight2"],
                                offsets=s["offsets"], ctx_width=case["width"])
        return o
    mark = dict(ctx_tokens=s["ctx"], key=KEY, gamma=case["gamma"], delta=case["delta"], scheme=case["scheme"]) \
        if case["delta"] else {}
    if case["op"] == "logprobs":
        o = s["out"]
        sbw.sbw_token_logprobs(s["logits"], s["tokens"], case["tau"], out_logprob=o["logprob"], out_entropy=o["entropy"],
                               out_rank=o["rank"], out_max=o["max"], out_sumexp=o["sumexp"],
                               out_top_ids=o.get("top_ids"), out_top_logprobs=o.get("top_logprobs"), **mark)
        return o
    return sbw.sbw_token_logprobs_backward(s["logits"], s["tokens"], case["tau"], s["max"], s["sumexp"], s["grad"],
                                           grad_logprob=s["grad_logprob"], entropy=s["entropy"],
                                           grad_entropy=s["grad_entropy"], **mark)


def work(case):
    if case["op"] == "weighted":
        # a token and its weight, a start and a length per text, four numbers per text back; the hash is whole-number work
        total = case["N"] * (case["lmin"] + case["lmax"]) / 2
        return dict(bytes=8 * total + 12 * case["N"] + 32 * case["N"], flops=0)
    size = 2 if case["dtype"] == "bf16" else 4
    rows = case["B"] * (1 - case["pad"])                      # nothing has to be read for a padded row
    context = 4 * case["width"] * rows if case["delta"] else 0
    if case["op"] == "logprobs":
        return dict(bytes=rows * case["V"] * size + context + case["B"] * (24 + 8 * case["top"]),
                    flops=4 * rows * case["V"])
    return dict(bytes=(rows + case["B"]) * case["V"] * size + context + case["B"] * 24, flops=4 * rows * case["V"])


# ---- the definition in 64 bits --------------------------------------------------------------


def _np_green(v, seeds, gamma):
    """Green tests on the host: ids and 64-bit seeds as uint64 arrays of one length."""
    lo, sh = np.uint64(MASK32), np.uint64(32)
    x = [v, np.zeros_like(v), np.zeros_like(v), np.zeros_like(v)]
    for n in range(10):
        key = [(seeds + np.uint64(n * 0x9E3779B9 & MASK32)) & lo, ((seeds >> sh) + np.uint64(n * 0xBB67AE85 & MASK32)) & lo]
        a, b = x[0] * np.uint64(0xD2511F53), x[2] * np.uint64(0xCD9E8D57)
        x = [(b >> sh) ^ x[1] ^ key[0], b & lo, (a >> sh) ^ x[3] ^ key[1], a & lo]
    return x[0].astype(np.float64) / 2.0 ** 32 < gamma


def _np_mix(a):
    """The integer hash of the self-salt seeds, on uint32 arrays (which wrap)."""
    u = np.uint32
    a = (a + u(0x7ED55D16)) + (a << u(12))
    a = (a ^ u(0xC761C23C)) ^ (a >> u(19))
    a = (a + u(0x165667B1)) + (a << u(5))
    a = (a + u(0xD3A2646C)) ^ (a << u(9))
    a = (a + u(0xFD7046C5)) + (a << u(3))
    return (a ^ u(0xB55A4F09)) ^ (a >> u(16))


def _np_seeds(v, windows, scheme):
    """64-bit seeds of ids `v` after the context ids `windows` [..., width], uint32 arrays."""
    if scheme == CONTEXT:
        return np.broadcast_to(windows.astype(np.uint64).sum(-1) * np.uint64(KEY), v.shape)
    j = _np_mix(v)
    least = np.minimum(j, _np_mix(windows).min(-1))
    return j.astype(np.uint64) * least.astype(np.uint64) * np.uint64(KEY)


def _exact_weighted(s):
    case, W = s["case"], s["case"]["width"]
    tok = s["tokens"].cpu().numpy().astype(np.uint32)
    w = s["weights"].cpu().numpy().astype(np.float64)
    starts, total = s["offsets"].cpu().numpy(), tok.size
    green, first = np.zeros(total, bool), np.ones(total, bool)
    for lo in range(W, total, 1 << 18):
        hi = min(total, lo + (1 << 18))
        windows = np.lib.stride_tricks.sliding_window_view(tok[lo - W:hi - 1], W)
        green[lo:hi] = _np_green(tok[lo:hi].astype(np.uint64), _np_seeds(tok[lo:hi], windows, case["scheme"]), case["gamma"])
    for k in range(W):                                    # the first tokens of a text only seed
        at = starts[:-1] + k
        first[at[at < starts[1:]]] = False
    w = np.where(first, w, 0.0)
    sums = [np.concatenate([[0.0], np.cumsum(v.astype(np.longdouble))]) for v in (w * green, w, w * w)]
    G, S1, S2 = ((c[starts[1:]] - c[starts[:-1]]).astype(np.float64) for c in sums)
    gone = S2 <= 0
    z = np.where(gone, 0.0, (G - case["gamma"] * S1) / np.sqrt(np.where(gone, 1.0, S2) * case["gamma"] * (1 - case["gamma"])))
    return dict(green=G, weight=S1, weight2=S2, z=z)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "weighted":
        return _exact_weighted(s)
    B, V, tau, dt = case["B"], case["V"], case["tau"], _dtype(case)
    ids = np.arange(V, dtype=np.uint32)
    parts = []
    step = max(1, 32_000_000 // V)
    for r in range(0, B, step):
        x = s["logits"][r:r + step]
        if case["delta"]:
            ctx = s["ctx"][r:r + step].cpu().numpy().astype(np.uint32)
            green = np.stack([_np_green(ids.astype(np.uint64), _np_seeds(ids, row, case["scheme"]), case["gamma"]) for row in ctx])
            add = torch.tensor(case["delta"]).to(dt).double()
            x = torch.where(torch.from_numpy(green).cuda(), (x.double() + add).to(dt), x)
        x, t = x.double(), s["tokens"][r:r + step].long()
        n = x.shape[0]
        pad = (t < 0) | (t >= V)
        at = t.clamp(0, V - 1)
        row = torch.arange(n, device="cuda")
        if case["op"] == "backward":
            d = (x - s["max"][r:r + step, None].double()) / tau
            logp = d - s["sumexp"][r:r + step, None].double().log()
            p = logp.exp()
            grad = -s["grad_logprob"][r:r + step, None].double() * p
            grad[row, at] += s["grad_logprob"][r:r + step].double()
            if s["grad_entropy"] is not None:
                surprise = torch.where(p > 0, p * (logp + s["entropy"][r:r + step, None].double()), 0.0)
                grad -= s["grad_entropy"][r:r + step, None].double() * surprise
            grad[pad] = 0
            parts.append(grad / tau)
            continue
        top = torch.logsumexp(x / tau, 1)
        logp = x / tau - top[:, None]
        p = logp.exp()
        m = x.amax(1)
        part = dict(logprob=logp[row, at], entropy=-torch.where(p > 0, p * logp, 0.0).sum(1),
                    max=m, sumexp=(top - m / tau).exp())
        for v in part.values():
            v[pad] = 0
        if case["top"]:
            best = logp.sort(dim=1, descending=True, stable=True).values[:, :case["top"]].clone()
            best[pad] = -math.inf
            part["top_logprobs"] = best
        parts.append(part)
    if case["op"] == "backward":
        return torch.cat(parts)
    return {k: torch.cat([p[k] for p in parts]) for k in parts[0]}
