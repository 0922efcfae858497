"""The projection to the vocabulary in 8-bit floating point, the quantiser before it and the sampler after it as
workloads: inputs, calls, and what they compute.

``run`` makes one call of an operator.  With ``own`` it is the library's call; without, the same result from
elementary torch operations.  ``exact`` computes it once more in 64 bits from the definition.

Operators (``op`` of a case):

* ``quantize``  values to e4m3 with one fp32 scale for each block of 128 columns (and of 1 or 128 rows);
* ``head``      logits of hidden states: the product with the vocabulary's weights, both in e4m3 with a scale for
  each block of 128, summed in 32 bits, optionally with the watermark (Eq. 1 and Eq. 2 of the paper) on the way out;
* ``sample``    one token per row from given random numbers, with temperature, top-k, top-p and min-p of its own for
  each row, optionally of the watermarked logits.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

KEY = 0x5EED
CONTEXT, SELFSALT = 0, 1
MASK32 = 0xFFFFFFFF
BLOCK = 128
# 2^f on [-1/2, 1/2]: (ln 2)^k / k!, highest power first, rounded to fp32 where it is used
EXP2 = [math.log(2.0) ** k / math.factorial(k) for k in range(7, -1, -1)]


def listed():
    return [
        # The hidden states of an ordinary decode batch on their way into the head.
        dict(name="quantize, decode batch", op="quantize", R=64, K=4096, block_rows=1, dtype="bf16"),
        # Weights of a head laid out once, as after a training step.
        dict(name="quantize, weights", op="quantize", R=128256, K=4096, block_rows=128, dtype="bf16"),
        # One user's decode step with a small model.
        dict(name="head, one token, small", op="head", B=1, V=32000, K=2048, dtype="f32", delta=0.0, gamma=0.5,
             scheme=CONTEXT, width=1),
        # One user's decode step with a large vocabulary.
        dict(name="head, one token", op="head", B=1, V=128256, K=4096, dtype="bf16", delta=0.0, gamma=0.5,
             scheme=CONTEXT, width=1),
        # A watermarked decode batch.
        dict(name="head, watermarked batch", op="head", B=64, V=128256, K=4096, dtype="bf16", delta=2.0, gamma=0.5,
             scheme=CONTEXT, width=1),
        # Odd sizes everywhere, fp32 logits.
        dict(name="head, odd", op="head", B=301, V=32003, K=2300, dtype="f32", delta=0.0, gamma=0.5, scheme=CONTEXT,
             width=1),
        # The positions of a few prompts that are scored.
        dict(name="head, prompts", op="head", B=2048, V=128256, K=4096, dtype="bf16", delta=0.0, gamma=0.5,
             scheme=CONTEXT, width=1),
        # One user's answer, top-p alone.
        dict(name="sample, one row", op="sample", B=1, V=128256, dtype="bf16", std=4.0, peak=True, mixed=False, tau=0.7,
             top_k=0, top_p=0.95, min_p=0.0, mask="none", delta=0.0, gamma=0.5, scheme=CONTEXT, width=1),
        # A serving batch in which every request has settings of its own, watermarked.
        dict(name="sample, mixed and watermarked", op="sample", B=64, V=128256, dtype="bf16", std=4.0, peak=True,
             mixed=True, tau=0.7, top_k=0, top_p=1.0, min_p=0.0, mask="none", delta=2.0, gamma=0.5, scheme=CONTEXT,
             width=1),
        # The paper's settings (temperature 0.7, top-p 0.8) on its vocabulary size, fp32 logits.
        dict(name="sample, top-p fp32", op="sample", B=256, V=151936, dtype="f32", std=4.0, peak=True, mixed=False,
             tau=0.7, top_k=0, top_p=0.8, min_p=0.0, mask="none", delta=0.0, gamma=0.5, scheme=CONTEXT, width=1),
        # Odd vocabulary, part of it masked out, all three filters.
        dict(name="sample, odd and masked", op="sample", B=301, V=32003, dtype="f32", std=3.0, peak=False, mixed=False,
             tau=1.0, top_k=50, top_p=0.9, min_p=0.02, mask="inf", delta=0.0, gamma=0.5, scheme=CONTEXT, width=1),
        # Many answers at once from the whole distribution (texts for a detector's evaluation).
        dict(name="sample, large batch", op="sample", B=1024, V=128256, dtype="bf16", std=4.0, peak=False, mixed=False,
             tau=1.0, top_k=0, top_p=1.0, min_p=0.0, mask="none", delta=0.0, gamma=0.5, scheme=CONTEXT, width=1),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["quantize", "head", "head", "sample", "sample"])
    dtype = rng.choice(["bf16", "f32"])
    if op == "quantize":
        K = _log_uniform(rng, 64, 16384)
        return dict(op=op, R=max(1, min(_log_uniform(rng, 1, 128256), 250_000_000 // K)), K=K,
                    block_rows=rng.choice([1, 128]), dtype=dtype)
    mark = dict(delta=rng.choice([0.0, 0.0, 2.0]), gamma=rng.choice([0.25, 0.5]), scheme=rng.choice([CONTEXT, SELFSALT]),
                width=rng.choice([1, 2, 4, 8]))
    V = _log_uniform(rng, 1000, 160000)
    if op == "head":
        K = _log_uniform(rng, 64, 8192)
        most = min(130_000_000 if mark["delta"] == 0.0 else 30_000_000, 1_000_000_000_000 // K)
        return dict(op=op, B=max(1, min(_log_uniform(rng, 1, 2048), most // V)), V=V, K=K, dtype=dtype, **mark)
    most = 130_000_000 if mark["delta"] == 0.0 else 30_000_000
    return dict(op=op, B=max(1, min(_log_uniform(rng, 1, 1024), most // V)), V=V, dtype=dtype,
                std=rng.choice([1.0, 3.0, 4.0]), peak=rng.random() < 0.5, mixed=rng.random() < 0.4,
                tau=rng.choice([0.5, 0.7, 1.0, 1.3]), top_k=rng.choice([0, 0, _log_uniform(rng, 1, 1000)]),
                top_p=rng.choice([1.0, 0.8, 0.95, rng.uniform(0.05, 1.0)]), min_p=rng.choice([0.0, 0.0, 0.02, 0.1]),
                mask=rng.choice(["none", "none", "inf", "lowest"]), **mark)


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _blocks(n):
    return -(-n // BLOCK)


def _hidden(R, K, g):
    """Activations as a model has them: a few channels are much larger than the others."""
    channel = torch.exp(0.8 * torch.randn(K, generator=g, device="cuda"))
    return torch.randn(R, K, generator=g, device="cuda").mul_(channel)


def _in_blocks(x, rows, fill=0.0):
    """[R, K] as [R / rows, rows, K / 128, 128], filled up."""
    R, K = x.shape
    x = torch.nn.functional.pad(x, (0, _blocks(K) * BLOCK - K, 0, -(-R // rows) * rows - R), value=fill)
    return x.view(-1, rows, _blocks(K), BLOCK)


def _quantized(x, rows):
    """Codes (e4m3) and scales of x."""
    R, K = x.shape
    b = _in_blocks(x, rows)
    scale = (b.abs().amax((1, 3)) / 448.0).clamp_min(2.0 ** -126)
    q = (b / scale[:, None, :, None]).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)
    return q.view(b.shape[0] * rows, -1)[:R, :K], scale


def _on_16(q):
    """The same codes with rows that start on 16-byte boundaries, as the head takes them."""
    R, K = q.shape
    full = torch.zeros(R, -(-K // 16) * 16, dtype=torch.uint8, device="cuda")
    full[:, :K] = q.view(torch.uint8)
    return full.view(torch.float8_e4m3fn)[:, :K]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 7919 + 29)
    dt = _dtype(case)
    if case["op"] == "quantize":
        R, K, rows = case["R"], case["K"], case["block_rows"]
        x = (_hidden(R, K, g) if rows == 1 else torch.randn(R, K, generator=g, device="cuda").mul_(0.02)).to(dt)
        return dict(case=case, x=x, codes=torch.empty(R, K, dtype=torch.float8_e4m3fn, device="cuda"),
                    scales=torch.empty(-(-R // rows), _blocks(K), dtype=torch.float32, device="cuda"))
    B, V = case["B"], case["V"]
    ctx = torch.randint(0, V, (B, case["width"]), generator=g, device="cuda", dtype=torch.int32)
    if case["op"] == "head":
        K = case["K"]
        x, xs = _quantized(_hidden(B, K, g), 1)
        w, ws = _quantized(torch.randn(V, K, generator=g, device="cuda").mul_(1.5 / math.sqrt(K)), BLOCK)
        return dict(case=case, x=_on_16(x), xs=xs, w=_on_16(w), ws=ws, ctx=ctx,
                    logits=torch.empty(B, V, dtype=dt, device="cuda"))
    logits = torch.randn(B, V, generator=g, device="cuda").mul_(case["std"])
    if case["peak"]:
        # half of the rows are steps at which the model is sure of itself
        at = torch.randint(0, V, (B, 8), generator=g, device="cuda")
        sure = (torch.rand(B, 1, generator=g, device="cuda") < 0.5) * torch.linspace(16.0, 4.0, 8, device="cuda")
        logits.scatter_add_(1, at, sure.expand(B, 8))
    logits = logits.to(dt)
    if case["mask"] != "none":
        low = -math.inf if case["mask"] == "inf" else torch.finfo(dt).min
        logits.masked_fill_(torch.rand(B, V, generator=g, device="cuda") < 0.3, low)
    if case["mixed"]:
        pick = lambda *of: torch.tensor(of, device="cuda")[torch.randint(0, len(of), (B,), generator=g, device="cuda")]  # noqa: E731
        tau, k = pick(0.0, 0.5, 0.7, 1.0, 1.3), pick(0, 0, 1, 20, 50, 1000).to(torch.int32)
        p, low_p = pick(1.0, 0.8, 0.95), pick(0.0, 0.0, 0.05)
    else:
        all_of = lambda v: torch.full((B,), v, device="cuda", dtype=torch.float32)  # noqa: E731
        tau, p, low_p = all_of(case["tau"]), all_of(case["top_p"]), all_of(case["min_p"])
        k = torch.full((B,), case["top_k"], device="cuda", dtype=torch.int32)
    return dict(case=case, logits=logits, ctx=ctx, uniforms=torch.rand(B, generator=g, device="cuda"),
                temperature=tau, top_k=k, top_p=p, min_p=low_p,
                out=dict(tokens=torch.empty(B, dtype=torch.int32, device="cuda"),
                         prob=torch.empty(B, dtype=torch.float32, device="cuda"),
                         kept=torch.empty(B, dtype=torch.int32, device="cuda")))


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


def _biased(x, s):
    """The watermarked logits, in the logits' own precision."""
    case = s["case"]
    if not case["delta"]:
        return x
    v = torch.arange(case["V"], device="cuda").expand(case["B"], -1)
    ctx = s["ctx"].to(torch.int64)
    if case["scheme"] == CONTEXT:
        r = (ctx.sum(1, keepdim=True) * KEY).expand_as(v)
    else:
        j = _jenkins(v)
        r = j * torch.minimum(j, _jenkins(ctx).amin(1, keepdim=True)) * KEY
    green = _philox0(v, r) < math.ceil(case["gamma"] * 2.0 ** 32)
    return torch.where(green, x + torch.tensor(case["delta"], dtype=x.dtype, device="cuda"), x)


def _plain_quantize(s):
    codes, scales = _quantized(s["x"].float(), s["case"]["block_rows"])
    return dict(codes=codes, scales=scales)


def _plain_head(s):
    K, V = s["case"]["K"], s["case"]["V"]
    x = s["x"].float() * s["xs"].repeat_interleave(BLOCK, 1)[:, :K]
    w = s["w"].float() * s["ws"].repeat_interleave(BLOCK, 1)[:, :K].repeat_interleave(BLOCK, 0)[:V]
    return _biased((x @ w.T).to(_dtype(s["case"])), s)


def _share(p32, Z):
    """floor(p32 Z / 2^32) and whether the division leaves a rest, for p32 of up to 33 bits and Z of up to 61."""
    hi, lo = Z >> 32, Z & MASK32
    a, b = (p32 >> 16) * lo, (p32 & 0xFFFF) * lo
    return p32 * hi + ((a + (b >> 16)) >> 16), ((a & 0xFFFF) << 16) + b & MASK32


def _plain_sample(s):
    V = s["case"]["V"]
    x = _biased(s["logits"], s).float()
    x = torch.where(x.isnan(), -math.inf, x)
    greedy = ~(s["temperature"] >= 1e-6)
    c = (1.4426950408889634 / torch.where(greedy, 1.0, s["temperature"]).double()).float()
    lowest = torch.where(s["min_p"] > 0, s["min_p"].double().log2().float(), -math.inf).clamp(-41.0, 0.0)
    lowest = torch.where(greedy, -41.0, lowest)
    k = torch.where(greedy, 1, torch.where(s["top_k"] > 0, s["top_k"], V))[:, None]
    p32 = torch.where(s["top_p"] < 1, (s["top_p"].double() * 2.0 ** 32).floor().clamp(1, 2.0 ** 32), 2.0 ** 32)
    p32 = p32.to(torch.int64)[:, None]
    u32 = (s["uniforms"].double().clamp(0, 1) * 2.0 ** 32).floor().clamp(max=2.0 ** 32 - 1).to(torch.int64)[:, None]

    x, order = torch.sort(x, dim=1, descending=True, stable=True)
    m = x[:, :1]
    y = torch.where(x == m, 0.0, (x - m) * c[:, None])
    n = y.clamp(-60.0, 0.0).round()
    f = (y.clamp(-60.0, 0.0) - n).double()
    e = torch.full_like(y, EXP2[0])
    for a in EXP2[1:]:                            # one rounding to 32 bits per step
        e = (e.double() * f + float(np.float32(a))).float()
    weight = (e.double() * (1 << (n.to(torch.int64) + 62)).double() * 2.0 ** -22).to(torch.int64)
    real = (y >= lowest[:, None]) & (m > -math.inf) & (torch.arange(V, device="cuda") < k)
    weight = torch.where(real, weight, 0)
    run = weight.cumsum(1)
    need, rest = _share(p32, run[:, -1:])
    weight = torch.where(run - weight < need + (rest > 0), weight, 0)
    total = weight.sum(1, keepdim=True)
    target, _ = _share(u32, total)
    at = (run <= target).sum(1, keepdim=True).clamp(max=V - 1)
    some = total[:, 0] > 0
    return dict(tokens=torch.where(some, order.gather(1, at)[:, 0], 0).to(torch.int32),
                prob=(weight.gather(1, at).double() / total.clamp_min(1).double())[:, 0].float(),
                kept=(weight > 0).sum(1).to(torch.int32))


# ---- one pass -------------------------------------------------------------------------------


def run(s):
    case = s["case"]
    if not own:
        return {"quantize": _plain_quantize, "head": _plain_head, "sample": _plain_sample}[case["op"]](s)
    import paper_2609_03844_b200 as sbw

    if case["op"] == "quantize":
        sbw.sbw_quantize_fp8(s["x"], s["codes"], s["scales"], block_rows=case["block_rows"])
        return dict(codes=s["codes"], scales=s["scales"])
    mark = dict(ctx_tokens=s["ctx"], key=KEY, gamma=case["gamma"], delta=case["delta"], scheme=case["scheme"]) \
        if case["delta"] else {}
    if case["op"] == "head":
        return sbw.sbw_head_logits(s["x"], s["xs"], s["w"], s["ws"], s["logits"], **mark)
    o = s["out"]
    sbw.sbw_sample_given(s["logits"], s["uniforms"], o["tokens"], temperature=s["temperature"], top_k=s["top_k"],
                         top_p=s["top_p"], min_p=s["min_p"], out_prob=o["prob"], out_kept=o["kept"], **mark)
    return o


def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "quantize":
        n = case["R"] * case["K"]
        return dict(bytes=n * (size + 1) + 4 * -(-case["R"] // case["block_rows"]) * _blocks(case["K"]), flops=2 * n)
    B, V = case["B"], case["V"]
    context = 4 * case["width"] * B if case["delta"] else 0
    if case["op"] == "head":
        K = case["K"]
        scales = 4 * _blocks(K) * (B + _blocks(V))
        return dict(bytes=(B + V) * K + scales + B * V * size + context, flops=2 * B * V * K)
    return dict(bytes=B * V * size + 32 * B + context, flops=20 * B * V)


# ---- the definition in 64 bits --------------------------------------------------------------


def _np_green(ids, seeds, gamma):
    """Green tests on the host: ids and 64-bit seeds as uint64 arrays of one length."""
    lo, sh = np.uint64(MASK32), np.uint64(32)
    x = [ids, np.zeros_like(ids), np.zeros_like(ids), np.zeros_like(ids)]
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


def _np_greens(s):
    """[B, V] truth values: which columns of which row are green."""
    case = s["case"]
    ids = np.arange(case["V"], dtype=np.uint32)
    rows = []
    for window in s["ctx"].cpu().numpy().astype(np.uint32):
        if case["scheme"] == CONTEXT:
            seeds = np.full(ids.shape, window.astype(np.uint64).sum() * np.uint64(KEY))
        else:
            j = _np_mix(ids)
            seeds = j.astype(np.uint64) * np.minimum(j, _np_mix(window).min()).astype(np.uint64) * np.uint64(KEY)
        rows.append(_np_green(ids.astype(np.uint64), seeds, case["gamma"]))
    return torch.from_numpy(np.stack(rows)).cuda()


def _exact_quantize(s):
    """The largest magnitudes over 448; codes are choices between neighbours, not numbers with a value in 64 bits."""
    x = s["x"].double()
    rows = s["case"]["block_rows"]
    return dict(codes=None, scales=(_in_blocks(x, rows).abs().amax((1, 3)) / 448.0).clamp_min(2.0 ** -126))


def _exact_head(s):
    case, K, V = s["case"], s["case"]["K"], s["case"]["V"]
    at = torch.arange(K, device="cuda") // BLOCK
    x = s["x"].double() * s["xs"].double()[:, at]
    out = torch.empty(case["B"], V, dtype=torch.float64, device="cuda")
    for v in range(0, V, 16384):
        rows = torch.arange(v, min(V, v + 16384), device="cuda") // BLOCK
        out[:, v:v + 16384] = x @ (s["w"][v:v + 16384].double() * s["ws"].double()[rows][:, at]).T
    if case["delta"]:
        out += _np_greens(s) * float(torch.tensor(case["delta"]).to(_dtype(case)))
    return out


def _exact_sample(s):
    """The token that the integer weights give, found on the host row by row, and its probability among the columns that
    were kept as an exponential and a sum in 64 bits."""
    case = s["case"]
    x = s["logits"]
    if case["delta"]:
        add = float(torch.tensor(case["delta"]).to(x.dtype))
        x = torch.where(_np_greens(s), (x.double() + add).to(x.dtype), x)
    x = x.float().cpu().numpy()
    given = [s[n].cpu().numpy() for n in ("temperature", "top_k", "top_p", "min_p", "uniforms")]
    tokens, prob, kept = [], [], []
    for row, tau, k, p, low, u in zip(x, *given):
        if not row.max() > -np.inf:
            tokens.append(0), prob.append(0.0), kept.append(0)
            continue
        c, least = np.float32(1.0), -41.0
        if tau >= 1e-6:
            c = np.float32(math.log2(math.e) / float(tau))
            least = max(-41.0, min(0.0, float(np.float32(math.log2(low))))) if low > 0 else -41.0
        else:
            k, p = 1, 1.0
        with np.errstate(over="ignore"):
            y = (row - row.max()) * c
        cols = np.flatnonzero(y >= least)
        cols = cols[np.argsort(-row[cols], kind="stable")]
        cols = cols[:k] if k > 0 else cols
        n = np.rint(y[cols])
        f = (y[cols] - n).astype(np.float64)
        e = np.zeros_like(n)
        for a in EXP2:
            e = (e.astype(np.float64) * f + np.float64(np.float32(a))).astype(np.float32)
        run = np.cumsum(np.floor(np.ldexp(e.astype(np.float64), n.astype(np.int64) + 40)).astype(np.int64))
        if p < 1:
            p32 = max(1, math.floor(float(p) * 2 ** 32))
            need = (p32 * int(run[-1]) + MASK32) >> 32
            run = run[:int(np.searchsorted(run, need)) + 1]
        at = int(np.searchsorted(run, math.floor(float(u) * 2 ** 32) * int(run[-1]) >> 32, side="right"))
        full = np.exp((row[cols[:len(run)]].astype(np.float64) - float(row.max())) / (float(tau) if tau >= 1e-6 else 1.0))
        tokens.append(int(cols[at])), prob.append(full[at] / full.sum())
        kept.append(int(np.count_nonzero(np.diff(run, prepend=0))))
    return dict(tokens=torch.tensor(tokens, dtype=torch.int32), prob=torch.tensor(prob, dtype=torch.float64),
                kept=torch.tensor(kept, dtype=torch.int32))


def exact(case, seed):
    if case["op"] == "sample" and case["B"] * case["V"] > 45_000_000 or case.get("delta") and case["B"] * case["V"] > 12_000_000:
        return None                               # the host takes too long over its rows
    s = prepare(case, seed)
    return {"quantize": _exact_quantize, "head": _exact_head, "sample": _exact_sample}[case["op"]](s)
