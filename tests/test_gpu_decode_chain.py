"""The calls of a decode step together: hidden states are quantised, projected to the vocabulary with the watermark on the
way out, and sampled from given random numbers; the texts are detected.  And the calls captured, on other streams, and
without allocations."""
import numpy as np
import pytest
import torch

import paper_2609_03844_b200 as sbw
from gpu_util import KEY, assert_same_bits, host_bits, require_gpu
from oracle import given

pytestmark = pytest.mark.gpu
V, K, N, L, GAMMA, DELTA = 2003, 384, 48, 60, 0.25, 4.0
E4M3 = torch.float8_e4m3fn


class Model:
    """A random language model: a hidden state per preceding token, and a head."""

    def __init__(self, dtype):
        g = torch.Generator().manual_seed(1)
        self.states = torch.randn(V, K, generator=g).cuda()
        w = torch.randn(V, K, generator=g).cuda() * (2.0 / K ** 0.5)
        self.w, self.ws = torch.empty(V, K, dtype=E4M3, device="cuda"), torch.empty(16, 3, device="cuda")
        sbw.sbw_quantize_fp8(w, self.w, self.ws, block_rows=128)
        self.x, self.xs = torch.empty(N, K, dtype=E4M3, device="cuda"), torch.empty(N, 3, device="cuda")
        self.logits = torch.empty(N, V, dtype=dtype, device="cuda")
        self.hidden = torch.empty(N, K, device="cuda")
        self.prev = torch.zeros(N, 1, dtype=torch.int32, device="cuda")
        self.u = torch.empty(N, device="cuda")
        self.settings = dict(temperature=torch.full((N,), 0.9, device="cuda"), top_k=torch.full((N,), 400, dtype=torch.int32, device="cuda"),
                             top_p=torch.full((N,), 0.95, device="cuda"), min_p=torch.full((N,), 0.001, device="cuda"))
        self.out = torch.empty(N, dtype=torch.int32, device="cuda")

    def step(self, delta=DELTA):
        torch.index_select(self.states, 0, self.prev[:, 0], out=self.hidden)
        sbw.sbw_quantize_fp8(self.hidden, self.x, self.xs)
        sbw.sbw_head_logits(self.x, self.xs, self.w, self.ws, self.logits, ctx_tokens=self.prev, key=KEY, gamma=GAMMA, delta=delta)
        sbw.sbw_sample_given(self.logits, self.u, self.out, **self.settings)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_decode_and_detect(dtype):
    require_gpu()
    m = Model(dtype)
    g = torch.Generator(device="cuda").manual_seed(2)
    texts = {}
    for delta in (DELTA, 0.0):
        tok = torch.empty(N, L, dtype=torch.int32, device="cuda")
        tok[:, 0] = torch.arange(N, device="cuda")
        for i in range(1, L):
            m.prev.copy_(tok[:, i - 1:i])
            m.u.uniform_(generator=g)
            m.step(delta)
            tok[:, i] = m.out
            if i % 20 == 1:
                # the fused projection against the two calls, the token against the definition
                plain = sbw.sbw_head_logits(m.x, m.xs, m.w, m.ws, torch.empty_like(m.logits))
                sbw.sbw_bias_logits(plain, m.prev, KEY, GAMMA, delta, 0)
                assert_same_bits(host_bits(m.logits), host_bits(plain))
                s = {k: v.cpu().numpy() for k, v in m.settings.items()}
                want = given.sample(plain.float().cpu().numpy(), m.u.cpu().numpy(), s["temperature"], s["top_k"], s["top_p"], s["min_p"])
                assert np.array_equal(m.out.cpu().numpy(), want[0])
                # sampling the plain logits with the watermark is the same draw
                again = torch.empty_like(m.out)
                sbw.sbw_head_logits(m.x, m.xs, m.w, m.ws, m.logits)
                sbw.sbw_sample_given(m.logits, m.u, again, ctx_tokens=m.prev, key=KEY, gamma=GAMMA, delta=delta, **m.settings)
                assert torch.equal(again, m.out)
        texts[delta] = tok
    z = {}
    for delta, tok in texts.items():
        z[delta] = torch.empty(N, dtype=torch.float64, device="cuda")
        counts = torch.empty(N, dtype=torch.int32, device="cuda")
        ws = torch.empty(sbw.sbw_detect_workspace_bytes(N), dtype=torch.uint8, device="cuda")
        sbw.sbw_detect(tok.reshape(-1).contiguous(), torch.full((N,), L, dtype=torch.int32, device="cuda"), KEY, GAMMA, 0, counts,
                       z[delta], workspace=ws)
    assert float(z[DELTA].min()) > 4 and abs(float(z[0.0].mean())) < 1


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_captured_step_and_other_streams(dtype):
    require_gpu()
    a, b = Model(dtype), Model(dtype)
    a.u.fill_(0.3)
    a.step()                                             # loads the kernels outside the capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.step()
        a.step()
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    side = torch.cuda.Stream()
    for seed in range(4):
        g = torch.Generator(device="cuda").manual_seed(seed)
        for m in (a, b):
            m.prev.copy_(torch.randint(0, V, (N, 1), generator=g, device="cuda", dtype=torch.int32))
            m.u.uniform_(generator=g)
            g.manual_seed(seed)
        torch.cuda.synchronize()
        graph.replay()
        with torch.cuda.stream(side):
            b.step()
            b.step()
        torch.cuda.synchronize()
        assert torch.equal(a.out, b.out) and torch.equal(a.logits, b.logits)
    assert torch.cuda.memory_allocated() == before


def test_the_library_allocates_nothing():
    require_gpu()
    m = Model(torch.bfloat16)
    m.u.fill_(0.7)
    for _ in range(3):
        m.step()
    torch.cuda.synchronize()
    free = torch.cuda.mem_get_info()[0]
    for _ in range(50):
        m.step()
    torch.cuda.synchronize()
    assert torch.cuda.mem_get_info()[0] == free


def test_rows_of_a_batch_do_not_depend_on_each_other():
    """The sampler's clusters, one CTA per row, and what is between: the same rows in batches of any size."""
    require_gpu()
    for dtype in (torch.float32, torch.bfloat16):
        x = (3 * torch.randn(300, 9000, generator=torch.Generator().manual_seed(3))).to(dtype).cuda()
        u, t = torch.rand(300, generator=torch.Generator().manual_seed(4)).cuda(), torch.full((300,), 0.8, device="cuda")
        p = torch.full((300,), 0.9, device="cuda")
        every = torch.empty(300, dtype=torch.int32, device="cuda")
        sbw.sbw_sample_given(x, u, every, temperature=t, top_p=p)
        for n in (1, 9, 40, 120, 200):
            out = torch.empty(n, dtype=torch.int32, device="cuda")
            sbw.sbw_sample_given(x[:n], u[:n], out, temperature=t[:n], top_p=p[:n])
            assert torch.equal(out, every[:n])


def test_elements_beyond_32_bits():
    """More than 2^31 logits in one batch: the last rows are what they are alone."""
    require_gpu()
    B, big_v, k = 17000, 128256, 64
    x, w = (torch.randint(0, 0x70, s, dtype=torch.uint8, device="cuda", generator=torch.Generator(device="cuda").manual_seed(5)).view(E4M3)
            for s in ((B, k), (big_v, k)))
    xs, ws = torch.full((B, 1), 0.01, device="cuda"), torch.full((1002, 1), 0.01, device="cuda")
    ctx = torch.arange(B, dtype=torch.int32, device="cuda")[:, None].contiguous()
    logits = torch.empty(B, big_v, dtype=torch.bfloat16, device="cuda")
    mark = dict(key=KEY, gamma=GAMMA, delta=DELTA)
    sbw.sbw_head_logits(x, xs, w, ws, logits, ctx_tokens=ctx, **mark)
    u, t = torch.rand(B, device="cuda"), torch.ones(B, device="cuda")
    out = torch.empty(B, dtype=torch.int32, device="cuda")
    sbw.sbw_sample_given(logits, u, out, temperature=t)
    n = 130
    last = sbw.sbw_head_logits(x[-n:], xs[-n:], w, ws, torch.empty(n, big_v, dtype=torch.bfloat16, device="cuda"),
                               ctx_tokens=ctx[-n:].contiguous(), **mark)
    assert torch.equal(last, logits[-n:])
    alone = torch.empty(n, dtype=torch.int32, device="cuda")
    sbw.sbw_sample_given(last, u[-n:], alone, temperature=t[-n:])
    assert torch.equal(alone, out[-n:])
    codes, s = torch.empty(B, big_v, dtype=E4M3, device="cuda"), torch.empty(B, 1002, device="cuda")
    sbw.sbw_quantize_fp8(logits, codes, s)
    codes2, s2 = torch.empty(n, big_v, dtype=E4M3, device="cuda"), torch.empty(n, 1002, device="cuda")
    sbw.sbw_quantize_fp8(last, codes2, s2)
    assert torch.equal(codes[-n:].view(torch.uint8), codes2.view(torch.uint8)) and torch.equal(s[-n:], s2)
