"""The ways out of the projection's kernel where a wait inside a CTA does not end, in the bounds-flag build: nothing is in flight
when the CTA leaves, the logits that were not made are NaN, the others have their bits, and the next call works."""
import ctypes

import pytest
import torch

import paper_2609_03844_b200 as sbw
from paper_2609_03844_b200 import inputs
from gpu_util import KEY, require_gpu
from test_gpu_head import blocks, codes, scales
from test_gpu_logprob_owed import _flags, dbg  # noqa: F401

pytestmark = pytest.mark.gpu

TILE = 128                                                # columns of a tile for up to 128 rows


class Case:
    """A call with `tiles` tiles per CTA and its logits from the release build."""

    def __init__(self, dbg, B, K, tiles, delta):  # noqa: F811
        self.dbg, self.B, self.K, self.delta = dbg, B, K, delta
        self.ctas = torch.cuda.get_device_properties(0).multi_processor_count
        self.V = self.ctas * tiles * TILE
        self.x, self.w, self.xs, self.ws = codes(B, K, 1), codes(self.V, K, 2), scales(B, K, 3), scales(blocks(self.V), K, 4)
        self.ctx = inputs.uniform_tokens((B, 1), self.V, seed=5).cuda()
        mark = dict(ctx_tokens=self.ctx, key=KEY, gamma=0.25, delta=delta) if delta else {}
        self.want = sbw.sbw_head_logits(self.x, self.xs, self.w, self.ws, torch.empty(B, self.V, device="cuda"), **mark)
        dbg.sbw_head_logits.argtypes = sbw.lib().sbw_head_logits.argtypes
        _flags(dbg)

    def run(self):
        """The logits of the bounds-flag build; no check of an access or of a copy failed."""
        out = torch.full((self.B, self.V), 7.0, device="cuda")
        rc = self.dbg.sbw_head_logits(self.x.data_ptr(), self.x.stride(0), self.xs.data_ptr(), self.xs.stride(0), self.w.data_ptr(),
                                      self.w.stride(0), self.ws.data_ptr(), self.ws.stride(0), self.B, self.V, self.K,
                                      out.data_ptr(), 0, self.V, 0, self.ctx.data_ptr(), 1, KEY, 0.25, self.delta, 0, None)
        assert rc == 0
        torch.cuda.synchronize()
        mask, failures, passed, _ = _flags(self.dbg)
        assert mask == 0 and failures == 0 and passed > 0
        return out

    def check(self, done):
        """The first `done` tiles of each CTA are whole, the others NaN; the call after that is whole."""
        out, cut = self.run(), self.ctas * done * TILE
        assert torch.equal(out[:, :cut], self.want[:, :cut]) and bool(out[:, cut:].isnan().all())


@pytest.mark.parametrize("delta", [0.0, 2.0])
@pytest.mark.parametrize("B,K,tiles,stop", [(1, 128, 1, 0), (3, 512, 1, 0), (40, 512, 1, 3), (128, 256, 3, 2), (5, 384, 3, 4),
                                            (2, 2048, 2, 17), (1, 1024, 3, 23)])
def test_copies_land_where_the_products_stop(dbg, B, K, tiles, stop, delta):  # noqa: F811
    """With few blocks, or near the end, every copy was issued before the products stop: nobody but the issuer waits for them."""
    require_gpu()
    case = Case(dbg, B, K, tiles, delta)
    dbg.sbw_debug_head_stop.argtypes = [ctypes.c_int64]
    assert dbg.sbw_debug_head_stop(stop) == 0
    try:
        case.check(stop // blocks(K))
    finally:
        dbg.sbw_debug_head_stop(-1)
    assert torch.equal(case.run(), case.want)


LIMIT = 100_000_000                                       # ns


def gave_up(dbg):  # noqa: F811
    out = ctypes.c_uint64()
    assert dbg.sbw_head_gave_up(ctypes.byref(out), None) == 0
    return out.value


@pytest.mark.parametrize("delta", [0.0, 2.0])
@pytest.mark.parametrize("B,K,tiles,withheld", [(1, 128, 1, 0), (40, 512, 2, 5), (128, 256, 3, 2), (2, 1024, 2, 8)])
def test_a_wait_that_runs_out_is_told(dbg, B, K, tiles, withheld, delta):  # noqa: F811
    """A copy that never comes: the wait for it ends at its limit, every CTA is counted once, the context stays usable."""
    require_gpu()
    case = Case(dbg, B, K, tiles, delta)
    dbg.sbw_debug_head_waits.argtypes = [ctypes.c_uint64, ctypes.c_int64]
    dbg.sbw_head_gave_up.argtypes = sbw.lib().sbw_head_gave_up.argtypes
    before = gave_up(dbg)
    assert dbg.sbw_debug_head_waits(LIMIT, withheld) == 0
    try:
        case.check(withheld // blocks(K))
    finally:
        dbg.sbw_debug_head_waits(2_000_000_000, -1)
    assert gave_up(dbg) == before + case.ctas
    assert torch.equal(case.run(), case.want) and gave_up(dbg) == before + case.ctas


def test_nothing_gave_up_in_the_release_build():
    require_gpu()
    x, w, xs, ws = codes(130, 300, 1), codes(700, 300, 2), scales(130, 300, 3), scales(blocks(700), 300, 4)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    sbw.sbw_head_logits(x, xs, w, ws, torch.empty(130, 700, device="cuda"), stream=s)
    assert sbw.sbw_head_gave_up(stream=s) == 0 and sbw.sbw_head_gave_up(0) == 0
    graph = torch.cuda.CUDAGraph()
    y = torch.zeros(1, device="cuda")
    with torch.cuda.graph(graph):
        y += 1
        with pytest.raises(sbw.SbwError, match="UNSUPPORTED"):
            sbw.sbw_head_gave_up()
    graph.replay()
    torch.cuda.synchronize()
    assert float(y) == 1.0
