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
