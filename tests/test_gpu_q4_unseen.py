"""Decode over 4-bit pages: what a page holds where a row does not see it is not used,
whatever it is.  The layout is public, so a page may hold scales that no call here writes."""
import numpy as np
import pytest

from paper_2505_23970_gb300 import binding as gcb

from . import _q4
from .test_gpu_q4_decode import Decode

pytestmark = pytest.mark.gpu

NAN, INF = 0x7FC0, 0x7F80


def set_scales(ctx, b, t, bits, planes=(0, 1)):
    """Every scale of token t of request b, K's and V's, in its 4-bit page."""
    ps, d = ctx.ps, ctx.d
    s = ctx.host[..., ps * d // 2:].reshape(ctx.L, 2, ctx.pages4, ctx.Hkv, ps, d // 16)
    for p in planes:
        s[ctx.layer, p, ctx.table4[b, t // ps], :, t % ps] = np.full(
            d // 32, bits, np.uint16).view(np.uint8)


@pytest.mark.parametrize("bits", [NAN, INF, INF | 0x8000])
@pytest.mark.parametrize("Hq,Hkv,d,ps,tokens,lens", [
    (4, 1, 64, 16, 4, [4, 5, 16, 17, 18, 19, 20, 31, 32, 33, 600]),
    (32, 8, 128, 16, 4, [4, 16, 17, 33, 500, 9000]),
    (16, 2, 128, 32, 2, [2, 16, 17, 32, 33]),
    (8, 8, 128, 16, 7, [7, 20, 23, 500]),
    (8, 8, 64, 16, 16, [16, 17, 32, 47, 48]),
])
def test_drafted_tokens_with_scales_that_are_not_finite(Hq, Hkv, d, ps, tokens, lens, bits):
    """The newest token's scales are NaN or infinite: its own row is the only one with it."""
    import torch
    ctx = _q4.Context(lens, Hkv, d, ps, seed=tokens + d)
    for b, T in enumerate(lens):
        set_scales(ctx, b, T - 1, bits)
    ctx.cache.copy_(torch.from_numpy(ctx.host))
    c = Decode(ctx, Hq, tokens).run()
    assert ctx.pool.check() == gcb.GC_OK
    got = c.out.double().cpu().numpy()
    for b, T in enumerate(lens):
        kv, s = ctx.keys(b)
        kv[:, -1], s[:, -1] = 0, 0
        want, bound = _q4.decode_reference(_q4.f32(c.q_bits[b]).astype(np.float64), kv, s, c.scale,
                                           tokens)
        if bits == NAN:  # (an infinite scale may be that of a score of -infinity)
            assert np.isnan(got[b, -1]).all(), T
        assert (np.abs(got[b, :-1] - want[:-1]) <= bound[:-1]).all(), T


@pytest.mark.parametrize("d,tokens", [(64, 3), (128, 2)])
def test_each_draft_is_seen_from_its_own_row_on(d, tokens):
    """V's scales of one drafted token are NaN, K's as they were: NaN from its row on."""
    import torch
    lens = [tokens, 16, 17, 30, 32, 300]
    for i in range(1, tokens):
        ctx = _q4.Context(lens, 2, d, 16, seed=i)
        for b, T in enumerate(lens):
            set_scales(ctx, b, T - tokens + i, NAN, planes=(1,))
        ctx.cache.copy_(torch.from_numpy(ctx.host))
        c = Decode(ctx, 8, tokens).run()
        assert ctx.pool.check() == gcb.GC_OK
        got = c.out.double().cpu().numpy()
        for b, T in enumerate(lens):
            kv, s = ctx.keys(b)
            kv[1, T - tokens + i], s[1, T - tokens + i] = 0, 0
            want, bound = _q4.decode_reference(_q4.f32(c.q_bits[b]).astype(np.float64), kv, s,
                                               c.scale, tokens)
            assert np.isnan(got[b, i:]).all(), (T, i)
            assert (np.abs(got[b, :i] - want[:i]) <= bound[:i]).all(), (T, i)
