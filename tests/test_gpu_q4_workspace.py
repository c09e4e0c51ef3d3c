"""Attention over 4-bit pages writes its rows, its workspace and nothing else."""
import numpy as np
import pytest

from paper_2505_23970_gb300 import binding as gcb

from . import _q4
from .test_gpu_q4_decode import Decode
from .test_gpu_q4_prefill import Prefill

pytestmark = pytest.mark.gpu

GUARD = 4096


def guarded(nbytes):
    """(the whole of a buffer, its middle): bytes of 0xA5 on either side."""
    import torch
    whole = torch.full((nbytes + 2 * GUARD,), 0xA5, dtype=torch.uint8, device="cuda")
    return whole, whole[GUARD:GUARD + nbytes]


def untouched(whole):
    side = np.full(GUARD, 0xA5, np.uint8)
    host = whole.cpu().numpy()
    return (host[:GUARD] == side).all() and (host[-GUARD:] == side).all()


def rows(like):
    import torch
    whole, mid = guarded(like.numel() * 2)
    mid.copy_(torch.full_like(like, float("nan")).view(torch.uint8).flatten())
    return whole, mid.view(torch.bfloat16).view(like.shape)


@pytest.mark.parametrize("Hq,Hkv,d,tokens,lens", [
    (4, 1, 64, 1, [321]),
    (16, 1, 64, 1, [100] * 40),
    (64, 8, 128, 1, [12 + 5 * i for i in range(60)]),
    (32, 8, 128, 4, [3000, 17, 4, 1234]),
    (8, 1, 128, 1, [40 + i % 50 for i in range(1025)]),
    (16, 1, 128, 1, [16 + i % 30 for i in range(1100)]),
])
def test_decode(Hq, Hkv, d, tokens, lens):
    c = Decode(_q4.Context(lens, Hkv, d, 16, seed=17), Hq, tokens)
    ws_whole, c.ws = guarded(c.need)
    out_whole, c.out = rows(c.out)
    cache = c.ctx.cache.clone()
    c.run().check()
    assert c.ctx.pool.check() == gcb.GC_OK
    assert untouched(ws_whole) and untouched(out_whole)
    assert bool((c.ctx.cache == cache).all())


@pytest.mark.parametrize("Hq,Hkv,d,P,n,recent", [
    (8, 2, 64, [300, 0, 5, 40], [64, 33, 1, 0], 0),
    (64, 8, 128, [1000, 17, 0], [300, 1, 129], 1),
])
def test_prefill(Hq, Hkv, d, P, n, recent):
    c = Prefill(P, n, Hq, Hkv, d, 16, recent=recent, seed=18)
    want = c.both_calls()
    ws_whole, c.ws = guarded(c.need)
    out_whole, c.out = rows(c.out)
    cache, pool = c.ctx.cache.clone(), c.ctx.pool.planes().clone()
    c.run()
    assert c.ctx.pool.check() == gcb.GC_OK
    assert untouched(ws_whole) and untouched(out_whole)
    assert np.array_equal(c.out.view(_int16()).cpu().numpy(), want.view(_int16()).cpu().numpy())
    assert bool((c.ctx.cache == cache).all())
    assert bool((c.ctx.pool.planes().view(_int16()) == pool.view(_int16())).all())


def _int16():
    import torch
    return torch.int16
