"""Calls write within the workspace that they ask for, the output's rows and nothing else:
every head dimension and number of q heads per kv head, on both routes of cross attention and
shared prefixes, and decode."""
import pytest

from paper_2505_23970_gb300 import binding as gcb

from . import test_gpu_cross_attn as cross
from . import test_gpu_shared_decode as shared
from .test_gpu_span_routes import wide_cross, wide_shared

pytestmark = pytest.mark.gpu

GUARD = 1 << 20


def guarded(need):
    import torch
    b = torch.full((need + 2 * GUARD,), 0xA5, dtype=torch.uint8, device="cuda")
    b[GUARD:GUARD + need] = 0xFF
    return b


def check_guards(b, need):
    assert (b[:GUARD] == 0xA5).all() and (b[GUARD + need:] == 0xA5).all()


def run_guarded(c, need):
    import torch
    b, planes = guarded(need), c.pool.planes().view(torch.int16).clone()
    out = torch.full((c.out.shape[0] + 2, *c.out.shape[1:]), 7.0, dtype=torch.bfloat16,
                     device="cuda")
    out[1:-1] = float("nan")
    c.run(workspace=b[GUARD:], workspace_bytes=need, out=out[1:-1])
    assert c.pool.check() == gcb.GC_OK
    check_guards(b, need)
    assert (out[0] == 7).all() and (out[-1] == 7).all()
    assert torch.equal(c.pool.planes().view(torch.int16), planes)
    c.out = out[1:-1]
    c.check()


@pytest.mark.parametrize("G", [1, 2, 4, 8, 16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("make", [cross.Call, wide_cross])
@pytest.mark.parametrize("kv,n", [([300, 0, 1700], [4, 3, 12]), ([20000], [3]), ([90] * 7, [5] * 7)])
def test_cross(make, d, G, kv, n):
    c = make(2 * G, 2, d, 16, kv, n, seed=G, reuse=64)
    run_guarded(c, gcb.gc_paged_cross_workspace_bytes(c.pool.handle, len(n), c.table.shape[1],
                                                      c.Hq, c.T))


@pytest.mark.parametrize("G", [1, 2, 4, 8, 16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("make", [shared.Call, wide_shared])
@pytest.mark.parametrize("sizes,S,own", [
    ([4, 1], [900, 257], [1, 70, 300, 2, 1999]), ([3], [8], [2700, 2000, 1]),
    ([60, 40], [300, 65], [1 + 17 * i % 300 for i in range(100)]),
])
def test_shared(make, d, G, sizes, S, own):
    c = make(2 * G, 2, d, 16, sizes, S, own, seed=G, reuse=64)
    run_guarded(c, gcb.gc_shared_prefix_decode_workspace_bytes(
        c.pool.handle, c.B, len(S), c.stable.shape[1], c.table.shape[1], c.Hq))


@pytest.mark.parametrize("G", [1, 2, 4, 8, 16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("own", [[2700, 2000, 1], [1 + 17 * i % 900 for i in range(100)]])
def test_decode(d, G, own):
    import torch
    c = shared.Call(2 * G, 2, d, 16, [len(own)], [0], own, seed=G, reuse=64)
    need = gcb.gc_paged_decode_workspace_bytes(c.pool.handle, c.B, c.table.shape[1], c.Hq)
    b = guarded(need)
    gcb.gc_paged_decode_attn(c.q, c.pool.handle, c.table, c.dev[2], c.out, None, 0, c.B,
                             c.table.shape[1], c.Hq, c.scale, b[GUARD:], need)
    assert c.pool.check() == gcb.GC_OK
    check_guards(b, need)
    c.check()
