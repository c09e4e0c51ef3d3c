"""Cross attention and shared-prefix decode on tiles as a program uses them: recorded in a
graph, on a stream of its own, between other calls on the pool, and through SharedContext.
(The tests of the operators themselves do these with small calls, which go row by row.)"""
import numpy as np
import pytest

from paper_2505_23970_gb300 import binding as gcb
from paper_2505_23970_gb300.harness import bf16_bits

from . import test_gpu_shared_context
from .test_gpu_span_counter import run_on, whole_items
from .test_gpu_span_routes import ROOM, wide_cross, wide_shared

pytestmark = pytest.mark.gpu

MAKE = {
    "cross-shares": lambda d: wide_cross(8, 1, d, 16, [20000, 77], [9, 30], seed=6, reuse=64),
    "cross-whole": whole_items,
    "shared": lambda d: wide_shared(8, 2, d, 16, [3, 2, 60], [900, 33, 5000],
                                    [1 + 9 * i % 500 for i in range(65)], seed=7, reuse=64),
    "shared-16-heads": lambda d: wide_shared(32, 2, d, 16, [40, 7], [2048, 300],
                                             [1 + 5 * i % 90 for i in range(47)], seed=8,
                                             reuse=64),
}


@pytest.fixture(params=[f"{k}-d{d}" for k in MAKE for d in (64, 128)])
def call(request):
    name, d = request.param.rsplit("-d", 1)
    return MAKE[name](int(d))


def test_recorded_in_a_graph(call):
    import torch
    call.run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        for _ in range(2):
            call.run(stream=torch.cuda.current_stream(), workspace=call.ws)
    for _ in range(2):
        call.out.fill_(float("nan"))
        g.replay()
        assert call.pool.check() == gcb.GC_OK
        call.check()


def test_same_bits_on_another_stream(call):
    import torch
    call.run()
    first = bf16_bits(call.out)
    s = torch.cuda.Stream()
    for _ in range(2):
        call.out.fill_(float("nan"))
        s.wait_stream(torch.cuda.current_stream())
        call.run(stream=s)
        assert call.pool.check(s) == gcb.GC_OK
        assert np.array_equal(bf16_bits(call.out), first)
        torch.cuda.current_stream().wait_stream(s)
    call.check()


@pytest.mark.parametrize("d", [64, 128])
def test_between_prefill_and_decode(d):
    """Each call leaves the pool's counters as the others want them."""
    import torch
    x, c = MAKE["cross-whole"](d), wide_shared(32, 8, d, 16, [30, 34], [900, 5000],
                                               [200 + 9 * i % 500 for i in range(64)], seed=7,
                                               reuse=64)
    pool, n = x.pool, 80
    need = gcb.gc_paged_decode_workspace_bytes(pool.handle, c.B, c.table.shape[1], 32)
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    new = torch.full((12,), n, dtype=torch.int32, device="cuda")
    cu = torch.arange(13, dtype=torch.int32, device="cuda") * n

    def others():
        run_on(pool, c)  # (c's pages are the pool's now)
        decoded = torch.full_like(c.out, float("nan"))
        gcb.gc_paged_decode_attn(c.q, pool.handle, c.table, c.dev[2], decoded, None, 0, c.B,
                                 c.table.shape[1], 32, c.scale, ws, need)
        prefilled = torch.full_like(x.out[:12 * n], float("nan"))
        gcb.gc_prefix_prefill_attn(x.q, pool.handle, c.table, c.dev[2] - n, new, prefilled, None,
                                   0, cu, 12, c.table.shape[1], 32, c.scale, 12 * n)
        assert pool.check() == gcb.GC_OK
        assert torch.isfinite(decoded).all() and torch.isfinite(prefilled).all()
        return bf16_bits(decoded), bf16_bits(prefilled)

    run_on(pool, x)
    before = others()
    for _ in range(2):
        run_on(pool, x)
        for got, want in zip(others(), before):
            assert np.array_equal(got, want)


@pytest.mark.parametrize("Hq,Hkv,d,ps,S,sizes,states", [
    (16, 2, 128, 16, [3000, 40], [40, 24], [1500] + [i % 90 for i in range(63)]),
    (16, 4, 64, 32, [4000, 0, 65], [30, 3, 3], [3000] + [i % 200 for i in range(35)]),
    (32, 2, 128, 64, [5000], [40], [2000] + [0, 7] * 19 + [64]),
])
def test_tokens_through_the_layers(Hq, Hkv, d, ps, S, sizes, states):
    B, most = sum(sizes), max(S) + 3
    assert B * most * Hkv > (262144 if d == 128 else 458752) and ROOM >= 458752
    assert B * max(states) * Hkv > (131072 if d == 128 else 163840)
    test_gpu_shared_context.test_tokens_through_the_layers(Hq, Hkv, d, ps, S, sizes, states)
