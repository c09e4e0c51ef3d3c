"""Cross attention and shared-prefix decode on tiles: the same cases as their own tests,
with block tables wide enough (unused columns) that a call is not small by their room, so
that the tensor-core kernels, the division of the SMs, shares, aligned runs and joins take them;
and calls that reach each of those."""
import numpy as np
import pytest

from paper_2505_23970_gb300 import binding as gcb
from paper_2505_23970_gb300.harness import bf16_bits

from . import test_gpu_cross_attn as cross
from . import test_gpu_shared_decode as shared

pytestmark = pytest.mark.gpu

ROOM = 600000  # rows x keys x kv heads, above every bound of the row-by-row route


def widen(table, rows, ps, Hkv):
    import torch
    need = -(-ROOM // (rows * ps * Hkv)) + 1
    extra = max(0, need - table.shape[1])
    return torch.cat([table, torch.full((table.shape[0], extra), -1, dtype=torch.int32,
                                        device="cuda")], 1).contiguous()


def wide_cross(*args, **kw):
    c = cross.Call(*args, **kw)
    c.table = widen(c.table, c.T, c.pages.ps, c.pages.Hkv)
    return c


def wide_shared(*args, **kw):
    c = shared.Call(*args, **kw)
    c.stable = widen(c.stable, c.B, c.pages.ps, c.pages.Hkv)
    return c


@pytest.mark.parametrize("name", list(cross.CASES))
def test_cross_on_tiles(name):
    c = wide_cross(*cross.CASES[name], seed=len(name))
    c.run()
    assert c.pool.check() == gcb.GC_OK
    c.check()


@pytest.mark.parametrize("name", list(shared.CASES))
def test_shared_on_tiles(name):
    c = wide_shared(*shared.CASES[name], seed=len(name))
    c.run()
    assert c.pool.check() == gcb.GC_OK
    c.check()


@pytest.mark.parametrize("Hq,Hkv,d,ps,kv,n", [
    (8, 1, 128, 16, [150000], [5]),                  # one item over many pairs
    (16, 2, 128, 64, [70000, 69000], [40, 35]),      # two tiles of long keys: aligned runs
    (16, 2, 64, 64, [70000, 69000], [40, 35]),
    (64, 8, 128, 16, [18000, 200, 3000], [90, 500, 10]),  # tiles that not all have
    (32, 8, 128, 16, [2000] * 12, [130] * 12),       # whole items, several rounds
    (32, 8, 64, 16, [2000] * 24, [130] * 24),
    (2, 1, 64, 32, [1, 128, 129, 60000], [1, 1, 1, 1]),
])
def test_cross_shares_and_runs(Hq, Hkv, d, ps, kv, n):
    c = wide_cross(Hq, Hkv, d, ps, kv, n, seed=Hq + d, reuse=64)
    for _ in range(2):  # the second call finds the counters as the first left them
        c.out.fill_(float("nan"))
        c.run()
        assert c.pool.check() == gcb.GC_OK
        c.check()


@pytest.mark.parametrize("Hq,Hkv,d,ps,sizes,S,own", [
    (8, 1, 128, 16, [3], [150000], [300, 1, 0]),
    (16, 2, 128, 64, [40], [70000], [1 + 3 * i for i in range(40)]),      # two tiles: aligned runs
    (16, 2, 64, 64, [40], [70000], [1 + 3 * i for i in range(40)]),
    (16, 2, 128, 64, [40, 3], [70000, 66000], [1 + 3 * i for i in range(43)]),  # and one
    (16, 2, 64, 64, [40, 3], [70000, 66000], [1 + 3 * i for i in range(43)]),
    (4, 1, 128, 16, [2, 1], [0, 0], [9000, 5, 12000]),                    # own keys alone
    (4, 1, 64, 16, [2, 1], [0, 0], [9000, 5, 12000]),
    (4, 1, 128, 16, [2, 1], [30000, 1], [0, 0, 0]),                       # shared alone
    (4, 1, 64, 16, [2, 1], [30000, 1], [0, 0, 0]),
    (32, 8, 128, 16, [100], [100], [1 + i % 100 for i in range(100)]),    # many short ones
    (32, 8, 64, 16, [100], [100], [1 + i % 100 for i in range(100)]),
    (32, 2, 128, 32, [30, 5], [5000, 77], [1 + 31 * i for i in range(35)]),  # 16 heads of 128
    (32, 2, 64, 32, [30, 5], [5000, 77], [1 + 31 * i for i in range(35)]),
    (8, 4, 128, 16, [1] * 530, [300 + i for i in range(530)], [1 + i % 9 for i in range(530)]),
    (8, 4, 64, 16, [1] * 530, [300 + i for i in range(530)], [1 + i % 9 for i in range(530)]),
])
def test_shared_division_of_the_sms(Hq, Hkv, d, ps, sizes, S, own):
    c = wide_shared(Hq, Hkv, d, ps, sizes, S, own, seed=Hq + d, reuse=64)
    for _ in range(2):
        c.out.fill_(float("nan"))
        c.run()
        assert c.pool.check() == gcb.GC_OK
        c.check()


@pytest.mark.parametrize("d", [64, 128])
def test_same_bits_again_on_tiles(d):
    c = wide_shared(8, 1, d, 16, [3, 4], [5000, 77], [9, 30, 700, 1, 2, 3, 4], seed=6, reuse=64)
    x = wide_cross(8, 1, d, 16, [50000, 77], [9, 30], seed=6, reuse=64)
    for call in (c, x):
        call.run()
        first = bf16_bits(call.out)
        call.out.fill_(float("nan"))
        call.run()
        assert np.array_equal(bf16_bits(call.out), first)


@pytest.mark.parametrize("d", [64, 128])
def test_bad_lengths_on_tiles(d):
    c = wide_cross(4, 1, d, 16, [40, 33, 100], [5, 6, 7], seed=1)
    c.dev[0][1] = c.table.shape[1] * 16 + 1
    c.run()
    assert c.pool.check() == gcb.GC_ERR_OUT_OF_RANGE
    c.check(skipped=(1,))
    c = wide_cross(4, 1, d, 16, [40, 33, 100], [5, 6, 7], seed=1)
    c.run(total_new_tokens=c.T - 1)
    assert c.pool.check() == gcb.GC_ERR_OUT_OF_RANGE
    c.check(skipped=(2,))

    def call():
        return wide_shared(4, 1, d, 16, [2, 3, 1], [40, 100, 7], [5, 6, 7, 33, 1, 20], seed=1)
    c = call()
    c.dev[2][3] = 3 * 16 + 1
    c.dev[2][0] = -1
    c.run()
    assert c.pool.check() == gcb.GC_ERR_OUT_OF_RANGE
    c.check(skipped=(0, 3))
    for bad in (c.stable.shape[1] * 16 + 1, -1):
        c = call()
        c.dev[0][1] = bad
        c.run()
        assert c.pool.check() == gcb.GC_ERR_OUT_OF_RANGE
        c.check(skipped=(2, 3, 4))
    for at, value, skipped in ((3, 5, (5,)), (0, 1, (0,)), (3, 7, (5,))):
        c = call()
        c.dev[1][at] = value
        c.run()
        assert c.pool.check() == gcb.GC_ERR_OUT_OF_RANGE
        c.check(skipped=skipped)


@pytest.mark.parametrize("d", [64, 128])
def test_bad_pages_on_tiles(d):
    c = wide_cross(4, 1, d, 16, [40, 33, 100], [5, 6, 7], seed=2)
    c.table[1, 1] = c.pages.num_pages
    c.run()
    assert c.pool.check() == gcb.GC_ERR_OUT_OF_RANGE
    c.out[c.cu[1]:c.cu[2]] = float("nan")
    c.check(skipped=(1,))
    c = wide_shared(4, 1, d, 16, [2, 3, 1], [40, 100, 7], [5, 6, 7, 33, 1, 20], seed=2)
    c.stable[1, 2] = c.pages.num_pages
    c.table[5, 0] = -1
    c.run()
    assert c.pool.check() == gcb.GC_ERR_OUT_OF_RANGE
    c.out[2:] = float("nan")
    c.check(skipped=(2, 3, 4, 5))


@pytest.mark.parametrize("d", [64, 128])
def test_overlapping_groups_stay_in_bounds(d):
    """Groups that do not divide the batch are an error; whatever they hold, nothing but
    the call's own rows is written."""
    import torch
    c = wide_shared(4, 1, d, 16, [2, 3, 1], [40, 100, 7], [5, 6, 7, 33, 1, 20], seed=3)
    rows = torch.full((c.B + 2,) + tuple(c.out.shape[1:]), 7.0, dtype=torch.bfloat16,
                      device="cuda")
    for cu in ([0, 6, 0, 6], [5, 3, 1, 6], [-4, 2, 8, 6], [0, 2, 1 << 30, 6]):
        c.dev[1].copy_(torch.tensor(cu, dtype=torch.int32))
        c.run(out=rows[1:-1])
        assert c.pool.check() == gcb.GC_ERR_OUT_OF_RANGE
        assert (rows[0] == 7).all() and (rows[-1] == 7).all()


@pytest.mark.parametrize("d", [64, 128])
def test_short_workspaces_are_refused_on_tiles(d):
    import torch
    for c in (wide_cross(8, 1, d, 16, [20000], [5], reuse=64),
              wide_shared(8, 1, d, 16, [2], [20000], [700, 3000], reuse=64)):
        c.run()
        assert c.need > 0
        for change in (dict(workspace_bytes=c.need - 1), dict(workspace=None)):
            c.out.fill_(float("nan"))
            with pytest.raises(gcb.GcError) as e:
                c.run(**change)
            assert e.value.status == gcb.GC_ERR_INVALID_ARG
            assert c.pool.check() == gcb.GC_OK
            assert torch.isnan(c.out).all()
