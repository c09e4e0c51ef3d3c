"""Work items of cross attention and shared-prefix decode that are claimed from a counter:
every call finds its counter at 0, whatever ran on the pool before it (the same call, calls
that are cut and calls that cannot be, calls with a join and without one).  A call that
starts from a raised counter leaves out items, and their rows hold what the output or the
workspace held before: NaN here."""
import pytest

from paper_2505_23970_gb300 import binding as gcb
from paper_2505_23970_gb300.harness import bf16_tensor

from . import test_gpu_cross_attn as cross
from . import test_gpu_shared_decode as shared
from .test_gpu_span_routes import wide_cross, wide_shared

pytestmark = pytest.mark.gpu


def run_on(pool, call):
    """The call on a pool of at least as many pages, after its own pages' bytes are there."""
    planes = bf16_tensor(call.pages.bits)
    pool.planes()[:, :, :planes.shape[2]] = planes
    call.out.fill_(float("nan"))
    call.run(pool=pool.handle)
    assert pool.check() == gcb.GC_OK
    call.check()


def whole_items(d):
    """Cross attention that can be cut, but is faster in whole items: four rounds of them."""
    return wide_cross(32, 8, d, 16, [2000] * (12 if d == 128 else 24),
                      [130] * (12 if d == 128 else 24), seed=d, reuse=64)


def uncut(d):
    """Cross attention over tables of at most 256 states, so that nothing can be cut, with
    more items than the GPU has SMs."""
    n = 16 if d == 128 else 24
    c = cross.Call(32, 8, d, 16, [100 + 6 * i for i in range(n)], [130] * n, seed=d, reuse=64)
    assert c.table.shape[1] * 16 <= 256
    return c


def many_groups(d):
    """More than 512 groups: nothing is cut, and each side has a kernel of its own."""
    return wide_shared(16, 8, d, 16, [1] * 530, [100 + i for i in range(530)],
                       [1 + i % 9 for i in range(530)], seed=d, reuse=64)


@pytest.mark.parametrize("sizes,S", [
    ([256], [2048]),         # 128 items: whole, in two rounds on 76 SM pairs
    ([16] * 10, [1000] * 10),  # 80 items
    ([7] * 8 + [8], [2048] * 9),  # fewer items than pairs, but as many as 96 by the bound
    ([40, 3], [70000, 66000]),    # cut, tile by tile
])
def test_sixteen_heads_again_and_again(sizes, S):
    B = sum(sizes)
    c = shared.Call(128, 8, 128, 16, sizes, S, [1 + 5 * i % 90 for i in range(B)], seed=B,
                    reuse=64)
    for _ in range(3):  # (the workspace is filled anew for every call)
        c.out.fill_(float("nan"))
        c.run()
        assert c.pool.check() == gcb.GC_OK
        c.check()


@pytest.mark.parametrize("sizes,S", [([256], [2048]), ([7] * 8 + [8], [2048] * 9)])
def test_whole_items_after_sixteen_heads(sizes, S):
    B = sum(sizes)
    first = shared.Call(128, 8, 128, 16, sizes, S, [1 + i % 90 for i in range(B)], seed=1,
                        reuse=64)
    x = whole_items(128)
    for _ in range(2):
        run_on(first.pool, first)
        run_on(first.pool, x)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("before", [uncut, many_groups])
def test_whole_items_after_calls_that_are_not_cut(before, d):
    first, x = before(d), whole_items(d)
    for _ in range(2):
        run_on(first.pool, first)
        run_on(first.pool, x)
    run_on(first.pool, x)


@pytest.mark.parametrize("d", [64, 128])
def test_calls_that_are_not_cut_after_each_other(d):
    first, x = uncut(d), many_groups(d)
    for call in (first, x, x, first, first):
        run_on(first.pool, call)
