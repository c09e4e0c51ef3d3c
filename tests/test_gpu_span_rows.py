"""Which rows cross attention and shared-prefix decode write, and what they record, is the
same whichever way a call goes (row by row on the decode kernel, or on tiles): a request's
rows are the new_lens[b] from cu_new_lens[b] on, and requests and groups that are not within
the call's rows are recorded."""
import pytest

from paper_2505_23970_gb300 import binding as gcb

from . import test_gpu_cross_attn as cross
from . import test_gpu_shared_decode as shared
from .test_gpu_span_routes import wide_cross, wide_shared

pytestmark = pytest.mark.gpu


def check_first(c, n):
    """Of request b the first n[b] rows are written, and no others."""
    import torch
    for b, m in enumerate(n):
        rows = c.out[c.cu[b]:c.cu[b + 1]]
        assert torch.isnan(rows[m:]).all(), b
    kept, c.n = c.n, n
    for b, m in enumerate(n):
        if m:
            q = c.q[c.cu[b]:c.cu[b] + m].double()
            want, bound = cross.attend(q, c.pages.keys(0, b, c.kv[b]), c.scale)
            cross.assert_within(c.out[c.cu[b]:c.cu[b] + m], want, bound, f"request {b}")
    c.n = kept


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("make", [cross.Call, wide_cross])
@pytest.mark.parametrize("n", [[3, 6, 7], [5, 0, 1], [0, 0, 7], [0, 0, 0], [4, 5, 6]])
def test_rows_past_new_lens_are_not_written(make, n, d):
    c = make(4, 1, d, 16, [40, 0, 100], [5, 6, 7], seed=1)
    for b, m in enumerate(n):
        c.dev[1][b] = m
    c.run()
    assert c.pool.check() == gcb.GC_OK
    check_first(c, n)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("make", [cross.Call, wide_cross])
@pytest.mark.parametrize("b,n", [(0, -1), (1, -(2 ** 31)), (2, -3), (2, 8), (2, 2 ** 31 - 1)])
def test_requests_that_are_skipped_are_recorded(make, b, n, d):
    c = make(4, 1, d, 16, [40, 33, 100], [5, 6, 7], seed=1)
    c.dev[1][b] = n
    c.run()
    assert c.pool.check() == gcb.GC_ERR_OUT_OF_RANGE
    c.check(skipped=(b,))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("make", [cross.Call, wide_cross])
def test_lengths_of_requests_without_rows_are_not_looked_at(make, d):
    c = make(4, 1, d, 16, [40, 33, 100], [5, 0, 7], seed=1)
    c.dev[0][1] = -5
    c.run()
    assert c.pool.check() == gcb.GC_OK
    c.check()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("make", [shared.Call, wide_shared])
@pytest.mark.parametrize("cu", [[0, 6, 0, 6], [5, 3, 1, 6], [-4, 2, 8, 6], [0, 2, 1 << 30, 6],
                                [0, 2, 6, 7], [-1, 2, 5, 6]])
def test_groups_that_do_not_divide_the_batch_are_recorded(make, cu, d):
    import torch
    c = make(4, 1, d, 16, [2, 3, 1], [40, 100, 7], [5, 6, 7, 33, 1, 20], seed=3)
    rows = torch.full((c.B + 2,) + tuple(c.out.shape[1:]), 7.0, dtype=torch.bfloat16,
                      device="cuda")
    c.dev[1].copy_(torch.tensor(cu, dtype=torch.int32))
    c.run(out=rows[1:-1])
    assert c.pool.check() == gcb.GC_ERR_OUT_OF_RANGE
    assert (rows[0] == 7).all() and (rows[-1] == 7).all()
