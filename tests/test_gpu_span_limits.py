"""Cross attention and shared-prefix decode at the largest batch (8192 requests or groups),
on both routes: the batch's tables lie in shared memory beside everything else."""
import pytest

from paper_2505_23970_gb300 import binding as gcb

from . import test_gpu_cross_attn as cross
from . import test_gpu_shared_decode as shared
from ._span import assert_within, attend
from .test_gpu_span_routes import wide_cross, wide_shared

pytestmark = pytest.mark.gpu

MOST = 8192


def check_some(c, step=97):
    import torch
    if isinstance(c, cross.Call):
        rows = [(int(c.cu[b]), c.pages.keys(0, b, c.kv[b])) for b in range(0, len(c.n), step)
                if c.n[b]]
    else:
        rows = [(b, torch.cat([c.pages.keys(0, int(c.group[b]), c.S[c.group[b]]),
                               c.pages.keys(1, b, c.own[b])], 1)) for b in range(0, c.B, step)]
    assert torch.isfinite(c.out).all()
    for row, kv in rows:
        want, bound = attend(c.q[row:row + 1].double(), kv, c.scale)
        assert_within(c.out[row:row + 1], want, bound, f"row {row}")


@pytest.mark.parametrize("G", [1, 8, 16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("make", [shared.Call, wide_shared])
@pytest.mark.parametrize("sizes", [[5000, 3192], [1] * MOST])
def test_requests_and_groups(make, sizes, d, G):
    own = [i % 15 for i in range(MOST)]
    own[4711] = 16 if make is shared.Call else 700
    S = [1 + i % 16 for i in range(len(sizes))]
    c = make(G, 1, d, 16, sizes, S, own, seed=G, reuse=64)
    rows_at_once = MOST * (c.stable.shape[1] + c.table.shape[1]) * 16 <= 262144
    assert rows_at_once == (make is shared.Call)
    for _ in range(2):
        c.out.fill_(float("nan"))
        c.run()
        assert c.pool.check() == gcb.GC_OK
        check_some(c)


@pytest.mark.parametrize("G", [1, 8, 16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("make,kv", [(cross.Call, 16), (wide_cross, 16), (wide_cross, 300)])
def test_requests_of_cross_attention(make, kv, d, G):
    c = make(G, 1, d, 16, [i * 7 % (kv + 1) for i in range(MOST)], [1] * MOST, seed=G, reuse=64)
    for _ in range(2):
        c.out.fill_(float("nan"))
        c.run()
        assert c.pool.check() == gcb.GC_OK
        check_some(c)
