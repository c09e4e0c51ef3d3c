"""Pages whose bytes lie past 32 bits of the pool: the rotated append, cross attention and
decode behind shared prefixes give the bits that they give in a small pool."""
import numpy as np
import pytest

from paper_2505_23970_gb300 import binding as gcb
from paper_2505_23970_gb300.harness import _i32, bf16_bits

from . import test_gpu_append_rope as rope
from . import test_gpu_cross_attn as cross
from . import test_gpu_shared_decode as shared
from .test_gpu_span_routes import wide_cross, wide_shared

pytestmark = pytest.mark.gpu


class Far:
    """A pool of two layers, 5 GiB a plane, in which page i of a small one is page
    num_pages - 1 - i of the second layer."""

    def __init__(self, Hkv, d, ps):
        self.num_pages = 5 * 2 ** 30 // (Hkv * ps * d * 2)
        self.pool = gcb.KVPool.create(2, Hkv, d, ps, self.num_pages)

    def take(self, planes):
        self.pool.planes()[1, :, self.num_pages - planes.shape[1]:] = planes.flip(1)

    def pages(self, table):
        import torch
        return torch.where(table < 0, table, self.num_pages - 1 - table).int().contiguous()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("make", [cross.Call, wide_cross])
def test_cross(make, d):
    c = make(16, 2, d, 16, [300, 0, 1700, 129], [40, 3, 33, 1], seed=d)
    c.run()
    assert c.pool.check() == gcb.GC_OK
    c.check()
    first = bf16_bits(c.out)
    far = Far(2, d, 16)
    far.take(c.pages.pool.planes()[0])
    c.out.fill_(float("nan"))
    c.run(pool=far.pool.handle, block_table=far.pages(c.table), layer=1)
    assert far.pool.check() == gcb.GC_OK
    assert np.array_equal(bf16_bits(c.out), first)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("make", [shared.Call, wide_shared])
def test_shared(make, d):
    c = make(16, 2, d, 16, [4, 1, 3], [900, 0, 257], [1, 70, 300, 2, 40, 999, 16, 3], seed=d)
    c.run()
    assert c.pool.check() == gcb.GC_OK
    c.check()
    first = bf16_bits(c.out)
    far = Far(2, d, 16)
    far.take(c.pages.pool.planes()[0])
    c.out.fill_(float("nan"))
    c.run(pool=far.pool.handle, shared_table=far.pages(c.stable), block_table=far.pages(c.table),
          layer=1)
    assert far.pool.check() == gcb.GC_OK
    assert np.array_equal(bf16_bits(c.out), first)


@pytest.mark.parametrize("n", [[1, 2, 1], [900, 3, 2000]])
def test_append(n):
    c = rope.Call([100, 0, 33], n, 8, 2, 128, 16, 128, seed=len(n) + n[0])
    c.run()
    c.check()
    first = bf16_bits(c.out)
    far = Far(2, 128, 16)
    far.take(c.pool.planes()[0] * 0)
    c.out.fill_(float("nan"))
    c.run(pool=far.pool.handle, block_table=far.pages(_i32(c.w.block_table, "cuda")), layer=1)
    assert far.pool.check() == gcb.GC_OK
    assert np.array_equal(bf16_bits(c.out), first)
    small = bf16_bits(c.pool.planes())[0]
    big = bf16_bits(far.pool.planes()[1, :, far.num_pages - small.shape[1]:].flip(1))
    written = small != 0x7FC1
    assert written.any() and np.array_equal(big[written], small[written])
