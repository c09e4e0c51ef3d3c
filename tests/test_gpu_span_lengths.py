"""Own lengths that decode behind a shared prefix has to skip, up to the largest number, on
the kernel that divides the SMs by them: they are recorded, their rows are not written, and
everyone else's are right."""
import pytest

from paper_2505_23970_gb300 import binding as gcb

from .test_gpu_span_routes import wide_shared

pytestmark = pytest.mark.gpu

LARGEST = 2 ** 31 - 1


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bad", [
    {0: LARGEST}, {3: LARGEST - 1023}, {5: LARGEST - 1024}, {2: 1 << 30},
    {0: LARGEST, 1: LARGEST, 4: LARGEST}, {0: 3 * 16 + 1, 2: LARGEST, 5: -1},
    {i: LARGEST for i in range(6)}, {0: -LARGEST - 1, 1: LARGEST // 2 + 1},
])
def test_own_lengths_out_of_range(d, bad):
    c = wide_shared(4, 1, d, 16, [2, 3, 1], [40, 100, 7], [5, 6, 7, 33, 1, 20], seed=1)
    for b, n in bad.items():
        c.dev[2][b] = n
    c.run()
    assert c.pool.check() == gcb.GC_ERR_OUT_OF_RANGE
    c.check(skipped=tuple(bad))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("sizes,S", [([60, 40], [700, 300]), ([20] * 5, [0, 65, 900, 1, 130])])
def test_many_requests_with_a_few_out_of_range(d, sizes, S):
    c = wide_shared(16, 4, d, 16, sizes, S, [1 + 11 * i % 400 for i in range(100)], seed=d,
                    reuse=64)
    bad = (0, 17, 31, 32, 63, 64, 99)
    for b in bad:
        c.dev[2][b] = LARGEST
    for _ in range(2):
        c.out.fill_(float("nan"))
        c.run()
        assert c.pool.check() == gcb.GC_ERR_OUT_OF_RANGE
        c.check(skipped=bad)
