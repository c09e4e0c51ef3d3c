"""Decode over a 4-bit cache's 16-bit pages with the smallest keys and values that the
header gives room for."""
import numpy as np
import pytest

from paper_2505_23970_gb300 import binding as gcb
from paper_2505_23970_gb300 import workloads as wl
from paper_2505_23970_gb300.harness import bf16_tensor

from . import _q4
from .test_gpu_q4_decode import Decode

pytestmark = pytest.mark.gpu


def times(bits, exp):
    return wl.f32_to_bf16_bits((_q4.f32(bits).astype(np.float64) * 2.0 ** exp).astype(np.float32))


@pytest.mark.parametrize("q_exp,k_exp,v_exp", [(30, -40, 0), (55, -66, 0), (0, 0, -60),
                                               (60, -66, -70)])
@pytest.mark.parametrize("d", [64, 128])
def test_small_keys_and_values(q_exp, k_exp, v_exp, d):
    """A key's element is off by 2^-74 at most, so a score by 2^-74 of the sum of |q|, and P,
    relative to the sum of all, by twice that (and its square); the rest as ever."""
    ctx = _q4.Context([90, 17], 1, d, 16, recent=100, seed=21)
    ctx.bits16[0, 0], ctx.bits16[0, 1] = times(ctx.bits16[0, 0], k_exp), times(ctx.bits16[0, 1], v_exp)
    ctx.pool.planes().copy_(bf16_tensor(ctx.bits16))
    bits = times(wl.normal_bf16(21, 71, (2, 1, 4, d)), q_exp)
    scale = float(np.float32(2.0 ** (-q_exp - k_exp) * d ** -0.5))
    c = Decode(ctx, 4, q_bits=bits, scale=scale).run()
    assert ctx.pool.check() == gcb.GC_OK
    got = c.out.double().cpu().numpy()
    for b in range(2):
        q = _q4.f32(bits[b]).astype(np.float64)
        kv, s = ctx.keys(b)
        want, bound = _q4.decode_reference(q, kv, s, scale, 1)
        e = np.abs(q).sum(-1)[..., None] * 2.0 ** -74 * scale
        A = np.abs(kv[1]).max()
        bound = bound + A * (2 * e + 4 * e * e)
        assert (np.abs(got[b] - want) <= bound).all(), (b, np.abs(got[b] - want).max(), bound.max())
