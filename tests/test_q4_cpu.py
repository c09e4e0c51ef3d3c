"""The 4-bit format's arithmetic, and refusals that need no GPU."""
import numpy as np
import pytest

from paper_2505_23970_gb300 import binding as gcb
from paper_2505_23970_gb300 import build as gbuild
from paper_2505_23970_gb300 import workloads as wl

from . import _q4


@pytest.fixture(scope="module", autouse=True)
def lib():
    gbuild.build()
    return gcb.load()


def test_a_value_is_half_a_step_off_at_most():
    """|x - c s| <= s / 2, and where s was rounded down by up to 2^-8 of itself the
    largest value is at most 7 * 2^-8 steps beyond its code."""
    x = wl.normal_bf16(3, 1, (500, 128))
    s = np.repeat(_q4.f32(_q4.quantise(x)[1]), 32, -1)
    off = np.abs(_q4.f32(x) - _q4.values(x))
    assert np.all(off <= s * (0.5 + 2.0 ** -20))
    assert np.all(np.abs(_q4.quantise(x)[0]).max(-1) == 7)


def test_special_values():
    inf, nan, zero, big, tiny = 0x7F80, 0x7FC0, 0, 0x7F7F, 0x0001
    rows = np.zeros((6, 32), np.uint16)
    rows[0, :3] = [inf, nan, 0xFF80]           # nothing finite but zeros
    rows[1, :4] = [inf, nan, 0xFF80, 0x40E0]   # 7: the scale is 1
    rows[2, :2] = [big, 0xBF80]
    rows[3, :2] = [tiny, 0x8001]
    rows[4, :2] = wl.f32_to_bf16_bits(np.array([7 * 2.0 ** -24, 2.0 ** -24], np.float32))
    rows[5, :3] = wl.f32_to_bf16_bits(np.array([7, 2.5, -3.5], np.float32))
    c, s = _q4.quantise(rows)
    c, s = c[:, 0], _q4.f32(s)[:, 0]
    assert s[0] == 0 and not c[0].any() and s[3] == 0 and not c[3].any()
    assert s[1] == 1 and list(c[1, :4]) == [7, 0, -7, 7]
    assert s[2] == 2.0 ** 15 and list(c[2, :2]) == [7, 0]
    assert s[4] == 2.0 ** -24 and list(c[4, :2]) == [7, 1]
    assert list(c[5, :3]) == [7, 2, -4]  # ties to even


@pytest.mark.parametrize("d", [64, 128])
def test_every_column_has_a_place_of_its_own(d):
    for is_k in (True, False):
        seen = set()
        for col in range(d):
            row = np.zeros((1, d), np.uint16)
            row[0, col] = 0x40E0
            codes = _q4.row_bytes(row, is_k)[0][0]
            nib = np.stack([codes & 15, codes >> 4], -1).reshape(-1)
            at = np.flatnonzero(nib != 8)
            assert at.size == 1 and nib[at[0]] == 15
            g, j = col // 32, col % 32
            word, n = (j // 8, _q4.K_NIBBLE[j % 8]) if is_k else (j // 4, j % 4)
            assert at[0] == (word * (d // 32) + g) * (8 if is_k else 4) + n
            seen.add(int(at[0]))
        assert seen == set(range(d))


def test_bytes():
    cfg = gcb.make_config(3, 8, 128, 16, 1)
    assert gcb.gc_kv_q4_bytes(cfg, 10) == 3 * 2 * 10 * 8 * 16 * (64 + 8)
    assert gcb.gc_kv_q4_bytes(cfg, 0) == 0
    assert gcb.gc_kv_q4_bytes(gcb.make_config(1, 2, 64, 32, 1), 5) == 2 * 5 * 2 * 32 * 36
    assert gcb.gc_kv_q4_bytes(gcb.make_config(1, 2, 96, 32, 1), 5) == 0
    assert gcb.gc_kv_q4_bytes(cfg, -1) == 0
    # past 32 bits
    assert gcb.gc_kv_q4_bytes(gcb.make_config(80, 8, 128, 128, 1), 2 ** 20) == \
        80 * 2 * 2 ** 20 * 8 * 128 * 72


def test_a_null_pool_is_refused():
    x = 16
    calls = [
        lambda: gcb.gc_kv_append_rope_q4(None, x, 64, x, x, 64, x, 64, x, 1, x, x, None, 0, x, 1,
                                         1, 1, 1),
        lambda: gcb.gc_kv_pack_q4(None, x, x, 1, x, 1, 0, 1),
        lambda: gcb.gc_kv_unpack_q4(None, x, 1, x, x, 1, 0, 1),
        lambda: gcb.gc_paged_decode_attn_q4(x, None, x, x, x, None, 0, 1, 1, 1, 1.0, x, 1 << 20, x,
                                            x, 1, 1),
        lambda: gcb.gc_prefix_prefill_attn_q4(x, None, x, x, x, x, None, 0, x, 1, 1, 1, 1.0, 1, x,
                                              x, 1, x, 1 << 20)]
    for call in calls:
        with pytest.raises(gcb.GcError) as e:
            call()
        assert e.value.status == gcb.GC_ERR_INVALID_ARG
    assert gcb.gc_paged_decode_q4_workspace_bytes(None, 1, 1, 8, 1) == 0
    assert gcb.gc_prefix_prefill_q4_workspace_bytes(None, 1, 1, 1) == 0
