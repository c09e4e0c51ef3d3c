"""gc_kv_append_rope against the rotation in 64 bits: both kinds of pairs, every
part of a head rotated, dense and strided inputs, positions that are not the
slots, and everything that is skipped or refused.

A rotated value x c - y s: the product y s and the sum are each rounded once in
binary32, so before its one rounding to bf16 it is within e = 2^-23 (|x| + |y|)
of the exact one (|c|, |s| <= 1); rounding is monotone, so the result lies
between the rounded ends of that interval, and mostly they are one value.
Everything copied is compared bit for bit."""
import numpy as np
import pytest

from paper_2505_23970_gb300 import binding as gcb
from paper_2505_23970_gb300 import workloads as wl
from paper_2505_23970_gb300.harness import _i32, bf16_bits, bf16_tensor

pytestmark = pytest.mark.gpu


def f64(bits):
    return wl.bf16_bits_to_f32(bits).astype(np.float64)


def angle_table(n, rot, seed=0):
    freq = 10000.0 ** (-np.arange(0, rot, 2) / rot)
    a = np.arange(n)[:, None] * freq + seed
    return np.stack([np.cos(a), np.sin(a)], 1).astype(np.float32)


def pairs(rot, interleaved):
    i = np.arange(rot // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)


def check_rotated(got, x, table, pos, rot, interleaved):
    """got, x: bits [T][heads][d]; the rows' positions pos [T]."""
    a, b = pairs(rot, interleaved)
    v, g = f64(x), f64(got)
    c = table[pos, 0][:, None].astype(np.float64)
    s = table[pos, 1][:, None].astype(np.float64)
    for at, want in ((a, v[..., a] * c - v[..., b] * s), (b, v[..., b] * c + v[..., a] * s)):
        # (2^-24 of the value: the ends pass through binary32 on their way to bf16)
        e = 2.0 ** -23 * (np.abs(v[..., a]) + np.abs(v[..., b])) + 2.0 ** -24 * np.abs(want)
        assert np.all(f64(wl.f32_to_bf16_bits(want - e)) <= g[..., at])
        assert np.all(g[..., at] <= f64(wl.f32_to_bf16_bits(want + e)))
    assert np.array_equal(got[..., rot:], x[..., rot:])


class Call:
    """One call's inputs on the device; q, k, v as parts of one projection's rows
    (fused) or dense tensors."""

    def __init__(self, P, n, Hq, Hkv, d, ps, rot, interleaved=False, fused=False, positions=None,
                 seed=0, angles=None):
        import torch
        self.w = w = wl.custom("append-rope", len(P), max(Hq, Hkv), Hkv, d, ps, P, n, seed=seed)
        self.Hq, self.rot, self.interleaved = Hq, rot, interleaved
        T = w.T_new
        self.bits = wl.normal_bf16(seed, 21, (T, Hq + 2 * Hkv, d))
        self.q_bits, self.k_bits = self.bits[:, :Hq], self.bits[:, Hq:Hq + Hkv]
        self.v_bits = self.bits[:, Hq + Hkv:]
        if fused:
            rows = bf16_tensor(self.bits)
            self.q, self.k, self.v = rows[:, :Hq], rows[:, Hq:Hq + Hkv], rows[:, Hq + Hkv:]
        else:
            self.q, self.k, self.v = (bf16_tensor(x) for x in (self.q_bits, self.k_bits,
                                                               self.v_bits))
        self.slots = np.concatenate([np.arange(p, p + m) for p, m in zip(P, n)]).astype(np.int64)
        self.pos = self.slots if positions is None else np.asarray(positions, np.int64)
        self.positions = None if positions is None else _i32(self.pos, "cuda")
        size = int(self.pos.max()) + 1 if angles is None else angles
        self.table = angle_table(size, rot, seed)
        self.cos_sin = torch.from_numpy(self.table).cuda()
        self.pool = gcb.KVPool.create(1, Hkv, d, ps, w.num_pages)
        self.pool.planes().view(torch.int16).fill_(0x7FC1)
        self.out = torch.full((T, Hq, d), float("nan"), dtype=torch.bfloat16, device="cuda")
        self.block_table = _i32(w.block_table, "cuda")
        self.prefix = _i32(w.prefix_lens, "cuda")
        self.cu = _i32(w.cu_new_lens, "cuda")

    def run(self, stream=None, **change):
        w = self.w
        a = dict(pool=self.pool.handle, q=self.q if self.Hq else None,
                 q_stride=self.q.stride(0) if self.Hq else 0, q_out=self.out if self.Hq else None,
                 k_new=self.k, k_stride=self.k.stride(0), v_new=self.v, v_stride=self.v.stride(0),
                 block_table=self.block_table, seq_lens=self.prefix, stream=stream, layer=0,
                 cu_new_lens=self.cu, batch=w.B, max_blocks_per_seq=w.max_blocks,
                 total_new_tokens=w.T_new, num_q_heads=self.Hq, cos_sin=self.cos_sin,
                 n_positions=self.table.shape[0], rot_dim=self.rot, positions=self.positions,
                 flags=gcb.GC_ROPE_INTERLEAVED if self.interleaved else 0)
        gcb.gc_kv_append_rope(**{**a, **change})

    def check(self, skipped_kv=(), skipped=()):
        """Everything but the skipped tokens is written, and nothing else."""
        w = self.w
        b = np.repeat(np.arange(w.B), w.new_lens)
        live = np.array([t not in skipped for t in range(w.T_new)], bool)
        kv = live & np.array([t not in skipped_kv for t in range(w.T_new)], bool)
        page, slot = w.block_table[b, np.minimum(self.slots // w.ps, w.max_blocks - 1)], \
            self.slots % w.ps
        got = bf16_bits(self.pool.planes())[0]
        if self.Hq:
            out = bf16_bits(self.out)
            check_rotated(out[live], self.q_bits[live], self.table, self.pos[live], self.rot,
                          self.interleaved)
            assert np.all(np.isnan(f64(out[~live])))
        check_rotated(got[0][page[kv], :, slot[kv]], self.k_bits[kv], self.table, self.pos[kv],
                      self.rot, self.interleaved)
        assert np.array_equal(got[1][page[kv], :, slot[kv]], self.v_bits[kv])
        rest = np.ones((w.num_pages, w.ps), bool)
        rest[page[kv], slot[kv]] = False
        assert np.all(got.transpose(0, 1, 3, 2, 4)[:, rest] == 0x7FC1)


@pytest.mark.parametrize("Hq,Hkv,d,ps,rot,interleaved,fused,P,n", [
    (4, 1, 64, 16, 64, False, False, [256], [64]),
    (4, 1, 64, 16, 64, True, True, [5, 0, 31, 16, 250], [1, 0, 33, 130, 7]),
    (6, 3, 64, 32, 16, False, True, [0, 100], [65, 3]),
    (5, 5, 128, 16, 128, False, False, [17, 0, 63], [1, 200, 15]),
    (64, 8, 128, 16, 128, False, True, [9215, 12, 400], [1, 1, 1]),
    (64, 8, 128, 128, 64, True, False, [127, 1], [2, 1000]),
    (32, 8, 128, 64, 48, True, True, [700], [1]),
    (16, 1, 128, 64, 112, False, True, [0, 3, 77, 63], [64, 0, 0, 66]),
    (0, 2, 64, 16, 32, False, False, [9, 40], [20, 5]),
    (0, 1, 64, 16, 64, True, True, [0], [513]),
])
def test_rotates_and_appends(Hq, Hkv, d, ps, rot, interleaved, fused, P, n):
    c = Call(P, n, Hq, Hkv, d, ps, rot, interleaved, fused, seed=Hq + d)
    c.run()
    assert c.pool.check() == gcb.GC_OK
    c.check()


@pytest.mark.parametrize("heads", [(0, 1), (4, 2)])
@pytest.mark.parametrize("batch", [7, 8, 9, 63, 64, 65, 200, 513])
def test_finds_each_request(batch, heads):
    """Few tokens of many requests, some with none, at the steps of the search."""
    rng = np.random.default_rng(batch)
    n = rng.choice([0, 1, 1, 1, 5], batch).astype(int)
    n[[0, -1]] = [0, 2]
    P = rng.integers(0, 70, batch)
    c = Call(P, n, *heads, 64, 16, 32, seed=batch, positions=rng.integers(0, 99, n.sum()))
    c.run()
    assert c.pool.check() == gcb.GC_OK
    c.check()


@pytest.mark.parametrize("interleaved", [False, True])
def test_positions_are_not_the_slots(interleaved):
    P, n = [0, 3, 40], [1, 17, 2]
    pos = np.random.default_rng(3).integers(0, 5000, sum(n))
    pos[:2] = [4999, 0]
    c = Call(P, n, 8, 2, 128, 16, 128, interleaved, positions=pos, seed=3)
    c.run()
    assert c.pool.check() == gcb.GC_OK
    c.check()


def test_angle_zero_and_half_turn_are_exact():
    c = Call([0], [2], 4, 1, 64, 16, 64, positions=[0, 1])
    c.table = np.zeros((2, 2, 32), np.float32)
    c.table[0, 0], c.table[1, 0] = 1.0, -1.0
    c.cos_sin.copy_(__import__("torch").from_numpy(c.table))
    c.run()
    out = bf16_bits(c.out)
    assert np.array_equal(f64(out[0]), f64(c.q_bits[0]))
    assert np.array_equal(f64(out[1]), -f64(c.q_bits[1]))


def test_q_in_place_and_another_stream():
    import torch
    c = Call([33, 7], [50, 3], 8, 2, 128, 32, 128, seed=8)
    c.out.copy_(c.q)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    c.run(stream=s, q=c.out, q_stride=8 * 128)
    assert c.pool.check(s) == gcb.GC_OK
    c.check()


def test_non_finite_values_stay_in_their_pairs():
    c = Call([0], [3], 4, 1, 64, 16, 64, seed=5)
    bits = c.q_bits.copy()
    bits[1, 2, 5], bits[2, 0, 40] = 0x7FC0, 0x7F80
    c.q.copy_(bf16_tensor(bits))
    c.run()
    bad = ~np.isfinite(f64(bf16_bits(c.out)))
    want = np.zeros_like(bad)
    want[1, 2, [5, 37]] = want[2, 0, [8, 40]] = True
    assert np.array_equal(bad, want)


def test_bad_positions_and_pages_are_skipped_and_recorded():
    c = Call([0, 20], [6, 4], 4, 1, 64, 16, 64, positions=np.arange(10), angles=10)
    c.positions[2], c.positions[7] = 10, -1
    c.run()
    assert c.pool.check() == gcb.GC_ERR_OUT_OF_RANGE
    c.check(skipped=(2, 7))
    # a page outside the pool, and a token past its block table
    c = Call([0, 20], [6, 4], 4, 1, 64, 16, 64, seed=1)
    c.block_table[1, 1] = c.w.num_pages
    c.run()
    assert c.pool.check() == gcb.GC_ERR_OUT_OF_RANGE
    c.check(skipped_kv=(6, 7, 8, 9))
    c = Call([12, 0], [30, 3], 4, 1, 64, 16, 64, seed=2)
    c.run(block_table=c.block_table[:, :1].contiguous(), max_blocks_per_seq=1)
    assert c.pool.check() == gcb.GC_ERR_OUT_OF_RANGE
    c.check(skipped_kv=range(4, 30))


def test_tokens_without_a_request_are_skipped():
    import torch
    c = Call([0, 5], [4, 4], 4, 1, 64, 16, 64)
    c.cu.copy_(torch.tensor([0, 4, 6], dtype=torch.int32))  # two tokens belong to nobody
    c.run()
    assert c.pool.check() == gcb.GC_ERR_OUT_OF_RANGE
    c.check(skipped=(6, 7))


def test_no_tokens_is_a_no_op():
    c = Call([4], [3], 4, 1, 64, 16, 64)
    c.run(total_new_tokens=0, q=None, k_new=None)
    c.run(batch=0, q=None, k_new=None)
    assert c.pool.check() == gcb.GC_OK
    c.check(skipped=range(3))


@pytest.mark.parametrize("status,change", [
    (gcb.GC_ERR_INVALID_ARG, dict(pool=None)),
    (gcb.GC_ERR_INVALID_ARG, dict(batch=-1)),
    (gcb.GC_ERR_INVALID_ARG, dict(total_new_tokens=-1)),
    (gcb.GC_ERR_INVALID_ARG, dict(max_blocks_per_seq=0)),
    (gcb.GC_ERR_INVALID_ARG, dict(n_positions=-1)),
    (gcb.GC_ERR_INVALID_ARG, dict(flags=2)),
    (gcb.GC_ERR_OUT_OF_RANGE, dict(layer=1)),
    (gcb.GC_ERR_OUT_OF_RANGE, dict(layer=-1)),
    (gcb.GC_ERR_INVALID_ARG, dict(num_q_heads=7)),
    (gcb.GC_ERR_INVALID_ARG, dict(num_q_heads=-2)),
    (gcb.GC_ERR_UNSUPPORTED, dict(num_q_heads=1 << 24, q_stride=1 << 30)),
    (gcb.GC_ERR_INVALID_ARG, dict(rot_dim=0)),
    (gcb.GC_ERR_INVALID_ARG, dict(rot_dim=24)),
    (gcb.GC_ERR_INVALID_ARG, dict(rot_dim=80)),
    (gcb.GC_ERR_INVALID_ARG, dict(q_stride=8 * 64 - 8)),
    (gcb.GC_ERR_INVALID_ARG, dict(k_stride=64)),
    (gcb.GC_ERR_INVALID_ARG, dict(v_stride=2 * 64 + 4)),
    (gcb.GC_ERR_INVALID_ARG, dict(q=None)),
    (gcb.GC_ERR_INVALID_ARG, dict(q_out=None)),
    (gcb.GC_ERR_INVALID_ARG, dict(k_new=None)),
    (gcb.GC_ERR_INVALID_ARG, dict(v_new=None)),
    (gcb.GC_ERR_INVALID_ARG, dict(block_table=None)),
    (gcb.GC_ERR_INVALID_ARG, dict(seq_lens=None)),
    (gcb.GC_ERR_INVALID_ARG, dict(cu_new_lens=None)),
    (gcb.GC_ERR_INVALID_ARG, dict(cos_sin=None)),
    (gcb.GC_ERR_INVALID_ARG, dict(k_new=8)),
    (gcb.GC_ERR_INVALID_ARG, dict(q_out=4096, q=4096, q_stride=8 * 64 + 8)),
])
def test_refusals(status, change):
    c = Call([0, 5], [4, 4], 8, 2, 64, 16, 64)
    with pytest.raises(gcb.GcError) as e:
        c.run(**change)
    assert e.value.status == status
    assert "gc_kv_append_rope: " in str(e.value)
    assert c.pool.check() == gcb.GC_OK
    c.check(skipped=range(8))
