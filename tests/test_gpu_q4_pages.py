"""Writing the 4-bit cache and reading it back, bit for bit: packed pages, appended
tokens (rotated or not), read-back pages, and everything that is skipped or refused."""
import numpy as np
import pytest

from paper_2505_23970_gb300 import binding as gcb
from paper_2505_23970_gb300 import workloads as wl
from paper_2505_23970_gb300.harness import _i32, bf16_bits, bf16_tensor

from . import _q4

pytestmark = pytest.mark.gpu


def special_rows(shape, seed=0):
    """Normal rows, some with infinities, NaN, zeros, huge, tiny and exactly tied values."""
    x = wl.normal_bf16(seed, 51, shape)
    rng = np.random.default_rng([seed, 52])
    flat = x.reshape(-1, 32)
    for bits in (0x7F80, 0xFF80, 0x7FC0, 0xFFC1, 0x7F7F, 0x0001, 0x8000, 0x4780):
        at = rng.integers(0, len(flat), max(1, len(flat) // 40))
        flat[at, rng.integers(0, 32, at.size)] = bits
    flat[rng.integers(0, len(flat), max(1, len(flat) // 40))] = 0
    for scale in (1e-9, 3e-7, 1e30, 2.0 ** 17):
        at = rng.integers(0, len(flat), max(1, len(flat) // 40))
        with np.errstate(over="ignore", invalid="ignore"):
            flat[at] = wl.f32_to_bf16_bits(_q4.f32(flat[at]) * np.float32(scale))
    # ties: multiples of half a step
    at = rng.integers(0, len(flat), max(1, len(flat) // 20))
    step = _q4.f32(wl.f32_to_bf16_bits(rng.uniform(0.5, 2, (at.size, 1)).astype(np.float32)))
    half = rng.integers(-14, 15, (at.size, 32)) * 0.5
    flat[at] = wl.f32_to_bf16_bits((half * step).astype(np.float32))
    flat[at, 0] = wl.f32_to_bf16_bits((7 * step[:, 0]).astype(np.float32))
    return x


def same(got, want):
    bad = np.argwhere(got != want)
    assert not len(bad), f"{len(bad)} of {got.size} differ, the first at {bad[0]}: " \
        f"{got[tuple(bad[0])]} for {want[tuple(bad[0])]}"


def pool_of(bits):
    L, _, n, Hkv, ps, d = bits.shape
    pool = gcb.KVPool.create(L, Hkv, d, ps, n)
    pool.planes().copy_(bf16_tensor(bits))
    return pool


@pytest.mark.parametrize("L,Hkv,d,ps,n,layers", [
    (1, 1, 64, 16, 1, (0, 1)), (3, 2, 64, 16, 5, (1, 2)), (2, 8, 128, 16, 33, (0, 2)),
    (1, 3, 128, 32, 7, (0, 1)), (4, 5, 64, 128, 3, (3, 1)), (2, 1, 128, 64, 20, (0, 1)),
    (1, 8, 128, 16, 700, (0, 1))])
def test_pages_are_packed_and_read_back(L, Hkv, d, ps, n, layers):
    import torch
    bits = special_rows((L, 2, n + 3, Hkv, ps, d), seed=L + n)
    pool = pool_of(bits)
    rng = np.random.default_rng(n)
    src, dst = rng.permutation(n + 3)[:n], rng.permutation(n + 2)[:n]
    cache = torch.full((L, 2, n + 2, Hkv, ps * (d // 2 + d // 16)), 0xA5, dtype=torch.uint8,
                       device="cuda")
    assert cache.numel() == gcb.gc_kv_q4_bytes(pool.cfg, n + 2)
    gcb.gc_kv_pack_q4(pool.handle, _i32(src, "cuda"), cache, n + 2, _i32(dst, "cuda"), n, *layers)
    assert pool.check() == gcb.GC_OK
    want = np.full(cache.shape, 0xA5, np.uint8)
    on = slice(layers[0], layers[0] + layers[1])
    want[on, :, dst] = _q4.cache_bytes(bits)[on, :, src]
    same(cache.cpu().numpy(), want)
    # back into other pages
    to = rng.permutation(n + 3)[:n]
    gcb.gc_kv_unpack_q4(pool.handle, cache, n + 2, _i32(dst, "cuda"), _i32(to, "cuda"), n, *layers)
    assert pool.check() == gcb.GC_OK
    back = bits.copy()
    back[on, :, to] = wl.f32_to_bf16_bits(_q4.values(bits))[on, :, src]
    # (a code 0 of a negative value is +0, c s being a product of whole numbers and s)
    back[on, :, to] = np.where(back[on, :, to] == 0x8000, 0, back[on, :, to])
    same(bf16_bits(pool.planes()), back)


def test_bad_pages_are_skipped_and_recorded():
    import torch
    bits = wl.normal_bf16(1, 2, (2, 2, 4, 2, 16, 64))
    pool = pool_of(bits)
    row = 16 * 36
    cache = torch.zeros((2, 2, 3, 2, row), dtype=torch.uint8, device="cuda")
    src, dst = _i32([0, 4, 2, -1, 3], "cuda"), _i32([1, 0, 3, 0, 2], "cuda")
    gcb.gc_kv_pack_q4(pool.handle, src, cache, 3, dst, 5, 0, 2)
    assert pool.check() == gcb.GC_ERR_OUT_OF_RANGE
    want = np.zeros(cache.shape, np.uint8)
    want[:, :, [1, 2]] = _q4.cache_bytes(bits)[:, :, [0, 3]]
    same(cache.cpu().numpy(), want)
    gcb.gc_kv_unpack_q4(pool.handle, cache, 3, _i32([-1, 3, 1, 2], "cuda"),
                        _i32([0, 1, 2, 4], "cuda"), 4, 1, 1)
    assert pool.check() == gcb.GC_ERR_OUT_OF_RANGE
    back = bits.copy()
    back[1, :, 2] = wl.f32_to_bf16_bits(_q4.values(bits[1, :, 0]) + 0.0)
    same(bf16_bits(pool.planes()), back)
    assert pool.check() == gcb.GC_OK


# ------------------------------------------------------------------ append
class Append:
    def __init__(self, P, n, Hq, Hkv, d, ps, rot, interleaved=False, fused=True, positions=None,
                 seed=0, L=1, layer=0, rows=None):
        import torch
        self.w = w = wl.custom("append-q4", len(P), max(Hq, Hkv), Hkv, d, ps, P, n, seed=seed)
        T = w.T_new
        self.Hq, self.rot, self.layer, self.L = Hq, rot, layer, L
        self.interleaved = interleaved
        self.bits = wl.normal_bf16(seed, 61, (T, Hq + 2 * Hkv, d)) if rows is None else rows
        dev = bf16_tensor(self.bits)
        parts = (dev[:, :Hq], dev[:, Hq:Hq + Hkv], dev[:, Hq + Hkv:])
        self.q, self.k, self.v = parts if fused else [x.contiguous() for x in parts]
        self.slots = np.concatenate([np.arange(p, p + m) for p, m in zip(P, n)] or [[]]).astype(np.int64)
        self.pos = self.slots if positions is None else np.asarray(positions, np.int64)
        self.positions = None if positions is None else _i32(self.pos, "cuda")
        angle = np.arange(int(self.pos.max(initial=0)) + 1)[:, None] * \
            1e4 ** (-np.arange(0, max(rot, 2), 2) / max(rot, 2))
        self.cs = np.stack([np.cos(angle), np.sin(angle)], 1).astype(np.float32)
        self.cos_sin = torch.from_numpy(self.cs).cuda()
        self.pool = gcb.KVPool.create(L, Hkv, d, ps, w.num_pages)
        self.pool.planes().zero_()
        self.cache = torch.full((L, 2, w.num_pages, Hkv, ps * (d // 2 + d // 16)), 0x5A,
                                dtype=torch.uint8, device="cuda")
        self.out = torch.full((T, Hq, d), float("nan"), dtype=torch.bfloat16, device="cuda")
        self.table, self.prefix = _i32(w.block_table, "cuda"), _i32(w.prefix_lens, "cuda")
        self.cu = _i32(w.cu_new_lens, "cuda")

    def args(self, **change):
        w = self.w
        a = dict(pool=self.pool.handle, q=self.q if self.Hq else None,
                 q_stride=self.q.stride(0) if self.Hq else 0, q_out=self.out if self.Hq else None,
                 k_new=self.k, k_stride=self.k.stride(0), v_new=self.v, v_stride=self.v.stride(0),
                 q4_cache=self.cache, n_q4_pages=w.num_pages, q4_table=self.table,
                 seq_lens=self.prefix, stream=None, layer=self.layer, cu_new_lens=self.cu,
                 batch=w.B, max_blocks_per_seq=w.max_blocks, total_new_tokens=w.T_new,
                 num_q_heads=self.Hq, cos_sin=self.cos_sin if self.rot else None,
                 n_positions=self.cs.shape[0] if self.rot else 0, rot_dim=self.rot,
                 positions=self.positions,
                 flags=gcb.GC_ROPE_INTERLEAVED if self.interleaved else 0)
        return {**a, **change}

    def run(self, **change):
        gcb.gc_kv_append_rope_q4(**self.args(**change))

    def turned(self, x):
        """The rotation's stated rounding, in 64 bits with its steps rounded."""
        v = _q4.f32(x).astype(np.float64)
        rot, half = self.rot, self.rot // 2
        if not rot:
            return x.copy()
        i = np.arange(half)
        a, b = (2 * i, 2 * i + 1) if self.interleaved else (i, i + half)
        c = self.cs[self.pos, 0][:, None].astype(np.float64)
        s = self.cs[self.pos, 1][:, None].astype(np.float64)
        r32 = lambda y: y.astype(np.float32).astype(np.float64)
        w = v.copy()
        w[..., a] = v[..., a] * c - r32(v[..., b] * s)
        w[..., b] = v[..., b] * c + r32(v[..., a] * s)
        out = x.copy()
        out[..., :rot] = wl.f32_to_bf16_bits(w[..., :rot].astype(np.float32))
        return out

    def check(self, skipped_kv=(), skipped=()):
        import torch
        w, Hq = self.w, self.Hq
        T = w.T_new
        live = np.array([t not in skipped for t in range(T)], bool)
        kv = live & np.array([t not in skipped_kv for t in range(T)], bool)
        if Hq:
            got = bf16_bits(self.out)
            same(got[live], self.turned(self.bits[:, :Hq])[live])
            assert np.all(np.isnan(_q4.f32(got[~live])))
        d, ps = w.d, w.ps
        want = np.full(self.cache.shape, 0x5A, np.uint8)
        b = np.repeat(np.arange(w.B), w.new_lens)
        page = w.block_table[b, np.minimum(self.slots // ps, w.max_blocks - 1)]
        slot = self.slots % ps
        for plane, x in enumerate((self.turned(self.bits[:, Hq:Hq + w.Hkv]),
                                   self.bits[:, Hq + w.Hkv:])):
            codes, scales = _q4.row_bytes(x, plane == 0)
            scales = np.ascontiguousarray(scales).view(np.uint8)
            wc = want[self.layer, plane, ..., :ps * d // 2].reshape(-1, w.Hkv, ps, d // 2)
            ws = want[self.layer, plane, ..., ps * d // 2:].reshape(-1, w.Hkv, ps, d // 16)
            wc[page[kv], :, slot[kv]] = codes[kv]
            ws[page[kv], :, slot[kv]] = scales[kv]
            want[self.layer, plane, ..., :ps * d // 2] = wc.reshape(-1, w.Hkv, ps * d // 2)
            want[self.layer, plane, ..., ps * d // 2:] = ws.reshape(-1, w.Hkv, ps * d // 16)
        same(self.cache.cpu().numpy(), want)
        assert not torch.any(self.pool.planes().view(torch.int16))  # the pool is not written


@pytest.mark.parametrize("Hq,Hkv,d,ps,rot,interleaved,fused,P,n", [
    (4, 1, 64, 16, 64, False, False, [256], [64]),
    (4, 1, 64, 16, 64, True, True, [5, 0, 31, 16, 250], [1, 0, 33, 130, 7]),
    (6, 3, 64, 32, 16, False, True, [0, 100], [65, 3]),
    (5, 5, 128, 16, 128, False, False, [17, 0, 63], [1, 200, 15]),
    (64, 8, 128, 16, 128, False, True, [9215, 12, 400], [1, 1, 1]),
    (64, 8, 128, 128, 64, True, False, [127, 1], [2, 1000]),
    (32, 8, 128, 64, 48, False, True, [700], [1]),
    (32, 8, 128, 16, 96, False, True, [3, 50], [90, 400]),
    (16, 1, 128, 64, 112, True, True, [0, 3, 77, 63], [64, 0, 0, 66]),
    (8, 2, 64, 16, 48, False, True, [1, 2], [40, 17]),
    (64, 8, 128, 16, 0, False, True, [30, 0], [700, 5]),
    (0, 2, 64, 16, 32, False, False, [9, 40], [20, 5]),
    (0, 1, 64, 16, 0, False, True, [0], [513]),
])
def test_rotates_quantises_and_appends(Hq, Hkv, d, ps, rot, interleaved, fused, P, n):
    c = Append(P, n, Hq, Hkv, d, ps, rot, interleaved, fused, seed=Hq + d)
    c.run()
    assert c.pool.check() == gcb.GC_OK
    c.check()


@pytest.mark.parametrize("d,rot", [(64, 0), (128, 0)])
def test_appends_special_values(d, rot):
    rows = special_rows((300, 4 + 2 * 2, d), seed=d)
    c = Append([7, 100], [200, 100], 4, 2, d, 16, rot, rows=rows)
    c.run()
    assert c.pool.check() == gcb.GC_OK
    c.check()


@pytest.mark.parametrize("heads", [(0, 1), (4, 2)])
@pytest.mark.parametrize("batch", [1, 7, 9, 64, 65, 513])
def test_finds_each_request(batch, heads):
    """Few tokens of many requests, some with none."""
    rng = np.random.default_rng(batch)
    n = rng.choice([0, 1, 1, 1, 5], batch).astype(int)
    n[[0, -1]] = [0, 2]
    P = rng.integers(0, 70, batch)
    c = Append(P, n, *heads, 64, 16, 32, seed=batch, positions=rng.integers(0, 99, n.sum()))
    c.run()
    assert c.pool.check() == gcb.GC_OK
    c.check()


def test_a_layer_of_several_and_positions_that_are_not_slots():
    c = Append([0, 3, 40], [1, 17, 2], 8, 2, 128, 16, 128, positions=np.arange(20) * 7, L=3,
               layer=2, seed=9)
    c.run()
    assert c.pool.check() == gcb.GC_OK
    c.check()


def test_in_place_q():
    import torch
    c = Append([10], [40], 8, 2, 128, 16, 128, fused=False, seed=4)
    q = c.q.clone()
    c.run(q=q, q_out=q)
    assert c.pool.check() == gcb.GC_OK
    c.out.copy_(q)
    c.check()
    # and without a rotation
    c = Append([10], [40], 8, 2, 128, 16, 0, fused=False, seed=4)
    c.run(q=c.q, q_out=c.q)
    assert c.pool.check() == gcb.GC_OK
    assert torch.equal(bf16_tensor(c.bits[:, :8]), c.q)


def test_tokens_without_a_page_are_skipped():
    import torch
    c = Append([10, 0, 30], [10, 5, 20], 4, 2, 64, 16, 64, seed=5)
    table = c.w.block_table.copy()
    table[0, 1], table[2, 2] = -1, c.w.num_pages  # slots 16-19 of the first, 32-47 of the third
    c.run(q4_table=_i32(table, "cuda"))
    torch.cuda.synchronize()
    assert c.pool.check() == gcb.GC_ERR_OUT_OF_RANGE
    c.check(skipped_kv=[*range(6, 10), *range(15 + 2, 15 + 18)])
    # a position past the angles: nothing of the token is written
    c = Append([10, 0], [10, 5], 4, 2, 64, 16, 64, seed=5)
    c.run(n_positions=18)
    assert c.pool.check() == gcb.GC_ERR_OUT_OF_RANGE
    c.check(skipped=[8, 9])
    # without a rotation there are no angles to be past
    c = Append([10, 0], [10, 5], 4, 2, 64, 16, 0, seed=5)
    c.run(n_positions=3, positions=_i32(np.full(15, 99), "cuda"))
    assert c.pool.check() == gcb.GC_OK
    c.check()


def test_equals_append_then_pack():
    """The page holds what packing the 16-bit page would give."""
    import torch
    c = Append([0, 16], [48, 32], 8, 2, 128, 16, 128, seed=6)
    c.run()
    w = c.w
    out = torch.empty_like(c.out)
    gcb.gc_kv_append_rope(c.pool.handle, c.q, c.q.stride(0), out, c.k, c.k.stride(0), c.v,
                          c.v.stride(0), c.table, c.prefix, None, 0, c.cu, w.B, w.max_blocks,
                          w.T_new, 8, c.cos_sin, c.cs.shape[0], 128)
    ids = np.concatenate([w.block_table[0, :3], w.block_table[1, 1:3]])
    packed = torch.full_like(c.cache, 0x5A)
    gcb.gc_kv_pack_q4(c.pool.handle, _i32(ids, "cuda"), packed, w.num_pages, _i32(ids, "cuda"), 5,
                      0, 1)
    assert c.pool.check() == gcb.GC_OK
    assert torch.equal(packed, c.cache) and torch.equal(out, c.out)


def refused(status, call, **change):
    with pytest.raises(gcb.GcError) as e:
        call(**change)
    assert e.value.status == status, change


def test_append_refusals():
    c = Append([10], [4], 4, 2, 64, 16, 32)
    for change in (dict(batch=-1), dict(total_new_tokens=-1), dict(n_q4_pages=-1), dict(flags=2),
                   dict(num_q_heads=3), dict(rot_dim=8), dict(rot_dim=80), dict(rot_dim=-16),
                   dict(k_stride=120), dict(q_stride=255 + 4), dict(q_stride=128),
                   dict(k_new=None), dict(q=None), dict(q4_table=None), dict(seq_lens=None),
                   dict(cos_sin=None), dict(q4_cache=None), dict(max_blocks_per_seq=0),
                   dict(q4_cache=c.cache.data_ptr() + 8), dict(k_new=c.k.data_ptr() + 2),
                   dict(q_out=c.q, q_stride=c.q.stride(0))):
        refused(gcb.GC_ERR_INVALID_ARG, lambda **k: c.run(**k), **change)
    refused(gcb.GC_ERR_OUT_OF_RANGE, lambda **k: c.run(**k), layer=1)
    c.run(batch=0)
    c.run(total_new_tokens=0, q4_cache=None)
    assert c.pool.check() == gcb.GC_OK
    assert bool((c.cache == 0x5A).all())
    c.run(n_q4_pages=0)  # a cache without pages: every token's page is outside it
    assert c.pool.check() == gcb.GC_ERR_OUT_OF_RANGE


def test_page_refusals():
    pool = pool_of(wl.normal_bf16(1, 2, (2, 2, 2, 1, 16, 64)))
    ids = _i32([0], "cuda")
    import torch
    cache = torch.zeros(gcb.gc_kv_q4_bytes(pool.cfg, 2), dtype=torch.uint8, device="cuda")
    ok = dict(pool=pool.handle, pool_ids=ids, q4_cache=cache, n_q4_pages=2, q4_ids=ids, n_blocks=1,
              layer_begin=0, layer_count=2)
    for fn in (gcb.gc_kv_pack_q4, gcb.gc_kv_unpack_q4):
        for change in (dict(pool_ids=None), dict(q4_ids=None), dict(q4_cache=None),
                       dict(q4_cache=cache.data_ptr() + 4), dict(n_blocks=-1),
                       dict(n_q4_pages=-1)):
            refused(gcb.GC_ERR_INVALID_ARG, lambda **k: fn(**{**ok, **k}), **change)
        for change in (dict(layer_begin=2, layer_count=1), dict(layer_begin=-1),
                       dict(layer_count=3)):
            refused(gcb.GC_ERR_OUT_OF_RANGE, lambda **k: fn(**{**ok, **k}), **change)
        fn(**{**ok, "n_blocks": 0, "q4_cache": None})
        fn(**{**ok, "layer_count": 0})
    assert pool.check() == gcb.GC_OK
    assert not bool(cache.any())
