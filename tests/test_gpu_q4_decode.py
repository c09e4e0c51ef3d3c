"""gc_paged_decode_attn_q4 against attention over the values that the 4-bit pages hold,
in 64 bits; the bound of a value is derived in _q4.decode_reference."""
import numpy as np
import pytest

from paper_2505_23970_gb300 import binding as gcb
from paper_2505_23970_gb300 import workloads as wl
from paper_2505_23970_gb300.harness import _i32, bf16_tensor

from . import _q4

pytestmark = pytest.mark.gpu


class Decode:
    def __init__(self, ctx, Hq, tokens=1, q_bits=None, scale=None, seed=0):
        import torch
        self.ctx, self.Hq, self.tokens = ctx, Hq, tokens
        self.B = len(ctx.lens)
        self.q_bits = wl.normal_bf16(seed, 71, (self.B, tokens, Hq, ctx.d)) if q_bits is None else q_bits
        self.q = bf16_tensor(self.q_bits)
        self.scale = ctx.d ** -0.5 if scale is None else scale
        self.out = torch.full((self.B, tokens, Hq, ctx.d), float("nan"), dtype=torch.bfloat16,
                              device="cuda")
        self.need = gcb.gc_paged_decode_q4_workspace_bytes(ctx.pool.handle, self.B, ctx.width, Hq,
                                                           tokens)
        self.ws = torch.full((self.need,), 0xFF, dtype=torch.uint8, device="cuda")

    def args(self, **change):
        c = self.ctx
        a = dict(q=self.q, pool=c.pool.handle, block_table=c.dev16, seq_lens=c.seq_lens,
                 out=self.out, stream=None, layer=c.layer, batch=self.B,
                 max_blocks_per_seq=c.width, num_q_heads=self.Hq, softmax_scale=self.scale,
                 workspace=self.ws, workspace_bytes=self.need, q4_cache=c.cache, q4_table=c.dev4,
                 n_q4_pages=c.pages4, tokens=self.tokens)
        return {**a, **change}

    def run(self, **change):
        gcb.gc_paged_decode_attn_q4(**self.args(**change))
        return self

    def check(self, skip=(), only=None):
        c = self.ctx
        got = self.out.double().cpu().numpy()
        for b in range(self.B) if only is None else only:
            if b in skip:
                assert np.isnan(got[b]).all(), b
                continue
            kv, s = c.keys(b)
            want, bound = _q4.decode_reference(_q4.f32(self.q_bits[b]).astype(np.float64), kv, s,
                                               self.scale, self.tokens)
            assert np.isfinite(got[b]).all(), (b, c.lens[b])
            over = np.abs(got[b] - want) - bound
            assert (over <= 0).all(), (b, c.lens[b], int((over > 0).sum()), over.max(),
                                       np.abs(got[b] - want).max())
        return self


@pytest.mark.parametrize("Hq,Hkv,d,ps,lens", [
    (4, 1, 64, 16, [321]),
    (4, 1, 128, 16, [1]),
    (1, 1, 64, 16, [1, 2, 15, 16, 17, 31, 32, 33, 64, 255, 256, 257]),
    (8, 8, 128, 16, [1, 2, 15, 16, 17, 31, 32, 33, 64, 255, 256, 257]),
    (16, 2, 128, 16, [9216, 1, 700]),
    (64, 8, 128, 16, [3000, 17, 1234, 5]),
    (16, 1, 128, 64, [2100, 63, 64, 65]),
    (32, 2, 64, 128, [130, 1000, 4097]),
    (2, 1, 64, 32, [40, 5000]),
    (6, 3, 128, 32, [777, 31]),
    (16, 1, 64, 16, [100] * 40),
    (64, 8, 128, 16, [12 + 5 * i for i in range(60)]),
])
def test_decode(Hq, Hkv, d, ps, lens):
    ctx = _q4.Context(lens, Hkv, d, ps, seed=len(lens) + d)
    Decode(ctx, Hq).run().check()
    assert ctx.pool.check() == gcb.GC_OK


@pytest.mark.parametrize("recent", [1, 3, 1000])
@pytest.mark.parametrize("Hq,Hkv,d,ps,lens", [
    (8, 2, 64, 16, [1, 16, 17, 300, 2000]),
    (16, 2, 128, 16, [1, 16, 33, 300, 2000]),
    (16, 1, 128, 64, [500, 129, 64]),
])
def test_newest_pages_in_16_bits(Hq, Hkv, d, ps, lens, recent):
    ctx = _q4.Context(lens, Hkv, d, ps, recent=recent, seed=recent)
    Decode(ctx, Hq).run().check()
    assert ctx.pool.check() == gcb.GC_OK


@pytest.mark.parametrize("recent", [0, 1])
@pytest.mark.parametrize("Hq,Hkv,d,ps,tokens,lens", [
    (4, 1, 64, 16, 4, [4, 5, 16, 17, 18, 19, 20, 600]),
    (32, 8, 128, 16, 4, [8192, 33, 4, 50]),
    (32, 8, 128, 32, 2, [64, 2, 3, 700]),
    (8, 8, 64, 16, 16, [16, 17, 31, 32, 47, 48, 1000]),
    (8, 8, 128, 16, 7, [7, 8, 16, 20, 22, 23, 500]),
    (4, 2, 128, 16, 3, [3, 17, 18, 33, 34] * 12),
])
def test_drafted_tokens(Hq, Hkv, d, ps, tokens, lens, recent):
    ctx = _q4.Context(lens, Hkv, d, ps, recent=recent, seed=tokens)
    Decode(ctx, Hq, tokens).run().check()
    assert ctx.pool.check() == gcb.GC_OK


def test_a_layer_of_several_and_a_wide_table():
    ctx = _q4.Context([100, 1500], 2, 64, 16, recent=1, L=3, layer=1, width=4000)
    Decode(ctx, 8).run().check()
    assert ctx.pool.check() == gcb.GC_OK


@pytest.mark.parametrize("size,q_size", [(1e-5, 1.0), (3e4, 1e-4), (1.0, 1e-20), (1e-3, 1e3),
                                         (1.0, 30.0)])
def test_sizes_of_values(size, q_size):
    """Small and large keys, values and queries; scores that leave one key."""
    ctx = _q4.Context([500, 33], 2, 128, 16, size=size, recent=1, seed=8)
    bits = wl.normal_bf16(8, 71, (2, 1, 8, 128))
    bits = wl.f32_to_bf16_bits((_q4.f32(bits) * np.float32(q_size)).astype(np.float32))
    Decode(ctx, 8, q_bits=bits).run().check()
    assert ctx.pool.check() == gcb.GC_OK


def test_columns_far_apart():
    """Columns of q that differ by up to 2^30 within a head: each product is exact."""
    ctx = _q4.Context([700, 40], 2, 128, 16, recent=1, seed=12)
    bits = wl.normal_bf16(12, 71, (2, 1, 8, 128))
    size = 2.0 ** -np.random.default_rng(12).integers(0, 31, (1, 1, 8, 128)).astype(np.float32)
    bits = wl.f32_to_bf16_bits((_q4.f32(bits) * size * 8).astype(np.float32))
    Decode(ctx, 8, q_bits=bits).run().check()
    assert ctx.pool.check() == gcb.GC_OK


@pytest.mark.parametrize("q_exp,k_exp", [(100, 0), (-110, 0), (40, 58), (3, -60)])
def test_the_ends_of_the_range(q_exp, k_exp):
    """|q| up to 2^100, keys of 16-bit pages up to 2^60, with scales that bring the scores
    back to the size of one (those of the other pages are then near 0 or one key's)."""
    ctx = _q4.Context([90], 1, 64, 16, recent=100 if k_exp else 0, seed=13)
    if k_exp:
        import torch
        k = _q4.f32(ctx.bits16[0, 0]) * np.float32(2.0 ** k_exp)
        ctx.bits16[0, 0] = wl.f32_to_bf16_bits(k.astype(np.float32))
        ctx.pool.planes().copy_(bf16_tensor(ctx.bits16))
    q = _q4.f32(wl.normal_bf16(13, 71, (1, 1, 4, 64))) / 4
    bits = wl.f32_to_bf16_bits((q * np.float32(2.0 ** q_exp)).astype(np.float32))
    scale = float(np.float32(2.0 ** (-q_exp - k_exp)))
    Decode(ctx, 4, q_bits=bits, scale=min(scale, 8192.0)).run().check()
    assert ctx.pool.check() == gcb.GC_OK


def test_scores_that_keep_rising():
    """Each group of keys far above the ones before: the reference maximum is raised."""
    ctx = _q4.Context([640], 1, 128, 16, seed=3)
    bits = ctx.bits4.copy()
    for j in range(40):
        p = ctx.table4[0, j]
        bits[0, 0, p] = wl.f32_to_bf16_bits(
            (_q4.f32(bits[0, 0, p]) * np.float32(0.05 + j * 0.3)).astype(np.float32))
    ctx.bits4 = bits
    import torch
    ctx.cache.copy_(torch.from_numpy(_q4.cache_bytes(bits)))
    Decode(ctx, 8).run().check()
    assert ctx.pool.check() == gcb.GC_OK


def test_queries_of_zero_and_not_finite():
    ctx = _q4.Context([300], 1, 64, 16, seed=4)
    bits = wl.normal_bf16(4, 71, (1, 1, 4, 64))
    bits[0, 0, 1] = 0
    bits[0, 0, 2, 5] = 0x7FC0
    d = Decode(ctx, 4, q_bits=bits).run()
    got = d.out.double().cpu().numpy()[0, 0]
    assert np.isnan(got[2]).all()
    kv, s = ctx.keys(0)
    keep = [0, 1, 3]
    want, bound = _q4.decode_reference(_q4.f32(bits[0][:, keep]).astype(np.float64)[:, :], kv, s,
                                       d.scale, 1)
    assert (np.abs(got[keep] - want[0]) <= bound[0]).all()


@pytest.mark.parametrize("Hq,Hkv,d,tokens,lens", [
    (4, 1, 64, 4, [4, 5, 16, 17, 18, 19, 20, 600]),
    (32, 8, 128, 4, [4, 17, 33, 500]),
    (16, 2, 128, 2, [2, 16, 17, 33]),
    (8, 8, 128, 7, [7, 20, 23, 500]),
    (8, 8, 64, 16, [16, 17, 32, 47]),
])
def test_drafted_tokens_that_are_not_finite(Hq, Hkv, d, tokens, lens):
    """The newest token's K and V in a 16-bit page are NaN and infinities: only its own
    row sees them."""
    ctx = _q4.Context(lens, Hkv, d, 16, recent=1, seed=14)
    for b, T in enumerate(lens):
        page = ctx.table16[b, (T - 1) // 16]
        ctx.bits16[0, 0, page, :, (T - 1) % 16] = 0x7FC0
        ctx.bits16[0, 1, page, :, (T - 1) % 16] = 0x7F80 | (np.arange(d) % 2) << 15
    ctx.pool.planes().copy_(bf16_tensor(ctx.bits16))
    c = Decode(ctx, Hq, tokens).run()
    assert ctx.pool.check() == gcb.GC_OK
    got = c.out.double().cpu().numpy()
    for b, T in enumerate(lens):
        kv, s = ctx.keys(b)
        kv[:, -1] = 0
        want, bound = _q4.decode_reference(_q4.f32(c.q_bits[b]).astype(np.float64), kv, s, c.scale,
                                           tokens)
        assert np.isnan(got[b, -1]).all(), T
        assert (np.abs(got[b, :-1] - want[:-1]) <= bound[:-1]).all(), T


@pytest.mark.parametrize("recent", [0, 1])
def test_the_smallest_queries_and_scale(recent):
    """Scores that are all 0 in binary32: the mean of the values."""
    ctx = _q4.Context([17, 300], 2, 64, 16, recent=recent, seed=15)
    bits = np.full((2, 1, 4, 64), 1, np.uint16)
    Decode(ctx, 4, q_bits=bits, scale=1e-30).run().check()
    assert ctx.pool.check() == gcb.GC_OK


def test_lengths_outside_the_table_are_skipped():
    ctx = _q4.Context([300, 40, 64, 20], 2, 64, 16, seed=5)
    cap = ctx.width * 16
    d = Decode(ctx, 4, tokens=2)
    d.run(seq_lens=_i32([300, 1, cap + 1, -5], "cuda"))
    assert ctx.pool.check() == gcb.GC_ERR_OUT_OF_RANGE
    d.check(skip=(1, 2, 3))
    d.out.fill_(float("nan"))
    d.run(seq_lens=_i32([0, 40, 64, 20], "cuda"))
    assert ctx.pool.check() == gcb.GC_ERR_OUT_OF_RANGE
    d.check(skip=(0,))


def test_bad_pages_are_left_out():
    ctx = _q4.Context([300, 40], 2, 64, 16, seed=6)
    t4, t16 = ctx.table4.copy(), ctx.table16.copy()
    t4[0, 3], t4[0, 7], t16[0, 7] = ctx.pages4, -1, ctx.pages16
    d = Decode(ctx, 4).run(q4_table=_i32(t4, "cuda"), block_table=_i32(t16, "cuda"))
    assert ctx.pool.check() == gcb.GC_ERR_OUT_OF_RANGE
    assert ctx.pool.check() == gcb.GC_OK
    kv, s = ctx.keys(0)
    left = np.array([t not in range(48, 64) and t not in range(112, 128) for t in range(300)])
    want, bound = _q4.decode_reference(_q4.f32(d.q_bits[0]).astype(np.float64), kv[:, left],
                                       s[:, left], d.scale, 1)
    assert (np.abs(d.out.double().cpu().numpy()[0] - want) <= bound).all()


def test_a_request_without_a_page_that_is_left():
    ctx = _q4.Context([300, 40], 2, 64, 16, seed=16)
    t4 = ctx.table4.copy()
    t4[0] = ctx.pages4
    d = Decode(ctx, 4).run(q4_table=_i32(t4, "cuda"))
    assert ctx.pool.check() == gcb.GC_ERR_OUT_OF_RANGE
    assert np.isnan(d.out[0].double().cpu().numpy()).all()
    d.check(only=[1])


def test_the_same_call_gives_the_same_bits():
    import torch
    ctx = _q4.Context([5000, 3, 800, 77], 8, 128, 16, recent=1, seed=7)
    d = Decode(ctx, 64)
    first = d.run().out.clone()
    for _ in range(5):
        d.out.zero_()
        d.ws.random_(0, 255)
        assert torch.equal(d.run().out, first)


def refused(status, d, **change):
    with pytest.raises(gcb.GcError) as e:
        d.run(**change)
    assert e.value.status == status, change


def test_refusals():
    ctx = _q4.Context([100], 2, 64, 16)
    d = Decode(ctx, 8)
    for change in (dict(batch=-1), dict(max_blocks_per_seq=-1), dict(n_q4_pages=-1), dict(tokens=0),
                   dict(tokens=-3), dict(num_q_heads=7), dict(num_q_heads=0),
                   dict(softmax_scale=0.0), dict(softmax_scale=float("inf")),
                   dict(softmax_scale=float("nan")), dict(q=None), dict(out=None),
                   dict(block_table=None), dict(seq_lens=None), dict(q4_table=None),
                   dict(q4_cache=None), dict(max_blocks_per_seq=0),
                   dict(q4_cache=ctx.cache.data_ptr() + 8), dict(q=d.q.data_ptr() + 2),
                   dict(workspace=None), dict(workspace_bytes=d.need - 1)):
        refused(gcb.GC_ERR_INVALID_ARG, d, **change)
    refused(gcb.GC_ERR_OUT_OF_RANGE, d, layer=1)
    for change in (dict(tokens=5), dict(num_q_heads=24), dict(batch=8193),
                   dict(max_blocks_per_seq=2 ** 28), dict(softmax_scale=8193.0)):
        refused(gcb.GC_ERR_UNSUPPORTED, d, **change)
    d.run(batch=0, workspace=None, workspace_bytes=0)
    assert ctx.pool.check() == gcb.GC_OK
    assert np.isnan(d.out.double().cpu().numpy()).all()


def test_a_cache_without_pages():
    ctx = _q4.Context([100, 7], 2, 64, 16, recent=100)
    Decode(ctx, 4).run(q4_cache=None, n_q4_pages=0).check()
    assert ctx.pool.check() == gcb.GC_OK


@pytest.mark.parametrize("B", [1024, 1025, 8192])
@pytest.mark.parametrize("Hq,Hkv,d", [(1, 1, 64), (16, 1, 128), (8, 1, 128)])
def test_batches_around_the_room_for_the_warps_parts(B, Hq, Hkv, d):
    """Short contexts and a few long ones that are cut between warps and CTAs."""
    rng = np.random.default_rng(B)
    lens = rng.integers(1, 40, B)
    lens[[3, B // 2, B - 1]] = [3000, 7000, 900]
    ctx = _q4.Context(list(map(int, lens)), Hkv, d, 16, seed=B)
    dec = Decode(ctx, Hq).run()
    assert ctx.pool.check() == gcb.GC_OK
    # (the long ones, their neighbours and some more)
    keep = sorted({0, 2, 3, 4, B // 2 - 1, B // 2, B // 2 + 1, B - 2, B - 1, *range(7, B, B // 60)})
    dec.check(skip=(), only=keep)
    assert np.isfinite(dec.out.double().cpu().numpy()).all()


def test_units_of_more_keys():
    """A table so wide that its pairs' keys, 32 to a unit, could not be numbered in 32 bits."""
    import torch
    lens = [5000, 1, 40, 333] + [17 + i for i in range(60)]
    ctx = _q4.Context(lens, 8, 64, 16, recent=1, seed=14)
    d = Decode(ctx, 8)
    wide = 2 ** 24
    assert len(lens) * 8 * (wide * 16 // 32) > 2 ** 31
    tables = []
    for t in (ctx.dev4, ctx.dev16):
        w = torch.full((len(lens), wide), -1, dtype=torch.int32, device="cuda")
        w[:, :t.shape[1]] = t
        tables.append(w)
    need = gcb.gc_paged_decode_q4_workspace_bytes(ctx.pool.handle, len(lens), wide, 8, 1)
    assert need == d.need
    d.run(q4_table=tables[0], block_table=tables[1], max_blocks_per_seq=wide)
    assert ctx.pool.check() == gcb.GC_OK
    d.check()
