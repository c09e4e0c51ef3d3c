"""gc_prefix_prefill_attn_q4 is gc_kv_unpack_q4 and gc_prefix_prefill_attn, bit for bit,
without writing the pool; that pair is checked against 64 bits elsewhere."""
import numpy as np
import pytest

from paper_2505_23970_gb300 import binding as gcb
from paper_2505_23970_gb300 import workloads as wl
from paper_2505_23970_gb300.harness import _i32, bf16_tensor

from . import _q4
from ._span import assert_within

pytestmark = pytest.mark.gpu


class Prefill:
    def __init__(self, P, n, Hq, Hkv, d, ps, recent=0, seed=0, spare=0, **more):
        import torch
        self.P, self.n, self.Hq = P, n, Hq
        self.ctx = c = _q4.Context([p + m for p, m in zip(P, n)], Hkv, d, ps, recent=recent,
                                   seed=seed, **more)
        self.T = int(sum(n))
        self.q_bits = wl.normal_bf16(seed, 81, (self.T, Hq, d))
        self.q = bf16_tensor(self.q_bits)
        self.scale = d ** -0.5
        self.prefix, self.new = _i32(P, "cuda"), _i32(n, "cuda")
        self.cu_host = np.concatenate([[0], np.cumsum(n)])
        self.cu = _i32(self.cu_host, "cuda")
        self.out = torch.full((self.T, Hq, d), float("nan"), dtype=torch.bfloat16, device="cuda")
        self.need = gcb.gc_prefix_prefill_q4_workspace_bytes(c.pool.handle, len(P), c.width,
                                                             c.pages4)
        self.ws = torch.full((max(self.need, 16),), 0xFF, dtype=torch.uint8, device="cuda")

    def run(self, **change):
        c = self.ctx
        a = dict(q=self.q, pool=c.pool.handle, block_table=c.dev16, prefix_lens=self.prefix,
                 new_lens=self.new, out=self.out, stream=None, layer=c.layer, cu_new_lens=self.cu,
                 batch=len(self.P), max_blocks_per_seq=c.width, num_q_heads=self.Hq,
                 softmax_scale=self.scale, total_new_tokens=self.T, q4_cache=c.cache,
                 q4_table=c.dev4, n_q4_pages=c.pages4, workspace=self.ws,
                 workspace_bytes=self.need)
        gcb.gc_prefix_prefill_attn_q4(**{**a, **change})
        return self

    def both_calls(self):
        """The 4-bit pages read back behind the 16-bit ones of a larger pool, then the
        attention over them."""
        import torch
        c = self.ctx
        pool = gcb.KVPool.create(c.L, c.Hkv, c.d, c.ps, c.pages16 + c.pages4)
        pool.planes()[:, :, :c.pages16].copy_(c.pool.planes())
        ids = np.arange(c.pages4)
        gcb.gc_kv_unpack_q4(pool.handle, c.cache, c.pages4, _i32(ids, "cuda"),
                            _i32(ids + c.pages16, "cuda"), c.pages4, 0, c.L)
        table = np.where(c.table4 >= 0, c.table4 + c.pages16, c.table16)
        out = torch.full_like(self.out, float("nan"))
        gcb.gc_prefix_prefill_attn(self.q, pool.handle, _i32(table, "cuda"), self.prefix, self.new,
                                   out, None, c.layer, self.cu, len(self.P), c.width, self.Hq,
                                   self.scale, self.T)
        assert pool.check() == gcb.GC_OK
        return out


@pytest.mark.parametrize("recent", [0, 1])
@pytest.mark.parametrize("Hq,Hkv,d,ps,P,n", [
    (4, 1, 64, 16, [256], [64]),
    (8, 2, 64, 16, [300, 0, 5, 40], [64, 33, 1, 0]),
    (64, 8, 128, 16, [1000, 17, 0], [300, 1, 129]),
    (32, 8, 128, 64, [4000], [43]),
    (16, 1, 128, 128, [127, 128, 1], [2, 500, 3]),
    (32, 8, 64, 32, [700] * 9, [120] * 9),
])
def test_equals_reading_back_first(Hq, Hkv, d, ps, P, n, recent):
    import torch
    p = Prefill(P, n, Hq, Hkv, d, ps, recent=recent, seed=len(P) + d)
    before = p.ctx.pool.planes().clone()
    p.run()
    assert p.ctx.pool.check() == gcb.GC_OK
    assert torch.equal(p.out.view(torch.int16), p.both_calls().view(torch.int16))
    assert torch.equal(p.ctx.pool.planes().view(torch.int16), before.view(torch.int16))


def test_against_64_bits():
    """(The bound of tests/_span.py's docstring; the values are c s rounded to bf16.)"""
    import torch
    p = Prefill([200, 31], [100, 70], 16, 2, 128, 16, recent=1, seed=3)
    p.run()
    assert p.ctx.pool.check() == gcb.GC_OK
    for b in range(2):
        kv = p.ctx.keys(b)[0]
        kv = _q4.f32(wl.f32_to_bf16_bits(kv.astype(np.float32))).astype(np.float64)
        q = _q4.f32(p.q_bits[p.cu_host[b]:p.cu_host[b + 1]]).astype(np.float64)
        n, T = q.shape[0], kv.shape[1]
        s = np.einsum("ihgd,thd->ihgt", q.reshape(n, 2, 8, 128), kv[0]) * p.scale
        s = np.where(np.arange(T) <= (p.P[b] + np.arange(n))[:, None, None, None], s, -np.inf)
        w = np.exp(s - s.max(-1, keepdims=True))
        w /= w.sum(-1, keepdims=True)
        o = np.einsum("ihgt,thd->ihgd", w, kv[1]).reshape(n, 16, 128)
        a = np.einsum("ihgt,thd->ihgd", w, np.abs(kv[1])).reshape(n, 16, 128)
        bound = a * (2.0 ** -8 + 2.0 ** -11 + T * 2.0 ** -23) + np.abs(o) * 2.0 ** -8
        assert_within(p.out[p.cu_host[b]:p.cu_host[b + 1]].cpu(), torch.from_numpy(o),
                      torch.from_numpy(bound))


def test_scratch_by_page_and_by_position():
    """A wide table over few pages, and requests that share them."""
    import torch
    p = Prefill([300, 0], [20, 90], 8, 2, 128, 16, seed=5, width=1000)
    assert p.need == p.ctx.pages4 * 2 * 2 * 16 * 128 * 2
    p.run()
    assert p.ctx.pool.check() == gcb.GC_OK
    assert torch.equal(p.out.view(torch.int16), p.both_calls().view(torch.int16))
    # the second request's pages are the first one's
    c = p.ctx
    c.table4[1, :7] = c.table4[0, :7]
    c.dev4.copy_(_i32(c.table4, "cuda"))
    p.run()
    assert torch.equal(p.out.view(torch.int16), p.both_calls().view(torch.int16))


def test_layers_and_bad_entries():
    import torch
    p = Prefill([100, 60], [20, 9], 4, 2, 64, 16, seed=6, L=2, layer=1)
    p.run()
    assert p.ctx.pool.check() == gcb.GC_OK
    want = p.both_calls()
    assert torch.equal(p.out.view(torch.int16), want.view(torch.int16))
    t = p.ctx.table4.copy()
    t[0, 2] = p.ctx.pages4
    p.out.fill_(0)
    p.run(q4_table=_i32(t, "cuda"))
    assert p.ctx.pool.check() == gcb.GC_ERR_OUT_OF_RANGE
    assert torch.equal(p.out[20:].view(torch.int16), want[20:].view(torch.int16))


def test_a_cache_without_pages():
    import torch
    p = Prefill([100], [20], 4, 2, 64, 16, recent=100)
    p.run(q4_cache=None, n_q4_pages=0, workspace=None, workspace_bytes=0)
    assert p.ctx.pool.check() == gcb.GC_OK
    assert torch.equal(p.out.view(torch.int16), p.both_calls().view(torch.int16))


def test_refusals():
    p = Prefill([100], [20], 4, 2, 64, 16)
    for change in (dict(batch=-1), dict(n_q4_pages=-1), dict(q4_table=None), dict(q4_cache=None),
                   dict(q=None), dict(workspace=None), dict(workspace_bytes=p.need - 1),
                   dict(workspace=p.ws.data_ptr() + 8), dict(q4_cache=p.ctx.cache.data_ptr() + 8),
                   dict(num_q_heads=3), dict(softmax_scale=0.0), dict(max_blocks_per_seq=0)):
        with pytest.raises(gcb.GcError) as e:
            p.run(**change)
        assert e.value.status == gcb.GC_ERR_INVALID_ARG, change
    for status, change in ((gcb.GC_ERR_OUT_OF_RANGE, dict(layer=1)),
                           (gcb.GC_ERR_UNSUPPORTED, dict(num_q_heads=6)),
                           (gcb.GC_ERR_UNSUPPORTED, dict(batch=8192, max_blocks_per_seq=2 ** 19,
                                                         workspace_bytes=2 ** 62))):
        with pytest.raises(gcb.GcError) as e:
            p.run(**change)
        assert e.value.status == status, change
    p.run(batch=0)
    p.run(total_new_tokens=0)
    assert p.ctx.pool.check() == gcb.GC_OK
    assert np.isnan(p.out.double().cpu().numpy()).all()
