"""gc_paged_cross_attn against attention in 64 bits: lengths around pages and
tiles, requests without states or without new tokens, every head grouping, keys of
a call split over the GPU, large scores; what is skipped and refused."""
import numpy as np
import pytest

from paper_2505_23970_gb300 import binding as gcb
from paper_2505_23970_gb300 import workloads as wl
from paper_2505_23970_gb300.harness import _i32, bf16_bits, bf16_tensor

from ._span import Pages, assert_within, attend

pytestmark = pytest.mark.gpu


class Call:
    def __init__(self, Hq, Hkv, d, ps, kv, n, seed=0, scale_k=1.0, L=1, layer=0, reuse=None):
        import torch
        self.Hq, self.kv, self.n, self.d = Hq, kv, n, d
        self.pages = Pages(Hkv, d, ps, kv, seed=seed, scale_k=scale_k, L=L, layer=layer, reuse=reuse)
        self.T = sum(n)
        self.cu = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
        self.q_bits = wl.normal_bf16(seed, 33, (self.T, Hq, d))
        self.q = bf16_tensor(self.q_bits)
        self.out = torch.full((self.T, Hq, d), float("nan"), dtype=torch.bfloat16, device="cuda")
        self.table = self.pages.dev_tables[0]
        self.dev = [_i32(x, "cuda") for x in (kv, n, self.cu)]
        self.scale = d ** -0.5
        self.pool = self.pages.pool

    def run(self, stream=None, **change):
        import torch
        need = gcb.gc_paged_cross_workspace_bytes(self.pool.handle, len(self.n),
                                                  self.table.shape[1], self.Hq, self.T)
        self.need = need
        self.ws = torch.full((max(need, 16),), 255, dtype=torch.uint8, device="cuda")
        a = dict(q=self.q, pool=self.pool.handle, block_table=self.table, kv_lens=self.dev[0],
                 new_lens=self.dev[1], out=self.out, stream=stream, layer=self.pages.layer,
                 cu_new_lens=self.dev[2], batch=len(self.n),
                 max_blocks_per_seq=self.table.shape[1], num_q_heads=self.Hq,
                 softmax_scale=self.scale, total_new_tokens=self.T, workspace=self.ws,
                 workspace_bytes=need)
        gcb.gc_paged_cross_attn(**{**a, **change})

    def check(self, skipped=()):
        import torch
        for b, (kv, n) in enumerate(zip(self.kv, self.n)):
            got = self.out[self.cu[b]:self.cu[b + 1]]
            if b in skipped:
                assert torch.isnan(got).all(), b
                continue
            if n == 0:
                continue
            q = self.q[self.cu[b]:self.cu[b + 1]].double()
            want, bound = attend(q, self.pages.keys(0, b, kv), self.scale)
            assert_within(got, want, bound, f"request {b} ({kv} states, {n} tokens)")


EDGES = [1, 2, 15, 16, 17, 127, 128, 129, 255, 256, 257]
CASES = {
    "one-of-one-d64": (1, 1, 64, 16, [1], [1]),
    "one-of-one-d128": (1, 1, 128, 16, [1], [1]),
    "edges-d64": (4, 1, 64, 16, EDGES, [3, 1, 64, 65, 31, 2, 63, 1, 17, 32, 33]),
    "edges-d128": (4, 1, 128, 16, EDGES, [3, 1, 64, 65, 31, 2, 63, 1, 17, 32, 33]),
    "no-states-d64": (8, 2, 64, 32, [0, 40, 0, 300, 0], [5, 1, 0, 70, 300]),
    "no-states-d128": (8, 2, 128, 32, [0, 40, 0, 300, 0], [5, 1, 0, 70, 300]),
    "none-at-all-d64": (2, 2, 64, 16, [0, 0], [3, 40]),
    "none-at-all-d128": (2, 2, 128, 16, [0, 0], [3, 40]),
    "g2-ps64": (6, 3, 128, 64, [500, 65, 1000], [130, 129, 1]),
    "g16-ps128": (32, 2, 128, 128, [385, 130, 1], [17, 33, 16]),
    "g16-d64": (16, 1, 64, 64, [385, 130, 1], [17, 33, 16]),
    "g8": (64, 8, 128, 16, [700, 12, 0, 333], [40, 3, 9, 65]),
    "single-tokens": (32, 8, 128, 16, [100, 1, 900, 17, 1300, 0], [1] * 6),
    "single-tokens-d64": (32, 8, 64, 16, [100, 1, 900, 17, 1300, 0], [1] * 6),
    "many-requests": (4, 2, 128, 16, [i % 70 for i in range(700)], [i % 5 for i in range(700)]),
    "many-requests-d64": (4, 2, 64, 16, [i % 70 for i in range(700)], [i % 5 for i in range(700)]),
}


@pytest.mark.parametrize("name", list(CASES))
def test_against_64_bits(name):
    c = Call(*CASES[name], seed=len(name))
    c.run()
    assert c.pool.check() == gcb.GC_OK
    c.check()


@pytest.mark.parametrize("Hq,Hkv,d,ps,kv,n", [
    (8, 1, 128, 16, [20000], [5]),          # few rows: the keys are split
    (64, 8, 128, 64, [9000, 300], [43, 2]),
    (4, 1, 64, 16, [20011], [7]),
    (8, 2, 64, 32, [5000, 129, 12345], [3, 60, 1]),
    (8, 8, 128, 32, [3000, 0, 2500], [300, 40, 700]),  # several row tiles
    (16, 4, 64, 16, [3000, 0, 2500], [300, 40, 700]),
    (32, 8, 128, 16, [400] * 24, [120] * 24),   # more work items than SM pairs
    (32, 8, 64, 16, [400] * 24, [120] * 24),
])
def test_long_and_wide(Hq, Hkv, d, ps, kv, n):
    c = Call(Hq, Hkv, d, ps, kv, n, seed=d + Hq, reuse=64)
    c.run()
    assert c.pool.check() == gcb.GC_OK
    c.check()


@pytest.mark.parametrize("d", [64, 128])
def test_scores_that_jump(d):
    """Later keys hundreds above the first ones: the reference maximum moves, and
    all but a few keys have no weight."""
    import torch
    c = Call(4, 2, d, 16, [1000, 300], [40, 150], seed=4)
    planes = c.pool.planes()[0]
    for b, at in ((0, 700), (0, 910), (1, 290)):
        page = int(c.pages.tables[0][b, at // 16])
        for view in (planes[0], c.pages.values[0]):
            view[page, :, at % 16] *= 100 if at != 910 else 200
    c.run()
    assert c.pool.check() == gcb.GC_OK
    # scores of size 10^3 carry 2^-24 * 128 * 10^3 < 2^-6 in binary32 where two keys
    # compete; the rows are compared where one key has nearly all of the weight
    for b in range(2):
        q = c.q[c.cu[b]:c.cu[b + 1]].double()
        kv = c.pages.keys(0, b, c.kv[b])
        s = torch.einsum("nhgd,thd->nhgt", q.view(-1, 2, 2, d), kv[0]) * c.scale
        top = s.topk(2, -1).values
        sure = (top[..., 0] - top[..., 1] > 20).reshape(-1, 4)
        assert sure.float().mean() > 0.3
        want, bound = attend(q, kv, c.scale)
        got = c.out[c.cu[b]:c.cu[b + 1]]
        assert_within(got[sure], want[sure], bound[sure], f"request {b}")
        assert torch.isfinite(got).all()


@pytest.mark.parametrize("d", [64, 128])
def test_same_bits_again_and_on_another_stream(d):
    import torch
    c = Call(8, 1, d, 16, [5000, 77], [9, 30], seed=6, L=3, layer=2, reuse=64)
    c.run()
    first = bf16_bits(c.out)
    s = torch.cuda.Stream()
    c.out.fill_(float("nan"))
    s.wait_stream(torch.cuda.current_stream())
    c.run(stream=s)
    assert c.pool.check(s) == gcb.GC_OK
    assert np.array_equal(bf16_bits(c.out), first)
    c.check()


def test_recorded_in_a_graph():
    import torch
    c = Call(8, 2, 128, 16, [900, 33], [3, 40], seed=7)
    s = torch.cuda.Stream()
    c.run()
    torch.cuda.synchronize()
    c.out.fill_(float("nan"))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        c.run(stream=torch.cuda.current_stream(), workspace=c.ws)
    g.replay()
    torch.cuda.synchronize()
    assert c.pool.check() == gcb.GC_OK
    c.check()


@pytest.mark.parametrize("d", [64, 128])
def test_bad_lengths_and_rows_are_skipped_and_recorded(d):
    c = Call(4, 1, d, 16, [40, 33, 100], [5, 6, 7], seed=1)
    c.dev[0][1] = 7 * 16 + 1  # past the table's capacity
    c.run()
    assert c.pool.check() == gcb.GC_ERR_OUT_OF_RANGE
    c.check(skipped=(1,))
    c = Call(4, 1, d, 16, [40, 33, 100], [5, 6, 7], seed=1)
    c.dev[0][0] = -1
    c.run()
    assert c.pool.check() == gcb.GC_ERR_OUT_OF_RANGE
    c.check(skipped=(0,))
    c = Call(4, 1, d, 16, [40, 33, 100], [5, 6, 7], seed=1)
    c.run(total_new_tokens=c.T - 1)  # the last request's rows would pass it
    assert c.pool.check() == gcb.GC_ERR_OUT_OF_RANGE
    c.check(skipped=(2,))


@pytest.mark.parametrize("d", [64, 128])
def test_a_bad_page_is_recorded_and_harms_no_other_request(d):
    import torch
    c = Call(4, 1, d, 16, [40, 33, 100], [5, 6, 7], seed=2)
    c.table[1, 1] = c.pages.num_pages
    c.run()
    assert c.pool.check() == gcb.GC_ERR_OUT_OF_RANGE
    c.out[c.cu[1]:c.cu[2]] = float("nan")
    c.check(skipped=(1,))


def test_nothing_to_do():
    import torch
    c = Call(4, 1, 64, 16, [40], [5])
    c.run(batch=0, q=None)
    c.run(total_new_tokens=0, q=None)
    assert c.pool.check() == gcb.GC_OK
    assert torch.isnan(c.out).all()


@pytest.mark.parametrize("status,change", [
    (gcb.GC_ERR_INVALID_ARG, dict(pool=None)),
    (gcb.GC_ERR_INVALID_ARG, dict(batch=-1)),
    (gcb.GC_ERR_INVALID_ARG, dict(total_new_tokens=-1)),
    (gcb.GC_ERR_INVALID_ARG, dict(max_blocks_per_seq=-1)),
    (gcb.GC_ERR_INVALID_ARG, dict(max_blocks_per_seq=0)),
    (gcb.GC_ERR_OUT_OF_RANGE, dict(layer=1)),
    (gcb.GC_ERR_OUT_OF_RANGE, dict(layer=-1)),
    (gcb.GC_ERR_INVALID_ARG, dict(num_q_heads=7)),
    (gcb.GC_ERR_INVALID_ARG, dict(num_q_heads=0)),
    (gcb.GC_ERR_UNSUPPORTED, dict(num_q_heads=6)),
    (gcb.GC_ERR_UNSUPPORTED, dict(num_q_heads=64)),
    (gcb.GC_ERR_UNSUPPORTED, dict(batch=8193)),
    (gcb.GC_ERR_UNSUPPORTED, dict(max_blocks_per_seq=1 << 28)),
    (gcb.GC_ERR_INVALID_ARG, dict(softmax_scale=0.0)),
    (gcb.GC_ERR_INVALID_ARG, dict(softmax_scale=float("nan"))),
    (gcb.GC_ERR_INVALID_ARG, dict(softmax_scale=float("inf"))),
    (gcb.GC_ERR_INVALID_ARG, dict(q=None)),
    (gcb.GC_ERR_INVALID_ARG, dict(out=None)),
    (gcb.GC_ERR_INVALID_ARG, dict(block_table=None)),
    (gcb.GC_ERR_INVALID_ARG, dict(kv_lens=None)),
    (gcb.GC_ERR_INVALID_ARG, dict(new_lens=None)),
    (gcb.GC_ERR_INVALID_ARG, dict(cu_new_lens=None)),
    (gcb.GC_ERR_INVALID_ARG, dict(q=4104)),
    (gcb.GC_ERR_INVALID_ARG, dict(workspace=4104)),
])
def test_refusals(status, change):
    import torch
    c = Call(4, 2, 64, 16, [40, 33], [5, 6])
    with pytest.raises(gcb.GcError) as e:
        c.run(**change)
    assert e.value.status == status
    assert "gc_paged_cross_attn: " in str(e.value)
    assert c.pool.check() == gcb.GC_OK
    assert torch.isnan(c.out).all()


def test_a_short_workspace_is_refused():
    import torch
    for d in (64, 128):
        c = Call(8, 1, d, 16, [20000], [5], reuse=64)
        c.run()
        if c.need == 0:
            continue
        for change in (dict(workspace_bytes=c.need - 1), dict(workspace=None)):
            c.out.fill_(float("nan"))
            with pytest.raises(gcb.GcError) as e:
                c.run(**change)
            assert e.value.status == gcb.GC_ERR_INVALID_ARG
            assert c.pool.check() == gcb.GC_OK
            assert torch.isnan(c.out).all()
