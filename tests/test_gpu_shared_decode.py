"""gc_shared_prefix_decode_attn against attention in 64 bits over the shared keys
followed by the own ones: groups of every size, empty ones too, shared and own
lengths of 0, 1 and around pages and tiles, every head grouping; the same as
gc_paged_decode_attn over joined tables; what is skipped and refused."""
import numpy as np
import pytest

from paper_2505_23970_gb300 import binding as gcb
from paper_2505_23970_gb300 import workloads as wl
from paper_2505_23970_gb300.harness import _i32, bf16_bits, bf16_tensor

from ._span import Pages, assert_within, attend

pytestmark = pytest.mark.gpu


class Call:
    def __init__(self, Hq, Hkv, d, ps, sizes, S, own, seed=0, L=1, layer=0, reuse=None):
        import torch
        assert sum(sizes) == len(own) and len(sizes) == len(S)
        self.Hq, self.S, self.own, self.d = Hq, S, own, d
        self.pages = Pages(Hkv, d, ps, S, own, seed=seed, L=L, layer=layer, reuse=reuse)
        self.B = len(own)
        self.cu = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
        self.group = np.repeat(np.arange(len(sizes)), sizes)
        self.q = bf16_tensor(wl.normal_bf16(seed, 33, (self.B, Hq, d)))
        self.out = torch.full((self.B, Hq, d), float("nan"), dtype=torch.bfloat16, device="cuda")
        self.stable, self.table = self.pages.dev_tables
        self.dev = [_i32(x, "cuda") for x in (S, self.cu, own)]
        self.scale = d ** -0.5
        self.pool = self.pages.pool

    def run(self, stream=None, **change):
        import torch
        need = gcb.gc_shared_prefix_decode_workspace_bytes(
            self.pool.handle, self.B, len(self.S), self.stable.shape[1], self.table.shape[1],
            self.Hq)
        self.need = need
        self.ws = torch.full((max(need, 16),), 255, dtype=torch.uint8, device="cuda")
        a = dict(q=self.q, pool=self.pool.handle, shared_table=self.stable,
                 shared_lens=self.dev[0], cu_requests=self.dev[1], num_groups=len(self.S),
                 max_shared_blocks=self.stable.shape[1], block_table=self.table,
                 seq_lens=self.dev[2], out=self.out, stream=stream, layer=self.pages.layer,
                 batch=self.B, max_blocks_per_seq=self.table.shape[1], num_q_heads=self.Hq,
                 softmax_scale=self.scale, workspace=self.ws, workspace_bytes=need)
        gcb.gc_shared_prefix_decode_attn(**{**a, **change})

    def check(self, skipped=()):
        import torch
        for b in range(self.B):
            got = self.out[b:b + 1]
            if b in skipped:
                assert torch.isnan(got).all(), b
                continue
            s = int(self.group[b])
            kv = torch.cat([self.pages.keys(0, s, self.S[s]),
                            self.pages.keys(1, b, self.own[b])], 1)
            want, bound = attend(self.q[b:b + 1].double(), kv, self.scale)
            assert_within(got, want, bound, f"request {b} ({self.S[s]} + {self.own[b]} keys)")


EDGES = [0, 1, 15, 16, 17, 127, 128, 129, 255, 256, 257]
CASES = {
    "one-d64": (1, 1, 64, 16, [1], [1], [1]),
    "one-d128": (1, 1, 128, 16, [1], [1], [1]),
    "shared-edges-d64": (4, 1, 64, 16, [1, 2, 3] * 3 + [1, 1], EDGES, [1 + 7 * i for i in range(20)]),
    "shared-edges-d128": (4, 1, 128, 16, [1, 2, 3] * 3 + [1, 1], EDGES,
                          [1 + 7 * i for i in range(20)]),
    "own-edges-d64": (8, 2, 64, 32, [11], [300], EDGES),
    "own-edges-d128": (8, 2, 128, 32, [11], [300], EDGES),
    "no-prefix-d64": (4, 2, 64, 16, [3, 2], [0, 0], [5, 0, 40, 300, 1]),
    "no-prefix-d128": (4, 2, 128, 16, [3, 2], [0, 0], [5, 0, 40, 300, 1]),
    "nothing-own-d64": (4, 2, 64, 16, [3, 2, 1], [40, 1, 0], [0] * 6),
    "nothing-own-d128": (4, 2, 128, 16, [3, 2, 1], [40, 1, 0], [0] * 6),
    "empty-groups": (8, 1, 128, 16, [0, 3, 0, 0, 2, 0], [9, 77, 0, 5, 200, 31], [1, 2, 3, 4, 50]),
    "empty-groups-d64": (8, 1, 64, 16, [0, 3, 0, 0, 2, 0], [9, 77, 0, 5, 200, 31], [1, 2, 3, 4, 50]),
    "rows-past-a-tile": (8, 2, 128, 16, [70], [500], [1 + i % 90 for i in range(70)]),
    "rows-past-a-tile-d64": (16, 1, 64, 16, [70], [500], [1 + i % 90 for i in range(70)]),
    "g1": (3, 3, 128, 64, [150, 130], [200, 131], [1 + i % 33 for i in range(280)]),
    "g2-d64": (6, 3, 64, 64, [150, 130], [200, 131], [1 + i % 33 for i in range(280)]),
    "g16": (32, 2, 128, 128, [17, 16, 1], [385, 130, 1], [1 + 13 * i for i in range(34)]),
    "llama-shape": (64, 8, 128, 16, [8, 5], [700, 333], [3 + 31 * i for i in range(13)]),
    "many-groups": (4, 2, 128, 16, [1] * 600, [i % 40 for i in range(600)], [i % 30 for i in range(600)]),
    "many-groups-d64": (4, 2, 64, 16, [1] * 600, [i % 40 for i in range(600)],
                        [i % 30 for i in range(600)]),
    "many-short": (8, 8, 128, 16, [200], [64], [1 + i % 250 for i in range(200)]),
    "many-short-d64": (8, 8, 64, 16, [200], [64], [1 + i % 250 for i in range(200)]),
}


@pytest.mark.parametrize("name", list(CASES))
def test_against_64_bits(name):
    c = Call(*CASES[name], seed=len(name))
    c.run()
    assert c.pool.check() == gcb.GC_OK
    c.check()


@pytest.mark.parametrize("Hq,Hkv,d,ps,sizes,S,own", [
    (8, 1, 128, 16, [5], [20000], [700, 1, 3000, 17, 256]),
    (64, 8, 128, 64, [9, 3], [9000, 4500], [1 + 211 * i for i in range(12)]),
    (4, 1, 64, 16, [5], [20011], [700, 1, 5000, 17, 256]),
    (8, 2, 64, 32, [3, 60, 1], [5000, 129, 12345], [1 + 37 * i for i in range(64)]),
    (32, 8, 128, 16, [90], [3000], [1 + i % 400 for i in range(90)]),
    (16, 4, 64, 128, [90], [3000], [1 + i % 400 for i in range(90)]),
    (16, 16, 128, 16, [20, 30], [1500, 40], [1 + 19 * i for i in range(50)]),
    (32, 8, 128, 32, [2] * 40, [130 + 17 * i for i in range(40)], [1 + 5 * i for i in range(80)]),
])
def test_long_and_wide(Hq, Hkv, d, ps, sizes, S, own):
    c = Call(Hq, Hkv, d, ps, sizes, S, own, seed=d + Hq, reuse=64)
    c.run()
    assert c.pool.check() == gcb.GC_OK
    c.check()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("where", ["shared", "own"])
def test_one_side_outweighs_the_other(d, where):
    """Scores of one side hundreds above the other's: the join must not lose the
    larger side or overflow on the smaller."""
    import torch
    c = Call(4, 2, d, 16, [3], [300], [40, 1, 200], seed=4)
    planes = c.pool.planes()[0]
    lists = [(0, 0, 211)] if where == "shared" else [(1, 0, 33), (1, 1, 0), (1, 2, 150)]
    for which, row, at in lists:
        page = int(c.pages.tables[which][row, at // 16])
        for view in (planes[0], c.pages.values[0]):
            view[page, :, at % 16] *= 150
    c.run()
    assert c.pool.check() == gcb.GC_OK
    sure_rows = 0
    for b in range(3):
        kv = torch.cat([c.pages.keys(0, 0, 300), c.pages.keys(1, b, c.own[b])], 1)
        q = c.q[b:b + 1].double()
        top = (torch.einsum("nhgd,thd->nhgt", q.view(1, 2, 2, d), kv[0]) * c.scale).topk(2, -1).values
        sure = (top[..., 0] - top[..., 1] > 20).reshape(1, 4)
        sure_rows += int(sure.sum())
        want, bound = attend(q, kv, c.scale)
        assert torch.isfinite(c.out[b]).all()
        assert_within(c.out[b:b + 1][sure], want[sure], bound[sure], f"request {b}")
    assert sure_rows >= 3


@pytest.mark.parametrize("Hq,Hkv,d,ps", [(8, 2, 128, 16), (4, 1, 64, 32)])
def test_equals_decode_over_joined_tables(Hq, Hkv, d, ps):
    import torch
    S = [ps * 20, 0, ps * 3]
    own = [1, 50, 300, 7, 90, 33]
    c = Call(Hq, Hkv, d, ps, [3, 1, 2], S, own, seed=9)
    c.run()
    width = max(-(-(S[g] + n) // ps) for g, n in zip(c.group, own))
    joined = np.full((6, width), -1, np.int32)
    for b, g in enumerate(c.group):
        k, m = S[g] // ps, -(-own[b] // ps)
        joined[b, :k] = c.pages.tables[0][g, :k]
        joined[b, k:k + m] = c.pages.tables[1][b, :m]
    out = torch.empty_like(c.out)
    need = gcb.gc_paged_decode_workspace_bytes(c.pool.handle, 6, width, Hq)
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    gcb.gc_paged_decode_attn(c.q, c.pool.handle, _i32(joined, "cuda"),
                             _i32([S[g] + n for g, n in zip(c.group, own)], "cuda"), out, None, 0,
                             6, width, Hq, c.scale, ws, need)
    assert c.pool.check() == gcb.GC_OK
    c.check()
    first = c.out.clone()
    c.out.copy_(out)
    c.check()
    rel = (first.double() - out.double()).norm() / out.double().norm()
    assert rel <= 1e-2


@pytest.mark.parametrize("d", [64, 128])
def test_same_bits_again_and_on_another_stream(d):
    import torch
    c = Call(8, 1, d, 16, [3, 4], [5000, 77], [9, 30, 700, 1, 2, 3, 4], seed=6, L=3, layer=2,
             reuse=64)
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
    c = Call(8, 2, 128, 16, [3, 2], [900, 33], [3, 40, 1, 500, 9], seed=7)
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


def test_other_calls_on_the_pool_before_and_after():
    """The counters in the pool's control block are as the other calls want them."""
    import torch
    c = Call(8, 1, 128, 16, [3, 4], [5000, 77], [900, 30, 700, 1, 2, 3, 4], seed=6, reuse=64)
    need = gcb.gc_paged_decode_workspace_bytes(c.pool.handle, c.B, c.table.shape[1], 8)
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")

    def decode():
        out = torch.empty_like(c.out)
        gcb.gc_paged_decode_attn(c.q, c.pool.handle, c.table, c.dev[2], out, None, 0, c.B,
                                 c.table.shape[1], 8, c.scale, ws, need)
        return bf16_bits(out)
    before = decode()
    for _ in range(3):
        c.run()
        assert np.array_equal(decode(), before)
    assert c.pool.check() == gcb.GC_OK
    c.check()


@pytest.mark.parametrize("d", [64, 128])
def test_bad_lengths_are_skipped_and_recorded(d):
    def call():
        return Call(4, 1, d, 16, [2, 3, 1], [40, 100, 7], [5, 6, 7, 33, 1, 20], seed=1)
    c = call()
    c.dev[2][3] = 3 * 16 + 1  # own length past its table
    c.dev[2][0] = -1
    c.run()
    assert c.pool.check() == gcb.GC_ERR_OUT_OF_RANGE
    c.check(skipped=(0, 3))
    for bad in (7 * 16 + 1, -1):
        c = call()
        c.dev[0][1] = bad  # a shared length out of range: all of its group
        c.run()
        assert c.pool.check() == gcb.GC_ERR_OUT_OF_RANGE
        c.check(skipped=(2, 3, 4))


@pytest.mark.parametrize("d", [64, 128])
def test_requests_without_a_group_are_skipped_and_recorded(d):
    c = Call(4, 1, d, 16, [2, 3, 1], [40, 100, 7], [5, 6, 7, 33, 1, 20], seed=1)
    c.dev[1][3] = 5
    c.run()
    assert c.pool.check() == gcb.GC_ERR_OUT_OF_RANGE
    c.check(skipped=(5,))
    c = Call(4, 1, d, 16, [2, 3, 1], [40, 100, 7], [5, 6, 7, 33, 1, 20], seed=1)
    c.dev[1][0] = 1
    c.run()
    assert c.pool.check() == gcb.GC_ERR_OUT_OF_RANGE
    c.check(skipped=(0,))
    c = Call(4, 1, d, 16, [2, 3, 1], [40, 100, 7], [5, 6, 7, 33, 1, 20], seed=1)
    c.dev[1][3] = 7  # a group that passes the batch
    c.run()
    assert c.pool.check() == gcb.GC_ERR_OUT_OF_RANGE
    c.check(skipped=(5,))


@pytest.mark.parametrize("d", [64, 128])
def test_a_bad_page_is_recorded_and_harms_no_other(d):
    c = Call(4, 1, d, 16, [2, 3, 1], [40, 100, 7], [5, 6, 7, 33, 1, 20], seed=2)
    c.stable[1, 2] = c.pages.num_pages
    c.table[5, 0] = -1
    c.run()
    assert c.pool.check() == gcb.GC_ERR_OUT_OF_RANGE
    c.out[2:] = float("nan")
    c.check(skipped=(2, 3, 4, 5))


def test_nothing_to_do():
    import torch
    c = Call(4, 1, 64, 16, [1], [40], [5])
    c.run(batch=0, q=None)
    assert c.pool.check() == gcb.GC_OK
    assert torch.isnan(c.out).all()


@pytest.mark.parametrize("status,change", [
    (gcb.GC_ERR_INVALID_ARG, dict(pool=None)),
    (gcb.GC_ERR_INVALID_ARG, dict(batch=-1)),
    (gcb.GC_ERR_INVALID_ARG, dict(num_groups=-1)),
    (gcb.GC_ERR_INVALID_ARG, dict(num_groups=0)),
    (gcb.GC_ERR_INVALID_ARG, dict(max_blocks_per_seq=0)),
    (gcb.GC_ERR_INVALID_ARG, dict(max_shared_blocks=0)),
    (gcb.GC_ERR_INVALID_ARG, dict(max_shared_blocks=-3)),
    (gcb.GC_ERR_OUT_OF_RANGE, dict(layer=1)),
    (gcb.GC_ERR_INVALID_ARG, dict(num_q_heads=7)),
    (gcb.GC_ERR_UNSUPPORTED, dict(num_q_heads=6)),
    (gcb.GC_ERR_UNSUPPORTED, dict(batch=8193)),
    (gcb.GC_ERR_UNSUPPORTED, dict(num_groups=8193)),
    (gcb.GC_ERR_UNSUPPORTED, dict(max_blocks_per_seq=1 << 28)),
    (gcb.GC_ERR_UNSUPPORTED, dict(max_shared_blocks=1 << 28)),
    (gcb.GC_ERR_INVALID_ARG, dict(softmax_scale=-1.0)),
    (gcb.GC_ERR_INVALID_ARG, dict(q=None)),
    (gcb.GC_ERR_INVALID_ARG, dict(out=None)),
    (gcb.GC_ERR_INVALID_ARG, dict(shared_table=None)),
    (gcb.GC_ERR_INVALID_ARG, dict(shared_lens=None)),
    (gcb.GC_ERR_INVALID_ARG, dict(cu_requests=None)),
    (gcb.GC_ERR_INVALID_ARG, dict(block_table=None)),
    (gcb.GC_ERR_INVALID_ARG, dict(seq_lens=None)),
    (gcb.GC_ERR_INVALID_ARG, dict(out=4104)),
    (gcb.GC_ERR_INVALID_ARG, dict(workspace=4104)),
])
def test_refusals(status, change):
    import torch
    c = Call(4, 2, 64, 16, [1, 1], [40, 33], [5, 6])
    with pytest.raises(gcb.GcError) as e:
        c.run(**change)
    assert e.value.status == status
    assert "gc_shared_prefix_decode_attn: " in str(e.value)
    assert c.pool.check() == gcb.GC_OK
    assert torch.isnan(c.out).all()


def test_a_short_workspace_is_refused():
    import torch
    for d in (64, 128):
        c = Call(8, 1, d, 16, [2], [20000], [700, 3000], reuse=64)
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
