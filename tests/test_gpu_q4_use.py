"""The 4-bit cache as a serving loop uses it: contexts loaded and packed, new tokens
prefilled, tokens and drafted tokens generated through the layers, against the same
steps in 64 bits on the values that the cache should hold; a captured step; streams."""
import numpy as np
import pytest

from paper_2505_23970_gb300 import binding as gcb
from paper_2505_23970_gb300 import workloads as wl
from paper_2505_23970_gb300.harness import FourBitContext, _i32, bf16_bits, bf16_tensor

from . import _q4

pytestmark = pytest.mark.gpu


class Mirror:
    """What every request's 4-bit rows should hold: values and scales [L][2][T][Hkv][.]."""

    def __init__(self, c):
        self.c = c
        shape = (c.L, 2, c.B, c.width * c.ps, c.Hkv)
        self.v, self.s = np.zeros((*shape, c.d)), np.zeros((*shape, c.d // 32))
        self.lens = np.zeros(c.B, int)

    def put(self, layer, plane, b, at, bits):
        """bits [n][Hkv][d] at slots at..."""
        self.v[layer, plane, b, at:at + len(bits)] = _q4.values(bits)
        self.s[layer, plane, b, at:at + len(bits)] = _q4.f32(_q4.quantise(bits)[1])

    def turned(self, bits, pos):
        rot, half = self.c.rot_dim, self.c.rot_dim // 2
        x = _q4.f32(bits).astype(np.float64)
        cs = self.c.cos_sin.cpu().numpy().astype(np.float64)[pos]
        cos, sin = cs[:, 0, None], cs[:, 1, None]
        r32 = lambda y: y.astype(np.float32).astype(np.float64)
        a, b = x[..., :half].copy(), x[..., half:rot].copy()
        x[..., :half] = a * cos - r32(b * sin)
        x[..., half:rot] = b * cos + r32(a * sin)
        return wl.f32_to_bf16_bits(x.astype(np.float32))

    def append(self, layer, rows, n):
        """The rows' rotated q bits, after k and v have gone to their slots."""
        c, at, q = self.c, 0, []
        for b in range(c.B):
            pos = self.lens[b] + np.arange(n[b])
            r = rows[at:at + n[b]]
            q.append(self.turned(r[:, :c.Hq], pos))
            self.put(layer, 0, b, self.lens[b], self.turned(r[:, c.Hq:c.Hq + c.Hkv], pos))
            self.put(layer, 1, b, self.lens[b], r[:, c.Hq + c.Hkv:])
            at += n[b]
        return q

    def check(self, layer, q, out, n, wide):
        """Attention of the n[b] last tokens of each request; wide: over values rounded to
        bf16 (prefill)."""
        c, at = self.c, 0
        got = out.double().cpu().numpy()
        for b in range(c.B):
            if n[b] == 0:
                continue
            T = self.lens[b] + n[b]
            v, s = self.v[layer, :, b, :T], self.s[layer, :, b, :T]
            if wide:
                v = _q4.f32(wl.f32_to_bf16_bits(v.astype(np.float32))).astype(np.float64)
            want, bound = _q4.decode_reference(_q4.f32(q[b]).astype(np.float64), v, s,
                                               c.d ** -0.5, n[b])
            g = got[at:at + n[b]]
            assert np.isfinite(g).all()
            assert (np.abs(g - want) <= bound).all(), (layer, b, np.abs(g - want).max())
            at += n[b]


@pytest.mark.parametrize("Hq,Hkv,d,ps,tokens,rot", [
    (16, 2, 128, 16, 1, None), (8, 2, 64, 32, 4, 32), (8, 4, 128, 16, 3, 64),
    (16, 1, 64, 16, 1, None), (4, 4, 64, 64, 2, 0)])
def test_a_serving_loop(Hq, Hkv, d, ps, tokens, rot):
    import torch
    L, B = 2, 3
    c = FourBitContext(Hq, Hkv, d, ps, B, 400, tokens, rot, L=L, staging_pages=3, seed=d + Hq)
    m = Mirror(c)
    c.cache.fill_(0xFF)  # scales of NaN wherever nothing is written
    # cached contexts of 5, 0 and 2 pages
    blocks = [5, 0, 2]
    req = np.repeat(np.arange(B), blocks)
    blk = np.concatenate([np.arange(n) for n in blocks])
    image = wl.normal_bf16(d, 3, (7, L, 2, Hkv, ps, d))
    c.load(bf16_tensor(image), req, blk)
    c.advance(_i32(np.array(blocks) * ps, "cuda"))
    for i, (b, j) in enumerate(zip(req, blk)):
        for layer in range(L):
            for p in range(2):
                m.put(layer, p, b, j * ps, image[i, layer, p].transpose(1, 0, 2))
    m.lens += np.array(blocks) * ps
    # a question each, of 20, 33 and 0 tokens
    n = [20, 33, 0]
    c.begin(n)
    for layer in range(L):
        rows = wl.normal_bf16(d, 10 + layer, (sum(n), Hq + 2 * Hkv, d))
        out = torch.full((sum(n), Hq, d), float("nan"), dtype=torch.bfloat16, device="cuda")
        c.prefill(bf16_tensor(rows), out, layer)
        q = m.append(layer, rows, n)
        assert np.array_equal(bf16_bits(c._new[3]), np.concatenate(q))
        m.check(layer, q, out, n, True)
    c.advance(_i32(n, "cuda"))
    m.lens += np.array(n)
    # answers: of a step's tokens one request keeps all, the others fewer
    for t in range(4):
        for layer in range(L):
            rows = wl.normal_bf16(d + 7 * t, 20 + layer, (B * tokens, Hq + 2 * Hkv, d))
            out = torch.full((B * tokens, Hq, d), float("nan"), dtype=torch.bfloat16,
                             device="cuda")
            c.step(bf16_tensor(rows), out, layer)
            q = m.append(layer, rows, [tokens] * B)
            assert np.array_equal(bf16_bits(c.q), np.concatenate(q))
            m.check(layer, q, out, [tokens] * B, False)
        kept = np.array([tokens, 1 + t % tokens, 1])
        c.advance(_i32(kept, "cuda"))
        m.lens += kept
    assert c.check() == gcb.GC_OK


@pytest.mark.parametrize("d,tokens", [(64, 1), (128, 2)])
def test_a_captured_step(d, tokens):
    """A step of two layers and its advance, replayed: the same bits as one by one."""
    import torch
    Hq, Hkv, ps, B, L = 8, 2, 16, 4, 2
    ctx = [FourBitContext(Hq, Hkv, d, ps, B, 600, tokens, L=L, seed=3) for _ in range(2)]
    start = [300, 0, 17, 250]
    rows0 = bf16_tensor(wl.normal_bf16(d, 1, (sum(start), Hq + 2 * Hkv, d)))
    for c in ctx:
        c.begin(start)
        for layer in range(L):
            c.prefill(rows0, torch.empty((sum(start), Hq, d), dtype=torch.bfloat16, device="cuda"),
                      layer)
        c.advance(_i32(start, "cuda"))
    rows = torch.empty((L, B * tokens, Hq + 2 * Hkv, d), dtype=torch.bfloat16, device="cuda")
    outs = [torch.empty((L, B * tokens, Hq, d), dtype=torch.bfloat16, device="cuda") for _ in ctx]

    def one(i, stream=None):
        for layer in range(L):
            ctx[i].step(rows[layer], outs[i][layer], layer, stream)
        ctx[i].advance(tokens)

    def new(t):
        rows.copy_(bf16_tensor(wl.normal_bf16(d + t, 2, tuple(rows.shape))))

    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    new(0)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        one(1, side)
    for t in range(6):
        new(t)
        one(0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0].view(torch.int16), outs[1].view(torch.int16)), t
        assert torch.equal(ctx[0].lens, ctx[1].lens)
    assert ctx[0].check() == gcb.GC_OK and ctx[1].check() == gcb.GC_OK


def test_two_contexts_on_two_streams():
    """Pools, caches and workspaces of their own: no order between them."""
    import torch
    Hq, Hkv, d, ps, B = 16, 2, 128, 16, 5
    rows = [bf16_tensor(wl.normal_bf16(s, 5, (B, Hq + 2 * Hkv, d))) for s in range(2)]
    new = [bf16_tensor(wl.normal_bf16(s, 6, (B * 200, Hq + 2 * Hkv, d))) for s in range(2)]
    results = {}
    for order in ("one", "both"):
        ctx = [FourBitContext(Hq, Hkv, d, ps, B, 400, seed=s) for s in range(2)]
        outs = [torch.zeros((8, B, Hq, d), dtype=torch.bfloat16, device="cuda") for _ in ctx]
        pre = [torch.zeros((B * 200, Hq, d), dtype=torch.bfloat16, device="cuda") for _ in ctx]
        for c in ctx:
            c.begin([200] * B)
        streams = [torch.cuda.Stream() for _ in ctx]
        torch.cuda.synchronize()
        for i, c in enumerate(ctx):
            s = streams[i]
            c.prefill(new[i], pre[i], 0, s)
            c.advance(200)
            if order == "one":
                torch.cuda.synchronize()
        for t in range(8):
            for i, c in enumerate(ctx):
                c.step(rows[i], outs[i][t], 0, streams[i])
                c.advance(1)
                if order == "one":
                    torch.cuda.synchronize()
        torch.cuda.synchronize()
        assert all(c.check() == gcb.GC_OK for c in ctx)
        results[order] = pre + outs
    for a, b in zip(results["one"], results["both"]):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))


def test_pages_past_32_bits():
    """Caches of 5 GiB a plane: the same bytes and bits as in a small one."""
    import torch
    Hq, Hkv, d, ps, B = 8, 2, 128, 16, 3
    small = FourBitContext(Hq, Hkv, d, ps, B, 300, seed=1, staging_pages=2)
    far = FourBitContext(Hq, Hkv, d, ps, B, 300, seed=1, staging_pages=2)
    page = Hkv * ps * (d // 2 + d // 16)
    n = 5 * 2 ** 30 // page
    far.cache = torch.empty(gcb.gc_kv_q4_bytes(far.pool.cfg, n), dtype=torch.uint8, device="cuda")
    assert far.cache.numel() == 2 * n * page
    far.table = (n - 1 - small.table).int()
    far.table_host = n - 1 - small.table_host
    far.pages = n
    image = bf16_tensor(wl.normal_bf16(1, 2, (2, 1, 2, Hkv, ps, d)))
    rows = [bf16_tensor(wl.normal_bf16(t, 3, (k, Hq + 2 * Hkv, d))) for t, k in ((0, 90), (1, B))]
    got = []
    for c in (small, far):
        c.load(image, [0, 0], [0, 1])
        c.advance(_i32([2 * ps, 0, 0], "cuda"))
        c.begin([40, 17, 33])
        pre = torch.zeros((90, Hq, d), dtype=torch.bfloat16, device="cuda")
        c.prefill(rows[0], pre)
        c.advance(_i32([40, 17, 33], "cuda"))
        out = torch.zeros((B, Hq, d), dtype=torch.bfloat16, device="cuda")
        c.step(rows[1], out)
        back = gcb.KVPool.create(1, Hkv, d, ps, 2)
        gcb.gc_kv_unpack_q4(back.handle, c.cache, c.pages, c.table[0, :2].contiguous(),
                            _i32([0, 1], "cuda"), 2, 0, 1)
        assert c.check() == gcb.GC_OK and back.check() == gcb.GC_OK
        got.append((pre, out, back.planes().clone()))
    for a, b in zip(*got):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))
