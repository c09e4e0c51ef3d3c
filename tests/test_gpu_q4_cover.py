"""Every key of a request counts once in decode over 4-bit pages, wherever the work is cut
between warps and CTAs: with q = 0 all keys weigh the same, and column t / 16 mod d of V is
7 at token t and 0 elsewhere, so that a group of 16 keys that is lost or counted twice moves
its column by at least a 32nd of itself."""
import numpy as np
import pytest

from paper_2505_23970_gb300 import binding as gcb
from paper_2505_23970_gb300.harness import _i32

pytestmark = pytest.mark.gpu


def column(t, d):
    return t // 16 % d


@pytest.mark.parametrize("recent", [0, 2])
@pytest.mark.parametrize("Hq,Hkv,d,ps,tokens,lens", [
    (8, 1, 128, 16, 1, [9216]),
    (64, 8, 128, 16, 1, [65536, 9217, 30000, 1, 16, 33, 12345, 64]),
    (16, 1, 128, 16, 1, [65535, 20001, 7]),
    (32, 8, 128, 64, 4, [50000, 4, 9300, 700, 17, 20000]),
    (8, 8, 128, 16, 7, [33333, 7, 8, 2000]),
    (64, 8, 64, 16, 1, [32768, 9217, 15, 30001, 31]),
    (16, 1, 64, 128, 1, [32000, 129, 10000]),
    (8, 2, 64, 16, 4, [32768, 4, 19, 11111, 300]),
    (8, 2, 64, 16, 2, [700 + 13 * i for i in range(200)]),
    (8, 1, 128, 16, 1, [100 + 41 * i % 3000 for i in range(700)]),
    (16, 2, 128, 16, 2, [2 + 37 * i % 900 for i in range(1100)]),
])
def test_every_key_counts_once(Hq, Hkv, d, ps, tokens, lens, recent):
    """The weights are equal powers of two, the codes, the scale 1 and the sums of up to
    2^16 equal terms exact; 1 / L is rounded and the result to bf16: 2^-8 and some 2^-22."""
    import torch
    B, G = len(lens), Hq // Hkv
    rng = np.random.default_rng([B, d])
    blocks = np.array([-(-n // ps) for n in lens])
    new = np.minimum(recent, blocks)
    n4, n16 = max(1, int((blocks - new).sum())), max(1, int(new.sum()))
    width = int(blocks.max())
    table4, table16 = np.full((B, width), -1), np.full((B, width), -1)
    p4, p16 = rng.permutation(n4), rng.permutation(n16)
    a = c = 0
    for b in range(B):
        m, r = blocks[b] - new[b], new[b]
        table4[b, :m], table16[b, m:m + r] = p4[a:a + m], p16[c:c + r]
        a, c = a + m, c + r
    # codes of 0 with scales of 0 (V), any codes with a scale of 1 (K)
    cache = torch.full((2, n4, Hkv, ps * (d // 2 + d // 16)), 0x88, dtype=torch.uint8, device="cuda")
    gen = torch.Generator(device="cuda")
    gen.manual_seed(B)
    cache[0, ..., :ps * d // 2].random_(0, 256, generator=gen)
    scales = cache[..., ps * d // 2:].view(torch.bfloat16).unflatten(-1, (ps, d // 32))
    scales[0], scales[1] = 1, 0
    pool = gcb.KVPool.create(1, Hkv, d, ps, n16)
    pool.planes().zero_()
    pool.planes()[0, 0] = 1
    for b, n in enumerate(lens):
        t = np.arange(n)
        col = column(t, d)
        page4, page16, slot = table4[b, t // ps], table16[b, t // ps], t % ps
        four = page4 >= 0
        at = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()
        # V: 16-bit word r (d / 32) + g has columns 32 g + 4 r + j, nibble j
        g, r, j = col // 32, col % 32 // 4, col % 4
        byte = slot * (d // 2) + (r * (d // 32) + g) * 2 + j // 2
        value = np.where(j % 2, 0xF8, 0x8F).astype(np.uint8)
        for h in range(Hkv):
            cache[1, :, h].index_put_((at(page4[four]), at(byte[four])), at(value[four]))
            scales[1, :, h].index_put_((at(page4[four]), at(slot[four]), at(g[four])),
                                       torch.ones(int(four.sum()), dtype=torch.bfloat16,
                                                  device="cuda"))
            pool.planes()[0, 1, :, h].index_put_((at(page16[~four]), at(slot[~four]),
                                                  at(col[~four])),
                                                 torch.full((int((~four).sum()),), 7.0,
                                                            dtype=torch.bfloat16, device="cuda"))
    q = torch.zeros((B, tokens, Hq, d), dtype=torch.bfloat16, device="cuda")
    out = torch.full_like(q, float("nan"))
    need = gcb.gc_paged_decode_q4_workspace_bytes(pool.handle, B, width, Hq, tokens)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    dev = [_i32(x, "cuda") for x in (table16, lens, table4)]
    gcb.gc_paged_decode_attn_q4(q, pool.handle, dev[0], dev[1], out, None, 0, B, width, Hq, 1.0, ws,
                                need, cache, dev[2], n4, tokens)
    assert pool.check() == gcb.GC_OK
    got = out.double().cpu().numpy()
    for b, n in enumerate(lens):
        for i in range(tokens):
            seen = n - tokens + 1 + i
            want = 7.0 * np.bincount(column(np.arange(seen), d), minlength=d) / seen
            off = np.abs(got[b, i] - want) - want * (2.0 ** -8 + 2.0 ** -20)
            bad = np.argwhere(~(off <= 0))
            assert not len(bad), (b, n, i, len(bad), bad[0], got[b, i][tuple(bad[0])],
                                  want[bad[0][1]])
    pool.close()
