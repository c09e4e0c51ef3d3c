"""Generation behind shared prefixes as a serving loop runs it: prefixes and encoder
states restored once, then tokens through every layer (rotated append, shared-prefix
decode, cross attention), against the same steps in 64 bits on the rotated values as
they were rounded into the cache."""
import numpy as np
import pytest

from paper_2505_23970_gb300 import binding as gcb
from paper_2505_23970_gb300 import workloads as wl
from paper_2505_23970_gb300.harness import SharedContext, bf16_tensor

from ._span import assert_within, attend

pytestmark = pytest.mark.gpu


def pages_of(table, b, n, ps, planes):
    """K and V [2][n][Hkv][d] of one list, in 64 bits."""
    import torch
    used = torch.from_numpy(table[b, :-(-n // ps)].astype(np.int64)).cuda()
    kv = planes[:, used].permute(0, 1, 3, 2, 4).flatten(1, 2)
    return kv[:, :n].double()


@pytest.mark.parametrize("Hq,Hkv,d,ps,S,sizes,states", [
    (8, 2, 128, 16, [300, 0, 45], [3, 1, 2], [100, 0, 7, 300, 33, 1]),
    (16, 1, 64, 32, [129], [5], None),
    (32, 2, 128, 64, [500, 64], [9, 4], [5] * 13),
])
def test_tokens_through_the_layers(Hq, Hkv, d, ps, S, sizes, states):
    import torch
    L, B, tokens = 2, sum(sizes), 3
    c = SharedContext(Hq, Hkv, d, ps, S, sizes, tokens, states, L=L, seed=Hq)
    c.pool.planes().fill_(float("nan"))
    for name, table in (("shared", c.shared_table), ("states", c.state_table)):
        n = int((table >= 0).sum())
        if n:
            c.restore(bf16_tensor(wl.normal_bf16(d, len(name), (n, L, 2, Hkv, ps, d))), name)
    group, scale = c.group, d ** -0.5
    out = torch.empty((B, Hq, d), dtype=torch.bfloat16, device="cuda")
    seen = torch.empty_like(out)
    for t in range(tokens):
        for layer in range(L):
            rows = bf16_tensor(wl.normal_bf16(d + 7 * t, layer, (B, Hq + 2 * Hkv, d)))
            c.step(rows, out, layer)
            c.cross(c.q, seen, layer)
            planes = c.pool.planes()[layer]
            # positions and slots: the appended key is the rotated one
            a = c.cos_sin[torch.from_numpy(c.shared_lens[group] + t).cuda().long()]
            k = rows[:, Hq:Hq + Hkv].double()
            x, y = k[..., :d // 2], k[..., d // 2:]
            cos, sin = a[:, 0, None].double(), a[:, 1, None].double()
            want = torch.cat([x * cos - y * sin, y * cos + x * sin], -1)
            for b in range(B):
                own = pages_of(c.own_table, b, t + 1, ps, planes)
                # one rounding to bf16 (2^-8 of the value) and binary32's before it
                err = (own[0, t] - want[b]).abs()
                pair = k[b].abs()
                pair = (pair + pair.roll(d // 2, -1)) * 2.0 ** -22
                assert (err <= want[b].abs() * 2.0 ** -8 + pair).all()
                assert torch.equal(own[1, t], rows[b, Hq + Hkv:].double())
                shared = pages_of(c.shared_table, group[b], int(c.shared_lens[group[b]]), ps,
                                  planes)
                w, bound = attend(c.q[b:b + 1].double(), torch.cat([shared, own], 1), scale)
                assert_within(out[b:b + 1], w, bound, f"token {t} layer {layer} request {b}")
                n = 0 if states is None else states[b]
                w, bound = attend(c.q[b:b + 1].double(),
                                  pages_of(c.state_table, b, n, ps, planes), scale)
                assert_within(seen[b:b + 1], w, bound, f"states of request {b}")
        c.advance()
    assert c.check() == gcb.GC_OK
    c.close()
