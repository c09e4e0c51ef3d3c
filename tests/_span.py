"""Inputs and the 64-bit form of the attention whose rows see all keys of one or
two page lists (cross attention, decode behind a shared prefix).

Bound of one output value, with A = sum p |v| / sum p over its row's n keys: P is
rounded to bf16 (2^-8 of each term: 2^-8 A) and the output too (2^-8 of it); the
scores are sums of d products in binary32 (with normal inputs |q_i k_i| sums up to
about 11 in units of the scaled score, so they are 128 * 2^-24 * 11 < 2^-13 off and
P and its sum 2^-12 A each); sums over n terms lose at most n 2^-23 A."""
import numpy as np

from paper_2505_23970_gb300 import binding as gcb
from paper_2505_23970_gb300 import workloads as wl
from paper_2505_23970_gb300.harness import _i32, bf16_tensor

NAN = 0x7FC0


class Pages:
    """A pool in which page lists of given lengths have scattered pages; every slot
    that is not in a list holds NaN.  `reuse`: long lists repeat that many pages."""

    def __init__(self, Hkv, d, ps, *lists, seed=0, L=1, layer=0, reuse=None, scale_k=1.0):
        import torch
        counts = [[-(-n // ps) for n in lens] for lens in lists]
        total = sum(map(sum, counts))
        self.num_pages = (reuse or total + total // 4) + 1
        self.layer, self.ps, self.Hkv, self.d = layer, ps, Hkv, d
        bits = np.full((L, 2, self.num_pages, Hkv, ps, d), NAN, np.uint16)
        rng = np.random.default_rng([seed, 31])
        perm = rng.permutation(self.num_pages).astype(np.int32)
        self.tables, at = [], 0
        filled = wl.normal_bf16(seed, 32, bits.shape[1:])
        if scale_k != 1.0:
            filled[0] = wl.f32_to_bf16_bits(wl.bf16_bits_to_f32(filled[0]) * scale_k)
        for lens, cnt in zip(lists, counts):
            t = np.full((len(lens), max(1, max(cnt, default=0))), -1, np.int32)
            for b, (n, k) in enumerate(zip(lens, cnt)):
                if reuse:
                    t[b, :k] = rng.integers(0, self.num_pages, k)
                    bits[layer][:, t[b, :k]] = filled[:, t[b, :k]]
                    continue
                t[b, :k] = perm[at:at + k]
                at += k
                for j, page in enumerate(t[b, :k]):
                    m = min(ps, n - j * ps)
                    bits[layer][:, page, :, :m] = filled[:, page, :, :m]
            self.tables.append(t)
        self.bits = bits
        self.pool = gcb.KVPool.create(L, Hkv, d, ps, self.num_pages)
        self.pool.planes().copy_(bf16_tensor(bits))
        self.dev_tables = [_i32(t, "cuda") for t in self.tables]
        self.values = torch.from_numpy(wl.bf16_bits_to_f32(bits[layer])).cuda()

    def keys(self, which, row, n):
        """K and V [n][Hkv][d] of list `row` of table `which`, in 64 bits."""
        import torch
        used = torch.from_numpy(self.tables[which][row, :-(-n // self.ps)].astype(np.int64)).cuda()
        kv = self.values[:, used].permute(0, 1, 3, 2, 4).reshape(2, -1, self.Hkv, self.d)
        return kv[:, :n].double()


def attend(q, kv, scale):
    """(out, bound) of rows q [n][Hq][d] over kv [2][T][Hkv][d], all in 64 bits."""
    import torch
    n, Hq, d = q.shape
    T, Hkv = kv.shape[1:3]
    if T == 0:
        return torch.zeros_like(q), torch.zeros_like(q)
    qs = q.view(n, Hkv, Hq // Hkv, d)
    p = torch.softmax(torch.einsum("nhgd,thd->nhgt", qs, kv[0]) * scale, -1)
    o = torch.einsum("nhgt,thd->nhgd", p, kv[1]).reshape(n, Hq, d)
    a = torch.einsum("nhgt,thd->nhgd", p, kv[1].abs()).reshape(n, Hq, d)
    return o, a * (2.0 ** -8 + 2.0 ** -11 + T * 2.0 ** -23) + o.abs() * 2.0 ** -8


def assert_within(got, want, bound, what=""):
    import torch
    got = got.double()
    assert torch.isfinite(got).all(), f"{what}: non-finite outputs"
    over = (got - want).abs() - bound
    assert (over <= 0).all(), f"{what}: {(over > 0).sum().item()} values off, by up to " \
        f"{over.max().item():.3g} past their bound"
