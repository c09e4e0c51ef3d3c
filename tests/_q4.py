"""The 4-bit cache's format in numpy, from its definition, and inputs in it."""
import numpy as np

from paper_2505_23970_gb300 import binding as gcb
from paper_2505_23970_gb300 import workloads as wl
from paper_2505_23970_gb300.harness import _i32, bf16_tensor

K_NIBBLE = [0, 4, 2, 6, 1, 5, 3, 7]  # of columns 0..7 of a K word


def f32(bits):
    return wl.bf16_bits_to_f32(bits)


def quantise(bits):
    """bf16 bits [..., d] -> (codes -7..7 [..., d/32, 32], scales [..., d/32] as bf16 bits)."""
    x = f32(np.asarray(bits, np.uint16)).reshape(*np.shape(bits)[:-1], np.shape(bits)[-1] // 32, 32)
    with np.errstate(all="ignore"):
        amax = np.where(np.isfinite(x), np.abs(x), 0).max(-1).astype(np.float32)
        s_bits = wl.f32_to_bf16_bits(np.minimum(amax / np.float32(7), np.float32(2.0 ** 15)))
        s = f32(s_bits)
        s_bits = np.where(s < 2.0 ** -24, 0, s_bits).astype(np.uint16)
        s = f32(s_bits)
        inv = np.where(s > 0, np.float32(1) / np.where(s > 0, s, 1), 0).astype(np.float32)
        p = x.astype(np.float64) * inv[..., None]  # exact
        c = np.where(np.isnan(p), 0, np.clip(np.rint(p), -7, 7))
    return c.astype(np.int64), s_bits


def values(bits):
    """What 4 bits hold of bf16 values, in binary32 (exact)."""
    c, s = quantise(bits)
    return (c.astype(np.float32) * f32(s)[..., None]).reshape(np.shape(bits))


def row_bytes(bits, is_k):
    """(codes [..., d/2] bytes, scales [..., d/32]) of rows [..., d]."""
    c, s = quantise(bits)
    u = (c + 8).astype(np.uint8)  # [..., g, 32]
    if is_k:
        u = u.reshape(*u.shape[:-1], 4, 8)                  # g, q, j
        n = np.empty_like(u)
        n[..., K_NIBBLE] = u
    else:
        n = u.reshape(*u.shape[:-1], 8, 4)                  # g, r, j
    n = np.swapaxes(n, -2, -3)                              # unit, group, nibble
    codes = (n[..., 0::2] | n[..., 1::2] << 4)
    return codes.reshape(*codes.shape[:-3], -1), s


def page_bytes(bits, is_k):
    """Rows [..., ps, d] of a head as its bytes of a 4-bit page."""
    codes, s = row_bytes(bits, is_k)
    lead = codes.shape[:-2]
    return np.concatenate([codes.reshape(*lead, -1),
                           np.ascontiguousarray(s).reshape(*lead, -1).view(np.uint8)], -1)


def cache_bytes(bits):
    """[L][2][pages][Hkv][ps][d] bf16 bits -> the cache's bytes [L][2][pages][Hkv][...]."""
    return np.stack([page_bytes(bits[:, 0], True), page_bytes(bits[:, 1], False)], 1)


class Cache4:
    """A 4-bit cache on the device and the bf16 values it was made from."""

    def __init__(self, bits):
        import torch
        self.bits, self.pages = bits, bits.shape[2]
        self.host = cache_bytes(bits)
        self.dev = torch.from_numpy(self.host.copy()).cuda()

    def now(self):
        return self.dev.cpu().numpy()


class Context:
    """Requests of the given lengths whose pages are in a 4-bit cache, the last `recent` of
    each in a 16-bit pool; slots that hold no token have scales (or values) of NaN."""

    def __init__(self, lens, Hkv, d, ps, recent=0, seed=0, L=1, layer=0, size=1.0, width=None):
        import torch
        self.lens, self.Hkv, self.d, self.ps, self.layer, self.L = lens, Hkv, d, ps, layer, L
        rng = np.random.default_rng([seed, 77])
        blocks = [-(-n // ps) for n in lens]
        self.width = width or max(1, max(blocks))
        new = [min(recent, k) for k in blocks]
        self.pages4 = max(1, sum(blocks) - sum(new)) + 2
        self.pages16 = max(1, sum(new)) + 1
        p4, p16 = rng.permutation(self.pages4), rng.permutation(self.pages16)
        self.table4 = np.full((len(lens), self.width), -1, np.int32)
        self.table16 = np.full((len(lens), self.width), -1, np.int32)
        a = b = 0
        for i, (k, r) in enumerate(zip(blocks, new)):
            self.table4[i, :k - r] = p4[a:a + k - r]
            self.table16[i, k - r:k] = p16[b:b + r]
            a, b = a + k - r, b + r
        raw = f32(wl.normal_bf16(seed, 41, (L, 2, self.pages4, Hkv, ps, d))) * size
        self.bits4 = wl.f32_to_bf16_bits(raw.astype(np.float32))
        self.bits16 = wl.f32_to_bf16_bits(
            (f32(wl.normal_bf16(seed, 42, (L, 2, self.pages16, Hkv, ps, d))) * size).astype(np.float32))
        host = cache_bytes(self.bits4)
        used4, used16 = np.zeros((self.pages4, ps), bool), np.zeros((self.pages16, ps), bool)
        for i, n in enumerate(lens):
            for j in range(blocks[i]):
                m = min(ps, n - j * ps)
                if self.table4[i, j] >= 0:
                    used4[self.table4[i, j], :m] = True
                else:
                    used16[self.table16[i, j], :m] = True
        scales = host[..., ps * d // 2:].reshape(L, 2, self.pages4, Hkv, ps, d // 16)
        scales.transpose(2, 4, 0, 1, 3, 5)[~used4] = np.array([0xC0, 0x7F] * (d // 32), np.uint8)
        self.bits16.transpose(2, 4, 0, 1, 3, 5)[~used16] = 0x7FC0
        self.host = host
        self.cache = torch.from_numpy(host).cuda()
        self.pool = gcb.KVPool.create(L, Hkv, d, ps, self.pages16)
        self.pool.planes().copy_(bf16_tensor(self.bits16))
        self.dev4, self.dev16 = _i32(self.table4, "cuda"), _i32(self.table16, "cuda")
        self.seq_lens = _i32(np.asarray(lens), "cuda")

    def keys(self, b):
        """(values [2][T][Hkv][d], scales [2][T][Hkv][d/32]) of a request, 64 bits; the
        scale of a 16-bit value is 0."""
        T, out, sc = self.lens[b], [], []
        for j in range(-(-T // self.ps)):
            p = self.table4[b, j]
            if p >= 0:
                x = self.bits4[self.layer][:, p]
                out.append(values(x))
                sc.append(f32(quantise(x)[1]))
            else:
                x = f32(self.bits16[self.layer][:, self.table16[b, j]])
                out.append(x)
                sc.append(np.zeros((*x.shape[:-1], self.d // 32)))
        v = np.concatenate(out, 2).transpose(0, 2, 1, 3)[:, :T].astype(np.float64)
        s = np.concatenate(sc, 2).transpose(0, 2, 1, 3)[:, :T].astype(np.float64)
        return v, s


def decode_reference(q, kv, scales, scale, tokens):
    """(out, bound) of rows q [tokens][Hq][d] of one request, in 64 bits.

    With A = sum p |v| / sum p and S = sum p s / sum p over a row's n keys:
    * P s (P, of a 16-bit key) is rounded to bf16, 2^-8 of a term: 2^-8 A (codes times
      the rounded P s, and the offset times the same, differ from c s by nothing else);
    * a group's score is a sum of 32 products q (c + 8) and a start of -8 sum q in
      binary32: at most 33 roundings of 2^-23 of sums up to 23 sum |q|, times s, and
      4 more of the sum over groups and its scalings; a 16-bit key's is d products;
    * O is a sum of n / 8 products' results, each off by 2^-23 of what it has reached
      (at most A + 23 S), and of the 16 terms inside it; sums of P are n additions;
    * the result is rounded to bf16.
    """
    T, Hkv, d = kv.shape[1:]
    Hq = q.shape[1]
    G = Hq // Hkv
    qg = q.reshape(tokens, Hkv, G, d)
    s = np.einsum("ihgd,thd->ihgt", qg, kv[0]) * scale
    sizes = np.abs(qg).reshape(tokens, Hkv, G, d // 32, 32).sum(-1)
    wide = scales[0].sum(-1) == 0                                       # 16-bit keys [t][h]
    err = np.einsum("ihgc,thc->ihgt", sizes, scales[0]) * 23 * 37 * 2.0 ** -23
    err += np.einsum("ihgd,thd->ihgt", np.abs(qg), np.abs(kv[0]) * wide[..., None]) * d * 2.0 ** -23
    seen = np.arange(T) <= (T - tokens + np.arange(tokens))[:, None]
    s = np.where(seen[:, None, None], s, -np.inf)
    e = np.where(seen[:, None, None], err * scale, 0).max(-1)[..., None]  # of the exponents
    p = np.exp(s - s.max(-1, keepdims=True))
    p /= p.sum(-1, keepdims=True)
    o = np.einsum("ihgt,thd->ihgd", p, kv[1])
    A = np.einsum("ihgt,thd->ihgd", p, np.abs(kv[1]))
    S = np.repeat(np.einsum("ihgt,thc->ihgc", p, scales[1]), 32, -1)
    n = T + 64.0
    bound = (A * (2.0 ** -8 + 2 * e + 2.0 ** -20 + n * 2.0 ** -23) + (A + 23 * S) * n / 4 * 2.0 ** -23 +
             23 * S * 16 * 2.0 ** -23 + np.abs(o) * 2.0 ** -8)
    return o.reshape(tokens, Hq, d), bound.reshape(tokens, Hq, d)
