"""Performance cases of a paged KV cache that is kept in 4 bits: what a serving
program has the library do with it, one layer at a time (pages: several).

A case is one pass through one operator, or through the two that write the cache
and read it back:

* ``write``    the new tokens' q and k are rotated to their positions, q stays in
               16 bits, k and v are quantised as they are written to the 4-bit
               pages (``gc_kv_append_rope_q4``); the pages written to are read
               back (``gc_kv_unpack_q4``)
* ``page``     whole 16-bit pages of several layers are quantised into 4-bit pages
               (``gc_kv_pack_q4``) and read back into other 16-bit pages
* ``decode``   generation: one token, or a few drafted ones, of every request over
               its context (``gc_paged_decode_attn_q4``)
* ``prefill``  causal attention of new tokens over the cached and the new ones
               (``gc_prefix_prefill_attn_q4``)

Fields: ``B`` requests; ``hq`` / ``hkv`` heads of size ``d``; pages of ``ps``
tokens; ``lens`` is the seed of the lengths alone and ``spread`` how they differ
("fixed": all the same; "uniform": from an eighth on; "lognormal": the given
length is the median).

write:   ``prefix`` cached and ``new`` new tokens; ``rot`` of a head's ``d``
         columns are rotated (0: none), in halves or (``interleaved``) neighbours.
page:    ``pages`` of ``layers`` layers.
decode:  contexts of ``kv`` tokens, the last ``tokens`` of them the queries', the
         last ``recent`` pages of each still in 16 bits.
prefill: ``prefix`` cached and ``new`` new tokens.

A 4-bit value is c s: per token, head and 32 columns one bf16 scale
s = amax / 7 and codes c = -7..7 (x times the binary32 reciprocal of s, rounded
once to the nearest whole number, ties to even).
"""
import math

import numpy as np
import torch

own = False

_BF16 = torch.bfloat16


def _case(name, c):
    return dict(c, name=name) if name else c


def _write(name, B, hq, hkv, d, ps, prefix, new, rot, interleaved, spread="fixed", lens=0):
    return _case(name, dict(kind="write", B=B, hq=hq, hkv=hkv, d=d, ps=ps, prefix=prefix, new=new,
                            rot=rot, interleaved=interleaved, spread=spread, lens=lens))


def _page(name, hkv, d, ps, pages, layers):
    return _case(name, dict(kind="page", hkv=hkv, d=d, ps=ps, pages=pages, layers=layers))


def _decode(name, B, hq, hkv, d, ps, kv, tokens, recent, spread="fixed", lens=0):
    return _case(name, dict(kind="decode", B=B, hq=hq, hkv=hkv, d=d, ps=ps, kv=kv, tokens=tokens,
                            recent=recent, spread=spread, lens=lens))


def _prefill(name, B, hq, hkv, d, ps, prefix, new, spread="fixed", lens=0):
    return _case(name, dict(kind="prefill", B=B, hq=hq, hkv=hkv, d=d, ps=ps, prefix=prefix,
                            new=new, spread=spread, lens=lens))


def listed():
    return [
        # generation on a Llama-3-70B-shaped layer: one new token of eight
        # requests; launch and latency are all there is
        _write("write-decode-70b", 8, 64, 8, 128, 16, 9215, 1, 128, False),
        # a batch of long cached prefixes on the same layer, 1024 new tokens each
        _write("write-prefill-70b", 8, 64, 8, 128, 16, 8192, 1024, 128, False),
        # ragged batch of a model with head size 64 that rotates half of each
        # head, neighbours as pairs
        _write("write-ragged-d64", 12, 32, 8, 64, 16, 3001, 701, 32, True, "uniform"),
        # the finished pages of one short conversation, small pages, head size 64
        _page("page-conversation-d64", 8, 64, 16, 21, 2),
        # contexts of an idle application move to 4 bits, some layers at a time
        _page("page-application-70b", 8, 128, 16, 576, 8),
        # the smallest decode: one request of a small GQA 4:1 model
        _decode("decode-tiny-d64", 1, 4, 1, 64, 16, 321, 1, 0),
        # eight long conversations, 70B-shaped layer
        _decode("decode-70b", 8, 64, 8, 128, 16, 9216, 1, 0),
        # multi-turn traffic, every request's newest page still in 16 bits
        _decode("decode-multi-turn-70b", 64, 64, 8, 128, 16, 3000, 1, 1, "lognormal"),
        # four drafted tokens of each request verified at once, 8B-shaped layer
        _decode("decode-drafts-8b", 16, 32, 8, 128, 16, 8192, 4, 0, "uniform"),
        # questions on long documents: the largest cache
        _decode("decode-documents-70b", 32, 64, 8, 128, 64, 65536, 1, 0, "uniform"),
        # a batch of long cached prefixes, 1024 new tokens each: the most work
        _prefill("prefill-70b", 8, 64, 8, 128, 16, 8192, 1024),
        # a ragged batch of the d 64 model
        _prefill("prefill-ragged-d64", 12, 32, 8, 64, 16, 3001, 701, "uniform"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["write", "page", "decode", "decode", "prefill"])
    d = rng.choice([64, 128, 128])
    hkv = rng.choice([1, 2, 4, 8, 8])
    group = rng.choice([1, 2, 4, 8, 8, 16])
    ps = rng.choice([16, 16, 32, 64, 128])
    lens = rng.randrange(1 << 20)
    spread = rng.choice(["fixed", "uniform", "lognormal"])
    if kind == "write":
        c = _write("", _log(rng, 1, 128), hkv * group, hkv, d, ps, _log(rng, 16, 4096),
                   _log(rng, 1, 1024), rng.choice([d, d, d // 2, 48, 0]), rng.random() < 0.5,
                   spread, lens)
    elif kind == "page":
        c = _page("", hkv, d, ps, _log(rng, 1, 1024), rng.randint(1, 8))
        while c["pages"] > 1 and work(c)["bytes"] > 1e9:
            c["pages"] //= 2
        return c
    elif kind == "decode":
        c = _decode("", _log(rng, 1, 128), hkv * group, hkv, d, ps, _log(rng, 32, 65536),
                    rng.randint(1, max(1, min(4, 16 // group))), rng.choice([0, 0, 1, 3]), spread,
                    lens)
    else:
        c = _prefill("", _log(rng, 1, 32), hkv * group, hkv, d, ps, _log(rng, 16, 16384),
                     _log(rng, 2, 1024), spread, lens)
    # no dearer than the largest listed cases, padded to the longest request too
    while c["B"] > 1 and (work(c)["bytes"] > 1.3e9 or work(c)["flops"] > 2e12 or
                          _padded(c) > 5e9):
        c["B"] //= 2
    return c


# ---------------------------------------------------------------- lengths
def _spread(c, length, stream, least, most):
    """`B` lengths around `length`."""
    rng = np.random.default_rng([c["lens"], stream])
    if c["spread"] == "fixed":
        return np.full(c["B"], max(least, length), np.int64)
    if c["spread"] == "lognormal":
        x = np.rint(rng.lognormal(math.log(max(length, 1)), 0.8, size=c["B"])).astype(np.int64)
        return np.clip(x, max(least, length // 12), min(most, 8 * length))
    return rng.integers(max(least, length // 8), max(least, length), size=c["B"], endpoint=True)


def _lens(c):
    """(cached tokens, new tokens) of every request; a decode's tokens are the new ones."""
    if c["kind"] == "decode":
        kv = _spread(c, c["kv"], 1, c["tokens"], 131072)
        return kv - c["tokens"], np.full(c["B"], c["tokens"], np.int64)
    return _spread(c, c["prefix"], 1, 0, 16384), _spread(c, c["new"], 2, 1, 4096)


def _padded(c):
    """Elements of the largest tensors when every request is as long as the longest."""
    if c["kind"] == "write":
        return 0
    P, n = _lens(c)
    keys, rows = int((P + n).max()), int(n.max())
    return c["B"] * keys * max(c["hq"] * rows, 2 * c["hkv"] * c["d"])


# ----------------------------------------------------------------- inputs
def _gen(seed, stream):
    gen = torch.Generator(device="cuda")
    gen.manual_seed((int(seed) * 1000003 + stream) & 0x7FFFFFFFFFFFFFFF)
    return gen


def _randn(gen, shape):
    return torch.randn(shape, generator=gen, device="cuda", dtype=_BF16)


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def _angles(n, rot):
    """[n][2][rot/2]: cosines and sines of position p, base 500000."""
    freq = 500000.0 ** (-np.arange(0, rot, 2) / rot)
    a = np.arange(n)[:, None] * freq
    return np.stack([np.cos(a), np.sin(a)], 1).astype(np.float32)


def _cached(seed, layers, pages, hkv, ps, d):
    """The values behind the 4-bit pages, [layers][2][pages][hkv][ps][d]; a head's
    scale differs from the others' as activations do."""
    x = _randn(_gen(seed, 1), (layers, 2, pages, hkv, ps, d))
    size = torch.exp2(torch.randn((layers, 2, 1, hkv, 1, d // 32, 1), generator=_gen(seed, 2),
                                  device="cuda"))
    x.view(layers, 2, pages, hkv, ps, d // 32, 32).mul_(size.to(_BF16))
    return x


def _inputs(c, seed):
    d, ps, hkv = c["d"], c["ps"], c["hkv"]
    x = dict(case=c)
    order = np.random.default_rng([int(seed) & 0x7FFFFFFF, 3])
    if c["kind"] == "page":
        # 16-bit pages, a quarter of them others'; the last ones take what is read back
        n = c["pages"]
        x.update(pages=n + n // 4 + 1, pool_ids=order.permutation(n + n // 4 + 1)[:n],
                 q4_ids=order.permutation(n + 3)[:n], n4=n + 3)
        x["pool"] = _randn(_gen(seed, 4), (c["layers"], 2, x["pages"], hkv, ps, d))
        return x
    P, n = _lens(c)
    B, hq = c["B"], c["hq"]
    blocks = -(-(P + n) // ps)
    width = int(blocks.max())
    # the tokens that are queries are in the cache already, but for a write
    recent = np.minimum(c.get("recent", 0), blocks)
    n4 = max(1, math.ceil(1.25 * int((blocks - recent).sum())))
    n16 = max(1, math.ceil(1.25 * int(recent.sum())))
    perm4, perm16 = order.permutation(n4), order.permutation(n16)
    table4, table16 = np.full((B, width), -1, np.int64), np.full((B, width), -1, np.int64)
    at4 = at16 = 0
    for b in range(B):
        m, r = int(blocks[b] - recent[b]), int(recent[b])
        table4[b, :m] = perm4[at4:at4 + m]
        table16[b, m:m + r] = perm16[at16:at16 + r]
        at4, at16 = at4 + m, at16 + r
    x.update(P=P, n=n, cu=np.concatenate([[0], np.cumsum(n)]), width=width, table4=table4,
             table16=table16, n4=n4, n16=n16)
    T = int(n.sum())
    gen = _gen(seed, 5)
    if c["kind"] == "write":
        rows = _randn(gen, (T, hq + 2 * hkv, d))
        x["q"], x["k"], x["v"] = rows[:, :hq], rows[:, hq:hq + hkv], rows[:, hq + hkv:]
        x["angles"] = torch.from_numpy(_angles(int((P + n).max()), max(c["rot"], 2))).cuda()
        # pages that new tokens go to, request after request
        x["touched"] = np.concatenate([table4[b, P[b] // ps:blocks[b]] for b in range(B)])
    else:
        x["q"] = _randn(gen, (T, hq, d))
    x["values"] = _cached(seed, 1, n4, hkv, ps, d)
    x["pool"] = _randn(_gen(seed, 6), (1, 2, n16, hkv, ps, d)) if c.get("recent") else None
    return x


def prepare(case, seed):
    c = {k: v for k, v in case.items() if k != "name"}
    x = _inputs(c, seed)
    d, ps, hkv, kind = c["d"], c["ps"], c["hkv"], c["kind"]
    s = dict(c, scale=d ** -0.5, n4=x["n4"])
    row = d // 2 + d // 16
    layers = c.get("layers", 1)
    if kind == "page":
        s.update(pool_ids=_i32(x["pool_ids"]), q4_ids=_i32(x["q4_ids"]),
                 back=_i32(x["pages"] + np.arange(c["pages"])), planes=x["pool"], n=c["pages"])
        s["cache"] = torch.zeros((layers, 2, x["n4"], hkv, ps * row), dtype=torch.uint8,
                                 device="cuda")
        pool_pages = x["pages"] + c["pages"]
    else:
        s.update(q=x["q"], P=_i32(x["P"]), n=_i32(x["n"]), cu=_i32(x["cu"]), T=int(x["n"].sum()),
                 table4=_i32(x["table4"]), table16=_i32(x["table16"]), width=x["width"],
                 total=_i32(x["P"] + x["n"]), most=int((x["P"] + x["n"]).max()),
                 rows=int(x["n"].max()))
        s["cache"] = torch.stack([_pack(x["values"][:, p], p == 0) for p in range(2)], 1)
        s["planes"], pool_pages = x["pool"], x["n16"]
        s["out"] = torch.zeros(x["q"].shape, dtype=_BF16, device="cuda")
        if kind == "write":
            s.update(k=x["k"], v=x["v"], angles=x["angles"], touched=_i32(x["touched"]),
                     back=_i32(np.arange(len(x["touched"]))))
            pool_pages = len(x["touched"])
    if own:
        from paper_2505_23970_gb300 import binding as gcb
        pool = gcb.KVPool.create(layers, hkv, d, ps, pool_pages)
        if s["planes"] is not None:
            pool.planes()[:, :, :s["planes"].shape[2]].copy_(s["planes"])
        need = 0
        if kind == "decode":
            need = gcb.gc_paged_decode_q4_workspace_bytes(pool.handle, c["B"], s["width"],
                                                          c["hq"], c["tokens"])
        elif kind == "prefill":
            need = gcb.gc_prefix_prefill_q4_workspace_bytes(pool.handle, c["B"], s["width"],
                                                            s["n4"])
        s.update(pool=pool, handle=pool.handle, planes=pool.planes(), gcb=gcb, need=need,
                 stream=torch.cuda.current_stream(),
                 work=torch.empty(max(16, need), dtype=torch.uint8, device="cuda"))
    return s


# ------------------------------------------------------------- plain forms
def _quantise(x):
    """Whole codes -7..7 and scales (both binary32) of groups of 32 columns."""
    x = x.float().unflatten(-1, (-1, 32))
    s = (x.abs().amax(-1, keepdim=True) / 7.0).clamp_(max=2.0 ** 15).to(_BF16).float()
    s = torch.where(s < 2.0 ** -24, 0.0, s)
    inv = torch.where(s > 0, 1.0 / s, 0.0)
    # (in 64 bits: many values lie on a border between two codes, or next to one)
    return (x.double() * inv).round_().clamp_(-7, 7).float(), s


def _pack(x, is_k):
    """Values [..., hkv, ps, d] as the bytes [..., hkv, ps * (d/2 + d/16)] of a page."""
    c, s = _quantise(x)
    n = (c + 8).to(torch.uint8)
    if is_k:  # 8 columns a word; words of the groups side by side
        n = n.unflatten(-1, (4, 8))[..., [0, 4, 2, 6, 1, 5, 3, 7]]
    else:     # 4 columns a half word
        n = n.unflatten(-1, (8, 4))
    n = n.transpose(-2, -3)
    codes = (n[..., 0::2] | n[..., 1::2] << 4).flatten(-4)
    scales = s.to(_BF16).contiguous().view(torch.uint8).flatten(-3)
    return torch.cat([codes, scales], -1)


def _unpack(b, is_k, ps, d):
    """The inverse: values [..., hkv, ps, d] in binary32."""
    at = ps * d // 2
    codes, scales = b[..., :at].unflatten(-1, (ps, -1)), b[..., at:].contiguous()
    n = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
    n = n.unflatten(-1, (4, d // 32, 8) if is_k else (8, d // 32, 4)).transpose(-2, -3)
    if is_k:
        n = n[..., [0, 4, 2, 6, 1, 5, 3, 7]]
    s = scales.view(_BF16).float().unflatten(-1, (ps, d // 32, 1))
    return ((n.flatten(-2).float() - 8) * s).flatten(-2)


def _rotate(x, cos, sin, rot, interleaved):
    """x' = x c - y s, y' = y c + x s: the second product rounded to binary32, the
    rest fused (in 64 bits here: a rounding apart, and the value is next to a border)."""
    x = x.double()
    r, rest = x[..., :rot], x[..., rot:]
    a, b = (r[..., 0::2], r[..., 1::2]) if interleaved else (r[..., :rot // 2], r[..., rot // 2:])
    a, b = a * cos - (b * sin).float().double(), b * cos + (a * sin).float().double()
    r = torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1)
    return torch.cat([r, rest], -1).float().to(_BF16)


def _plain_write(s):
    t = torch.arange(s["T"], device="cuda")
    b = torch.searchsorted(s["cu"], t, right=True) - 1
    slot = s["P"][b] + t - s["cu"][b]
    q, k = s["q"], s["k"]
    if s["rot"]:
        row = s["angles"][slot].double()
        cos, sin = row[:, 0, None], row[:, 1, None]
        q = _rotate(q, cos, sin, s["rot"], s["interleaved"])
        k = _rotate(k, cos, sin, s["rot"], s["interleaved"])
    page, at = s["table4"][b, slot // s["ps"]].long(), (slot % s["ps"]).long()
    where = torch.empty(s["n4"], dtype=torch.int64, device="cuda")
    where[s["touched"].long()] = torch.arange(s["touched"].numel(), device="cuda")
    planes = []
    for p, new in enumerate((k, s["v"])):
        old = _unpack(s["cache"][0, p, s["touched"].long()], p == 0, s["ps"], s["d"])
        c, scale = _quantise(new)
        old[where[page], :, at] = (c * scale).flatten(-2)
        planes.append(old.to(_BF16))
    return {"q": q.contiguous(), "kv": torch.stack(planes)[None]}


def _plain_page(s):
    c, scale = _quantise(s["planes"][:, :, s["pool_ids"].long()])
    return {"kv": (c * scale).flatten(-2).to(_BF16)}


def _keys(s):
    """K and V of every request, padded: [2][B][hkv][most][d] in binary32."""
    table, out = s["table4"].clamp(min=0).long(), []
    for p in range(2):
        x = _unpack(s["cache"][0, p, table], p == 0, s["ps"], s["d"])
        if s["planes"] is not None:
            y = s["planes"][0, p, s["table16"].clamp(min=0).long()].float()
            x = torch.where((s["table4"] >= 0)[..., None, None, None], x, y)
        out.append(x.transpose(1, 2).flatten(2, 3)[:, :, :s["most"]])
    return out


def _plain_attention(s):
    B, hkv, d, T, rows = s["B"], s["hkv"], s["d"], s["T"], s["rows"]
    t = torch.arange(T, device="cuda")
    b = torch.searchsorted(s["cu"], t, right=True) - 1
    i = torch.arange(rows, device="cuda")
    at = (s["cu"][:-1, None] + i).clamp(max=T - 1).long()
    q = s["q"][at].float().view(B, rows, hkv, -1, d).transpose(1, 2)  # [B][hkv][rows][G][d]
    k, v = _keys(s)
    if s["kind"] == "prefill":  # the tokens are read as 16-bit values
        k, v = k.to(_BF16).float(), v.to(_BF16).float()
    p = torch.matmul(q.flatten(2, 3), k.transpose(-1, -2)).mul_(s["scale"])
    p = p.view(B, hkv, rows, -1, s["most"])
    # row i of a request sees the keys up to its own position
    past = torch.arange(s["most"], device="cuda") > (s["P"][:, None] + i)[..., None]
    p.masked_fill_(past[:, None, :, None], -math.inf)
    p.sub_(p.amax(-1, keepdim=True)).exp_()
    o = torch.matmul(p.flatten(2, 3), v).view(B, hkv, rows, -1, d) / p.sum(-1, keepdim=True)
    o = o.transpose(1, 2).flatten(2, 3)
    return {"out": o[b, (t - s["cu"][b]).long()].to(_BF16)}


# ------------------------------------------------------------------- pass
def run(s):
    kind = s["kind"]
    if not own:
        return {"write": _plain_write, "page": _plain_page, "decode": _plain_attention,
                "prefill": _plain_attention}[kind](s)
    gcb, h, st = s["gcb"], s["handle"], s["stream"]
    if kind == "write":
        gcb.gc_kv_append_rope_q4(h, s["q"], s["q"].stride(0), s["out"], s["k"], s["k"].stride(0),
                                 s["v"], s["v"].stride(0), s["cache"], s["n4"], s["table4"],
                                 s["P"], st, 0, s["cu"], s["B"], s["width"], s["T"], s["hq"],
                                 s["angles"], s["angles"].shape[0], s["rot"], None,
                                 gcb.GC_ROPE_INTERLEAVED if s["interleaved"] else 0)
        gcb.gc_kv_unpack_q4(h, s["cache"], s["n4"], s["touched"], s["back"], s["touched"].numel(),
                            0, 1, st)
        return {"q": s["out"], "kv": s["planes"]}
    if kind == "page":
        gcb.gc_kv_pack_q4(h, s["pool_ids"], s["cache"], s["n4"], s["q4_ids"], s["n"], 0,
                          s["layers"], st)
        gcb.gc_kv_unpack_q4(h, s["cache"], s["n4"], s["q4_ids"], s["back"], s["n"], 0,
                            s["layers"], st)
        return {"kv": s["planes"][:, :, -s["n"]:]}
    if kind == "decode":
        gcb.gc_paged_decode_attn_q4(s["q"], h, s["table16"], s["total"], s["out"], st, 0, s["B"],
                                    s["width"], s["hq"], s["scale"], s["work"], s["need"],
                                    s["cache"], s["table4"], s["n4"], s["tokens"])
    else:
        gcb.gc_prefix_prefill_attn_q4(s["q"], h, s["table16"], s["P"], s["n"], s["out"], st, 0,
                                      s["cu"], s["B"], s["width"], s["hq"], s["scale"], s["T"],
                                      s["cache"], s["table4"], s["n4"], s["work"], s["need"])
    return {"out": s["out"]}


def work(c):
    d, ps, hkv = c["d"], c["ps"], c["hkv"]
    row16, row4 = 2 * hkv * d * 2, 2 * hkv * (d // 2 + d // 16)  # K and V of one token
    if c["kind"] == "page":
        tokens = c["pages"] * c["layers"] * ps
        # 16-bit pages read and written, 4-bit pages written in between
        return {"bytes": tokens * (2 * row16 + row4), "flops": 4.0 * tokens * row16 / 2}
    P, n = _lens(c)
    T, qo = int(n.sum()), 2 * int(n.sum()) * c["hq"] * d * 2
    if c["kind"] == "write":
        back = int((-(-(P + n) // ps) - P // ps).sum()) * ps  # tokens read back
        # q read and written, k and v read, 4-bit rows written, the rest of their
        # pages read, 16-bit pages written
        return {"bytes": qo + T * (row16 + row4 + c["rot"] * 4) + (back - T) * row4 + back * row16,
                "flops": 3.0 * T * (c["hq"] + hkv) * c["rot"] + 4.0 * back * row16 / 2}
    keys = P + n
    recent = np.minimum(c.get("recent", 0), -(-keys // ps))
    in4 = np.maximum(0, np.minimum(keys, (-(-keys // ps) - recent) * ps))
    return {"bytes": int(in4.sum()) * row4 + int((keys - in4).sum()) * row16 + qo,
            "flops": 4.0 * d * c["hq"] * float((n * P + n * (n + 1) / 2).sum())}


# -------------------------------------------------------------- 64 bits
def _nearest4(x):
    """What 4 bits hold of the bf16 values x, from the definition, in 64 bits."""
    shape = x.shape
    g = x.double().reshape(-1, 32)
    top = g.abs().max(1).values / 7
    s = torch.minimum(top, torch.full_like(top, 32768.0)).bfloat16().double()
    s[s < 2.0 ** -24] = 0
    inv = torch.zeros_like(s)
    inv[s > 0] = (1 / s[s > 0]).float().double()
    c = torch.clamp(torch.round(g * inv[:, None]), -7, 7)
    return (c * s[:, None]).reshape(shape)


def _turned(x, c, angles):
    """Rows x [n][heads][d] of one request at positions whose angles are given."""
    x, rot = x.double(), c["rot"]
    re, im = ((x[..., 0:rot:2], x[..., 1:rot:2]) if c["interleaved"] else
              (x[..., :rot // 2], x[..., rot // 2:rot]))
    z = torch.complex(re, im) * torch.complex(angles[:, 0].double(), angles[:, 1].double())[:, None]
    re.copy_(z.real)
    im.copy_(z.imag)
    return x


def exact(case, seed):
    c = {k: v for k, v in case.items() if k != "name"}
    x = _inputs(c, seed)
    ps, hkv, d = c["ps"], c["hkv"], c["d"]
    if c["kind"] == "page":
        ids = torch.from_numpy(x["pool_ids"]).cuda()
        return {"kv": torch.stack([_nearest4(l[:, ids]) for l in x["pool"]])}
    if c["kind"] == "write":
        q = torch.empty(x["q"].shape, dtype=torch.float64, device="cuda")
        touched = torch.from_numpy(x["touched"]).cuda()
        kv = _nearest4(x["values"][:, :, touched])
        first = 0  # of the request's pages
        for b in range(c["B"]):
            lo, n, P = int(x["cu"][b]), int(x["n"][b]), int(x["P"][b])
            k, turn = x["k"][lo:lo + n], x["angles"][P:P + n]
            q[lo:lo + n] = x["q"][lo:lo + n].double()
            if c["rot"]:
                q[lo:lo + n] = _turned(q[lo:lo + n].clone(), c, turn)
                k = _turned(k, c, turn).bfloat16()
            at = torch.arange(P, P + n, device="cuda")
            page, slot = first + at // ps - P // ps, at % ps
            kv[0, 0, page, :, slot] = _nearest4(k.contiguous())
            kv[0, 1, page, :, slot] = _nearest4(x["v"][lo:lo + n].contiguous())
            first += -(-(P + n) // ps) - P // ps
        return {"q": q, "kv": kv}
    out = torch.empty(x["q"].shape, dtype=torch.float64, device="cuda")
    G = c["hq"] // hkv
    for b in range(c["B"]):
        lo, n, P = int(x["cu"][b]), int(x["n"][b]), int(x["P"][b])
        length = P + n
        t4 = x["table4"][b]
        parts = _nearest4(x["values"][0][:, torch.from_numpy(t4[t4 >= 0]).cuda()])
        t16 = x["table16"][b]
        if (t16 >= 0).any():
            more = x["pool"][0][:, torch.from_numpy(t16[t16 >= 0]).cuda()].double()
            parts = torch.cat([parts, more], 1)
        if c["kind"] == "prefill":
            parts = parts.bfloat16().double()
        kv = parts.transpose(2, 3).reshape(2, -1, hkv, d)[:, :length]
        step = max(1, int(2e8 / (G * length)))
        for g in range(hkv):
            k, v = kv[0, :, g], kv[1, :, g]
            for i in range(0, n, step):
                q = x["q"][lo + i:lo + min(i + step, n), g * G:(g + 1) * G].double()
                s = (q.reshape(-1, d) @ k.T).view(q.shape[0], G, length) * d ** -0.5
                pos = P + i + torch.arange(q.shape[0], device="cuda")
                s = s.masked_fill(torch.arange(length, device="cuda") > pos[:, None, None],
                                  -math.inf)
                out[lo + i:lo + i + q.shape[0], g * G:(g + 1) * G] = torch.softmax(s, -1) @ v
    return {"out": out}
