"""Performance cases of the operators around a cached context that several
requests or several layers of one model use: what a serving program has the
library do with it, one layer at a time.

A case is one pass through one operator:

* ``rope``    the new tokens' q and k are rotated to their positions, q stays
              dense, k and v go into the paged cache
              (``gc_kv_append_rope``)
* ``cross``   attention of every request's new tokens to all of the request's
              cached states of another sequence, an encoder's
              (``gc_paged_cross_attn``)
* ``shared``  generation, one token per request, for groups of requests whose
              contexts begin with the same cached pages
              (``gc_shared_prefix_decode_attn``)

Fields: ``B`` requests; ``hq`` / ``hkv`` heads of size ``d``; pages of ``ps``
tokens; ``lens`` is the seed of the lengths alone and ``spread`` how they
differ ("fixed": all the same; "uniform": from an eighth on; "lognormal": the
given length is the median; "ragged": uniform, and one in eight is 0).

rope:   ``prefix`` cached and ``new`` new tokens; ``rot`` of a head's ``d``
        columns are rotated, in halves or (``interleaved``) neighbours; q, k, v
        are parts of one projection's rows (``fused``) or tensors of their own;
        ``placed``: the positions are given (behind a shared prefix of that
        many tokens), 0: they follow from the cached lengths.
cross:  ``kv`` cached states, ``new`` tokens.
shared: ``groups`` of requests (their sizes drawn unless "fixed"), ``shared``
        tokens in common, ``own`` tokens of each request after them.
"""
import math

import numpy as np
import torch

own = False

_BF16 = torch.bfloat16


def _rope(name, B, hq, hkv, d, ps, prefix, new, rot, interleaved, fused, placed, spread="fixed",
          lens=0):
    c = dict(kind="rope", B=B, hq=hq, hkv=hkv, d=d, ps=ps, prefix=prefix, new=new, rot=rot,
             interleaved=interleaved, fused=fused, placed=placed, spread=spread, lens=lens)
    return dict(c, name=name) if name else c


def _cross(name, B, hq, hkv, d, ps, kv, new, spread="fixed", lens=0):
    c = dict(kind="cross", B=B, hq=hq, hkv=hkv, d=d, ps=ps, kv=kv, new=new, spread=spread,
             lens=lens)
    return dict(c, name=name) if name else c


def _shared(name, B, hq, hkv, d, ps, groups, shared, own_, spread="fixed", lens=0):
    c = dict(kind="shared", B=B, hq=hq, hkv=hkv, d=d, ps=ps, groups=groups, shared=shared,
             own=own_, spread=spread, lens=lens)
    return dict(c, name=name) if name else c


def listed():
    return [
        # generation on a Llama-3-70B-shaped layer: one new token of eight
        # requests; launch and latency are all there is
        _rope("rope-decode-70b", 8, 64, 8, 128, 16, 9215, 1, 128, False, True, 0),
        # a batch of long cached prefixes on the same layer, 1024 new tokens each
        _rope("rope-prefill-70b", 8, 64, 8, 128, 16, 8192, 1024, 128, False, True, 0),
        # ragged batch of a model with head size 64 that rotates half of each
        # head, neighbours as pairs, behind a shared prefix
        _rope("rope-ragged-d64", 12, 32, 8, 64, 16, 3001, 701, 32, True, False, 1873, "uniform"),
        # the smallest cross attention: one short request of a small GQA 4:1 model
        _cross("cross-tiny-d64", 1, 4, 1, 64, 16, 256, 64),
        # continuous batching on a Llama-3-8B-shaped layer, encoder states and
        # texts of all lengths, some requests without an encoder input
        _cross("cross-ragged-8b", 16, 32, 8, 128, 16, 4096, 512, "ragged"),
        # long encoder states and long texts on the 70B-shaped layer
        _cross("cross-70b", 8, 64, 8, 128, 16, 8192, 1024),
        # a short question on each of two long documents
        _cross("cross-question", 2, 64, 8, 128, 64, 131072, 43),
        # the smallest batch with a prefix in common
        _shared("shared-tiny-d64", 4, 4, 1, 64, 16, 1, 256, 64, "uniform"),
        # eight conversations that began alike, 70B-shaped layer
        _shared("shared-chat-70b", 8, 64, 8, 128, 16, 1, 8192, 1024, "uniform"),
        # a busy server's system prompt, 8B-shaped layer
        _shared("shared-system-prompt-8b", 128, 32, 8, 128, 16, 1, 2048, 200, "lognormal"),
        # multi-turn traffic of several applications on the 70B-shaped layer
        _shared("shared-applications-70b", 64, 64, 8, 128, 16, 9, 2048, 600, "lognormal"),
        # questions of many users on two long documents: the largest call
        _shared("shared-documents-70b", 64, 64, 8, 128, 64, 2, 131072, 2048, "uniform"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rope", "cross", "shared", "shared"])
    d = rng.choice([64, 128, 128])
    hkv = rng.choice([1, 2, 4, 8, 8])
    hq = hkv * rng.choice([1, 2, 4, 8, 8, 16])
    ps = rng.choice([16, 16, 32, 64, 128])
    lens = rng.randrange(1 << 20)
    if kind == "rope":
        c = _rope("", _log(rng, 1, 128), hq, hkv, d, ps, _log(rng, 16, 4096), _log(rng, 1, 1024),
                  rng.choice([d, d, d // 2, 16]), rng.random() < 0.5, rng.random() < 0.5,
                  rng.choice([0, 0, 777]), rng.choice(["fixed", "uniform", "lognormal", "ragged"]),
                  lens)
    elif kind == "cross":
        c = _cross("", _log(rng, 1, 64), hq, hkv, d, ps, _log(rng, 16, 65536), _log(rng, 1, 1024),
                   rng.choice(["fixed", "uniform", "lognormal", "ragged"]), lens)
    else:
        B = _log(rng, 1, 256)
        c = _shared("", B, hq, hkv, d, ps, rng.randint(1, min(B, 12)), _log(rng, 64, 131072),
                    _log(rng, 1, 2048), rng.choice(["fixed", "uniform", "lognormal", "ragged"]),
                    lens)
    # no dearer than the largest listed case, padded to the longest request too
    while c["B"] > 1 and (work(c)["bytes"] > 1.2e9 or work(c)["flops"] > 2e12 or
                          _padded(c) > 5e9):
        c["B"] //= 2
        if kind == "shared":
            c["groups"] = min(c["groups"], c["B"])
    return c


# ---------------------------------------------------------------- lengths
def _spread(c, length, stream, least, most):
    """`B` lengths (groups of a shared case: `groups`) around `length`."""
    rng = np.random.default_rng([c["lens"], stream])
    n = c["groups"] if stream == 3 else c["B"]
    if c["spread"] == "fixed":
        return np.full(n, length, np.int64)
    if c["spread"] == "lognormal":
        x = np.rint(rng.lognormal(math.log(max(length, 1)), 0.8, size=n)).astype(np.int64)
        return np.clip(x, max(least, length // 12), min(most, 8 * length))
    x = rng.integers(max(least, length // 8), length, size=n, endpoint=True)
    if c["spread"] == "ragged" and least == 0:
        x[rng.random(n) < 0.125] = 0
    return x


def _lens(c):
    """rope: (cached, new, first position); cross: (kv, new); shared: (first
    request of each group and their number, shared, own)."""
    if c["kind"] == "rope":
        P, n = _spread(c, c["prefix"], 1, 0, 16384), _spread(c, c["new"], 2, 1, 8192)
        return P, n, P + c["placed"]
    if c["kind"] == "cross":
        return _spread(c, c["kv"], 1, 0, 131072), _spread(c, c["new"], 2, 1, 4096)
    B, groups = c["B"], c["groups"]
    if c["spread"] == "fixed":
        cu = np.arange(groups + 1, dtype=np.int64) * B // groups
    else:
        cut = np.random.default_rng([c["lens"], 4]).integers(0, B, size=groups - 1, endpoint=True)
        cu = np.concatenate([[0], np.sort(cut), [B]]).astype(np.int64)
    return cu, _spread(c, c["shared"], 3, 0, 131072), _spread(c, c["own"], 2, 1, 4096)


def _padded(c):
    """Elements of the largest tensors when every request is as long as the longest."""
    if c["kind"] == "rope":
        return 0
    if c["kind"] == "cross":
        kv, n = _lens(c)
        k = int(kv.max())
        return c["B"] * k * max(c["hq"] * int(n.max()), 2 * c["hkv"] * c["d"])
    cu, S, t = _lens(c)
    rows = int(np.diff(cu).max())
    return (c["groups"] * int(S.max()) * max(c["hq"] * rows, 2 * c["hkv"] * c["d"]) +
            c["B"] * int(t.max()) * max(c["hq"], 2 * c["hkv"] * c["d"]))


# ----------------------------------------------------------------- inputs
def _randn(gen, shape):
    return torch.randn(shape, generator=gen, device="cuda", dtype=_BF16)


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def _tables(c, seed, *lens):
    """Block tables for lists of lengths, their pages scattered over one pool,
    and the pool's number of pages (a quarter belongs to others)."""
    counts = [-(-np.asarray(n) // c["ps"]) for n in lens]
    pages = max(1, math.ceil(1.25 * sum(int(k.sum()) for k in counts)))
    perm = np.random.default_rng([int(seed) & 0x7FFFFFFF, 3]).permutation(pages)
    at, tables = 0, []
    for k in counts:
        table = np.full((len(k), max(1, int(k.max()))), -1, np.int64)
        for b, m in enumerate(k):
            table[b, :m] = perm[at:at + m]
            at += int(m)
        tables.append(table)
    return tables, pages


def _angles(n, rot):
    """[n][2][rot/2]: cosines and sines of position p, base 500000."""
    freq = 500000.0 ** (-np.arange(0, rot, 2) / rot)
    a = np.arange(n)[:, None] * freq
    return np.stack([np.cos(a), np.sin(a)], 1).astype(np.float32)


def _inputs(c, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    hq, hkv, d, ps, B = c["hq"], c["hkv"], c["d"], c["ps"], c["B"]
    x = dict(case=c)
    if c["kind"] == "shared":
        cu, S, t = _lens(c)
        (x["shared_table"], x["table"]), pages = _tables(c, seed, S, t)
        x.update(cu=cu, S=S, t=t, q=_randn(gen, (B, hq, d)))
    elif c["kind"] == "cross":
        kv, n = _lens(c)
        (x["table"],), pages = _tables(c, seed, kv)
        x.update(kv=kv, n=n, cu=np.concatenate([[0], np.cumsum(n)]))
        x["q"] = _randn(gen, (int(n.sum()), hq, d))
    else:
        P, n, first = _lens(c)
        (x["table"],), pages = _tables(c, seed, P + n)
        T = int(n.sum())
        x.update(P=P, n=n, cu=np.concatenate([[0], np.cumsum(n)]), first=first)
        if c["fused"]:
            rows = _randn(gen, (T, hq + 2 * hkv, d))
            x["q"], x["k"], x["v"] = rows[:, :hq], rows[:, hq:hq + hkv], rows[:, hq + hkv:]
        else:
            x["q"], x["k"], x["v"] = (_randn(gen, (T, h, d)) for h in (hq, hkv, hkv))
        x["angles"] = torch.from_numpy(_angles(int((first + n).max()), c["rot"])).cuda()
    x["pool"] = _randn(gen, (1, 2, pages, hkv, ps, d))
    return x


def prepare(case, seed):
    c = {k: v for k, v in case.items() if k != "name"}
    x = _inputs(c, seed)
    s = dict(c, planes=x["pool"], q=x["q"], table=_i32(x["table"]), width=x["table"].shape[1],
             scale=c["d"] ** -0.5)
    if c["kind"] == "shared":
        s.update(cu=_i32(x["cu"]), S=_i32(x["S"]), t=_i32(x["t"]), stable=_i32(x["shared_table"]),
                 swidth=x["shared_table"].shape[1], most_S=max(1, int(x["S"].max())),
                 most_t=int(x["t"].max()), rows=int(np.diff(x["cu"]).max()))
    elif c["kind"] == "cross":
        s.update(kv=_i32(x["kv"]), n=_i32(x["n"]), cu=_i32(x["cu"]), T=int(x["n"].sum()),
                 most_kv=max(1, int(x["kv"].max())), most_n=int(x["n"].max()))
    else:
        s.update(k=x["k"], v=x["v"], angles=x["angles"], P=_i32(x["P"]), cu=_i32(x["cu"]),
                 T=int(x["n"].sum()), positions=None)
        if c["placed"]:
            s["positions"] = _i32(np.concatenate([np.arange(f, f + m)
                                                  for f, m in zip(x["first"], x["n"])]))
    s["out"] = torch.zeros(x["q"].shape, dtype=_BF16, device="cuda")
    if own:
        from paper_2505_23970_gb300 import binding as gcb
        pool = gcb.KVPool.create(1, c["hkv"], c["d"], c["ps"], x["pool"].shape[2])
        pool.planes().copy_(x["pool"])
        need = 0
        if c["kind"] == "shared":
            need = gcb.gc_shared_prefix_decode_workspace_bytes(
                pool.handle, c["B"], c["groups"], s["swidth"], s["width"], c["hq"])
        elif c["kind"] == "cross":
            need = gcb.gc_paged_cross_workspace_bytes(pool.handle, c["B"], s["width"], c["hq"],
                                                      s["T"])
        s.update(pool=pool, handle=pool.handle, planes=pool.planes(), gcb=gcb, need=need,
                 stream=torch.cuda.current_stream(),
                 work=torch.empty(max(16, need), dtype=torch.uint8, device="cuda"))
    return s


# ------------------------------------------------------------- plain forms
def _pages(planes, table, keys):
    """K and V of the first `keys` slots of each table row: [n][hkv][keys][d]."""
    kv = planes[0][:, table.clamp(min=0).long()]  # [2][n][blocks][hkv][ps][d]
    kv = kv.transpose(2, 3).flatten(3, 4)[:, :, :, :keys].float()
    return kv[0], kv[1]


def _scores(q, k, lens, scale):
    """[n][hkv][rows][keys], -inf at and past each length."""
    s = torch.matmul(q, k.transpose(-1, -2)).mul_(scale)
    past = torch.arange(k.shape[2], device=k.device)[None] >= lens[:, None]
    return s.masked_fill_(past[:, None, None], -math.inf)


def _rotate(x, cos, sin, rot, interleaved):
    x = x.float()
    r, rest = x[..., :rot], x[..., rot:]
    a, b = (r[..., 0::2], r[..., 1::2]) if interleaved else (r[..., :rot // 2], r[..., rot // 2:])
    a, b = a * cos - b * sin, b * cos + a * sin
    r = torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1)
    return torch.cat([r, rest], -1)


def _plain_rope(s):
    t = torch.arange(s["T"], device="cuda")
    b = torch.searchsorted(s["cu"], t, right=True) - 1
    slot = s["P"][b] + t - s["cu"][b]
    row = s["angles"][slot if s["positions"] is None else s["positions"]]
    cos, sin = row[:, 0, None], row[:, 1, None]
    out = _rotate(s["q"], cos, sin, s["rot"], s["interleaved"]).to(_BF16)
    page = s["table"][b, slot // s["ps"]].long()
    layer, at = s["planes"][0], (slot % s["ps"]).long()
    layer[0][page, :, at] = _rotate(s["k"], cos, sin, s["rot"], s["interleaved"]).to(_BF16)
    layer[1][page, :, at] = s["v"]
    return {"q": out, "kv": s["planes"]}


def _plain_cross(s):
    B, hkv, d, T, n = s["B"], s["hkv"], s["d"], s["T"], s["most_n"]
    t = torch.arange(T, device="cuda")
    b = torch.searchsorted(s["cu"], t, right=True) - 1
    at = (s["cu"][:-1, None] + torch.arange(n, device="cuda")).clamp(max=T - 1).long()
    q = s["q"][at].float().view(B, n, hkv, -1, d).transpose(1, 2).reshape(B, hkv, -1, d)
    k, v = _pages(s["planes"], s["table"], s["most_kv"])
    p = _scores(q, k, s["kv"], s["scale"])
    m = p.amax(-1, keepdim=True)
    p = p.sub_(m.masked_fill(m == -math.inf, 0)).exp_()
    l = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / l.masked_fill(l == 0, 1)
    o = o.view(B, hkv, n, -1, d).transpose(1, 2).reshape(B, n, -1, d)
    return {"out": o[b, t - s["cu"][b]].to(_BF16)}


def _plain_shared(s):
    B, hkv, d, groups, rows = s["B"], s["hkv"], s["d"], s["groups"], s["rows"]
    r = torch.arange(B, device="cuda")
    g = torch.searchsorted(s["cu"], r, right=True) - 1
    in_group = r - s["cu"][g]
    q = s["q"].float().view(B, hkv, -1, d)
    at = (s["cu"][:-1, None] + torch.arange(rows, device="cuda")).clamp(max=B - 1).long()
    qg = q[at].transpose(1, 2).reshape(groups, hkv, -1, d)
    k, v = _pages(s["planes"], s["stable"], s["most_S"])
    ps = _scores(qg, k, s["S"], s["scale"])
    k, vo = _pages(s["planes"], s["table"], s["most_t"])
    po = _scores(q, k, s["t"], s["scale"])
    # (own lengths are at least 1, so every row has a key)
    mg = ps.amax(-1).view(groups, hkv, rows, -1)[g, :, in_group]
    m = torch.maximum(mg, po.amax(-1))
    mg = m.new_zeros(groups, rows, hkv, m.shape[-1]).index_put((g, in_group), m)
    ps = ps.sub_(mg.transpose(1, 2).reshape(groups, hkv, -1, 1)).exp_()
    po = po.sub_(m[..., None]).exp_()
    og = torch.matmul(ps, v).view(groups, hkv, rows, -1, d)[g, :, in_group]
    lg = ps.sum(-1).view(groups, hkv, rows, -1)[g, :, in_group]
    o = (og + torch.matmul(po, vo)) / (lg + po.sum(-1))[..., None]
    return {"out": o.view(B, -1, d).to(_BF16)}


# ------------------------------------------------------------------- pass
def run(s):
    kind = s["kind"]
    if not own:
        return {"rope": _plain_rope, "cross": _plain_cross, "shared": _plain_shared}[kind](s)
    gcb, h, st = s["gcb"], s["handle"], s["stream"]
    if kind == "rope":
        gcb.gc_kv_append_rope(h, s["q"], s["q"].stride(0), s["out"], s["k"], s["k"].stride(0),
                              s["v"], s["v"].stride(0), s["table"], s["P"], st, 0, s["cu"], s["B"],
                              s["width"], s["T"], s["hq"], s["angles"], s["angles"].shape[0],
                              s["rot"], s["positions"],
                              gcb.GC_ROPE_INTERLEAVED if s["interleaved"] else 0)
        return {"q": s["out"], "kv": s["planes"]}
    if kind == "cross":
        gcb.gc_paged_cross_attn(s["q"], h, s["table"], s["kv"], s["n"], s["out"], st, 0, s["cu"],
                                s["B"], s["width"], s["hq"], s["scale"], s["T"], s["work"],
                                s["need"])
    else:
        gcb.gc_shared_prefix_decode_attn(s["q"], h, s["stable"], s["S"], s["cu"], s["groups"],
                                         s["swidth"], s["table"], s["t"], s["out"], st, 0, s["B"],
                                         s["width"], s["hq"], s["scale"], s["work"], s["need"])
    return {"out": s["out"]}


def work(c):
    row = c["hkv"] * c["d"] * 2 * 2  # one token's K and V
    if c["kind"] == "rope":
        T = int(_lens(c)[1].sum())
        # q, k and v read and written, each token's angles read
        return {"bytes": T * (2 * c["hq"] * c["d"] * 2 + 2 * row + c["rot"] * 4),
                "flops": 3.0 * T * (c["hq"] + c["hkv"]) * c["rot"]}
    if c["kind"] == "cross":
        kv, n = _lens(c)
        qo = 2 * int(n.sum()) * c["hq"] * c["d"] * 2
        return {"bytes": int(kv.sum()) * row + qo,
                "flops": 4.0 * c["d"] * c["hq"] * float((kv * n).sum())}
    cu, S, t = _lens(c)
    size = np.diff(cu)
    qo = 2 * c["B"] * c["hq"] * c["d"] * 2
    return {"bytes": (int(S[size > 0].sum()) + int(t.sum())) * row + qo,
            "flops": 4.0 * c["d"] * c["hq"] * float((S * size).sum() + t.sum())}


# -------------------------------------------------------------- 64 bits
def _attend(q, k, v, scale):
    """Softmax attention of all rows to all keys: q [n][hq][d], k, v [T][hkv][d]."""
    n, hq, d = q.shape
    T, hkv, _ = k.shape
    out = torch.zeros((n, hq, d), dtype=torch.float64, device=q.device)
    if T == 0 or n == 0:
        return out
    G = hq // hkv
    step = max(1, int(4e8 / (G * T)))
    for g in range(hkv):
        kg, vg = k[:, g].double(), v[:, g].double()
        for i in range(0, n, step):
            qi = q[i:i + step, g * G:(g + 1) * G].double()
            p = torch.softmax((qi.reshape(-1, d) @ kg.T) * scale, -1)
            out[i:i + step, g * G:(g + 1) * G] = (p @ vg).view(-1, G, d)
    return out


def _sequence(c, pool, table, length):
    """K and V [length][hkv][d] of one sequence, read page by page."""
    used = torch.from_numpy(table[:-(-int(length) // c["ps"])]).cuda()
    kv = pool[0][:, used].permute(0, 1, 3, 2, 4).reshape(2, -1, c["hkv"], c["d"])
    return kv[:, :int(length)]


def exact(case, seed):
    c = {k: v for k, v in case.items() if k != "name"}
    x = _inputs(c, seed)
    pool, scale = x["pool"], c["d"] ** -0.5
    if c["kind"] == "rope":
        q, kv = x["q"].double(), pool.double()
        half = c["rot"] // 2
        for b in range(c["B"]):
            lo, n, P = int(x["cu"][b]), int(x["n"][b]), int(x["P"][b])
            f = int(x["first"][b])
            turn = torch.complex(x["angles"][f:f + n, 0].double(), x["angles"][f:f + n, 1].double())
            k = x["k"][lo:lo + n].double()
            for t in (q[lo:lo + n], k):
                if c["interleaved"]:
                    re, im = t[..., 0:c["rot"]:2], t[..., 1:c["rot"]:2]
                else:
                    re, im = t[..., :half], t[..., half:c["rot"]]
                z = torch.complex(re, im) * turn[:, None]
                re.copy_(z.real)
                im.copy_(z.imag)
            at = np.arange(P, P + n)
            page = torch.from_numpy(x["table"][b][at // c["ps"]]).cuda()
            slot = torch.from_numpy(at % c["ps"]).cuda()
            kv[0, 0, page, :, slot] = k
            kv[0, 1, page, :, slot] = x["v"][lo:lo + n].double()
        return {"q": q, "kv": kv}
    out = torch.empty(x["q"].shape, dtype=torch.float64, device="cuda")
    if c["kind"] == "cross":
        for b in range(c["B"]):
            rows = slice(int(x["cu"][b]), int(x["cu"][b + 1]))
            k, v = _sequence(c, pool, x["table"][b], x["kv"][b])
            out[rows] = _attend(x["q"][rows], k, v, scale)
        return {"out": out}
    for g in range(c["groups"]):
        first, end = int(x["cu"][g]), int(x["cu"][g + 1])
        if first == end:
            continue
        common = _sequence(c, pool, x["shared_table"][g], x["S"][g])
        for b in range(first, end):
            kv = torch.cat([common, _sequence(c, pool, x["table"][b], x["t"][b])], 1)
            out[b:b + 1] = _attend(x["q"][b:b + 1], kv[0], kv[1], scale)
    return {"out": out}
