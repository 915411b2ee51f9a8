"""Operators around the compressed cache as cases that can be timed and compared: rotary positions, attention of a batch
over a prefix that its sequences share, attention that adds up what each cached position receives, and the eviction that
goes by these sums.

  table    cos / sin of a range of positions, scaled for a long context
  rope     q, k, v of some tokens out of a projection: rounded to bf16, q and k turned to given positions
  shared   one decode step of several sequences whose first positions are one prefix, stored once
  weights  one decode step of one sequence, and the sums of attention weights per kv head and position
  evict    which positions stay, and the encoded vectors and sums of these moved to the front of a run of pages

The cache holds, per vector of 128 values, a bitmap of the K kept ones, K fields with their leading bits (raw, or sign and
magnitude under one exponent per 32 values) and, for the exact form, the dropped bits and the other values; 64 vectors of
one head are a tile, and a page table names the pages of a sequence.  Vectors are seeded stand-ins: keys with four outlier
channels per head x10, the rest normal.
"""
import math

import numpy as np
import torch

own = False

HD = 128  # values of a vector
HALF, INTERLEAVED = 0, 1
PLAIN, LINEAR, BASE, BANDS = 0, 1, 2, 3


# ---- cases ------------------------------------------------------------------------------------
def listed():
    return [
        # a decode step's five columns before attention: one launch between two others
        {"name": "rope_step", "kind": "rope", "tokens": 5, "n_q": 32, "n_kv": 8, "dim": 128, "rot": 128, "layout": HALF,
         "fp32": True, "pad": 0, "table": 8704},
        # a packed batch of prompts of a model that turns a quarter of wide heads, neighbours in pairs, padded rows
        {"name": "rope_prompt_part", "kind": "rope", "tokens": 4099, "n_q": 24, "n_kv": 8, "dim": 256, "rot": 64,
         "layout": INTERLEAVED, "fp32": False, "pad": 40, "table": 33001},
        # the table of a model taken from 8K to 128K positions
        {"name": "table_131072", "kind": "table", "rot": 128, "pos0": 0, "n": 131072, "base": 500000.0, "scaling": BANDS,
         "factor": 16.0, "trained": 8192},
        # two short conversations behind one system prompt, draft pass: latency
        {"name": "shared_pair", "kind": "shared", **_attn(8, 4), "seqs": 2, "prefix": 703, "tail": 90, "cols": 1, "new": 3,
         "full": False},
        # a serving batch behind a long system prompt, draft pass
        {"name": "shared_draft_16", "kind": "shared", **_attn(8, 4), "seqs": 16, "prefix": 8192, "tail": 500, "cols": 1,
         "new": 4, "full": False},
        # the verification of four drafts of eight sequences, prefix that ends inside a page
        {"name": "shared_verify_8", "kind": "shared", **_attn(8, 4), "seqs": 8, "prefix": 8229, "tail": 300, "cols": 5,
         "new": 5, "full": True},
        # a long document asked about by 32 users, exact pass over a cache with shared exponents, 64 query heads
        {"name": "shared_doc_32", "kind": "shared", **_attn(8, 8, form="shared"), "seqs": 32, "prefix": 32768, "tail": 200,
         "cols": 1, "new": 1, "full": True},
        # plain decoding with sums at 8K of context
        {"name": "weights_step", "kind": "weights", **_attn(8, 4), "len": 8192, "cols": 1, "new": 1, "full": True},
        # the verification of six drafts at a long context that ends inside a page
        {"name": "weights_verify", "kind": "weights", **_attn(8, 4), "len": 30011, "cols": 7, "new": 7, "full": True},
        # one layer of a short conversation cut to half
        {"name": "evict_layer", "kind": "evict", **_attn(8, 4), "layers": 1, "len": 2049, "keep_n": 1024, "first": 4,
         "last": 128},
        # all layers of an 8B-shaped model at once, 8K of context cut to a quarter
        {"name": "evict_model", "kind": "evict", **_attn(8, 4), "layers": 32, "len": 8192, "keep_n": 2048, "first": 4,
         "last": 512},
    ]


def _attn(n_kv, grp, keep=600, trunc=4, form="raw"):
    return {"n_kv": n_kv, "grp": grp, "keep": keep, "trunc": trunc, "form": form}


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rope", "rope", "table", "shared", "shared", "shared", "weights", "weights", "evict", "evict"])
    if kind == "table":
        rot, scaling = 2 * rng.randint(2, 128), rng.choice([PLAIN, LINEAR, BASE, BANDS])
        n = min(_log(rng, 1, 131072), 131072 * 64 * 2 // rot)
        return {"kind": kind, "rot": rot, "pos0": rng.choice([0, 0, rng.randint(0, 900000)]), "n": n,
                "base": rng.choice([10000.0, 500000.0, 1000000.0]), "scaling": scaling,
                "factor": 1.0 if scaling == PLAIN else round(rng.uniform(1.0, 40.0), 3),
                "trained": rng.choice([2048, 4096, 8192, 32768])}
    n_kv, grp = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 5, 7, 8])
    if kind == "rope":
        dim = rng.choice([64, 80, 96, 128, 128, 128, 256])
        rot = rng.choice([dim, dim, dim // 2, dim // 4, 2 * rng.randint(1, dim // 2)])
        rot -= rot % 2
        tokens = min(_log(rng, 1, 8192), 42_000_000 // ((n_kv * (grp + 2)) * dim))
        return {"kind": kind, "tokens": tokens, "n_q": n_kv * grp, "n_kv": n_kv, "dim": dim, "rot": rot,
                "layout": rng.choice([HALF, INTERLEAVED]), "fp32": rng.random() < 0.5,
                "pad": rng.choice([0, 0, 8, rng.randint(1, 63)]), "table": _log(rng, 64, 65536)}
    keep, trunc = rng.choice([250, 400, 500, 600, 600, 600, 700, rng.randint(100, 1000)]), rng.choice([4, 4, 4, 0, 1, 2, 3, 5, 7])
    c = {"kind": kind, **_attn(n_kv, grp, keep, trunc, rng.choice(["raw", "raw", "raw", "shared"]))}
    if kind == "evict":
        c["layers"] = rng.choice([1, 1, 2, 4, 16])
        c["len"] = _log(rng, 1, min(32768, 2_000_000 // (c["layers"] * n_kv)))
        c["keep_n"] = rng.choice([c["len"] // 2, c["len"] // 4, rng.randint(1, c["len"])])
        c["first"] = rng.randint(0, min(8, c["keep_n"]))
        c["last"] = rng.randint(0, (c["keep_n"] - c["first"]) // 2)
        return c
    c["full"] = rng.random() < 0.5
    c["cols"] = 1 if not c["full"] and rng.random() < 0.8 else rng.randint(1, min(8, (80 if c["full"] else 48) // grp))
    c["new"] = c["cols"] + rng.choice([0, 0, 1, 3])
    if kind == "weights":
        c["len"] = rng.choice([0, _log(rng, 1, 32768), _log(rng, 64, 32768)])
        return c
    c["seqs"] = _log(rng, 1, 32)
    c["tail"] = _log(rng, 1, 1000)
    c["prefix"] = rng.choice([0, _log(rng, 1, 32768), _log(rng, 64, 32768), _log(rng, 64, 32768)])
    c["prefix"] = min(c["prefix"], 70_000_000 // (c["seqs"] * c["cols"] * grp * n_kv))
    return c


# ---- the encoded cache ------------------------------------------------------------------------
def _geometry(c):
    """Words of a vector in each stream and of a tile in each pool."""
    mx, t = c["form"] == "shared", c["trunc"]
    words = lambda bits: (bits + 31) // 32  # noqa: E731
    k = (c["keep"] * HD + 500) // 1000
    g = {"mx": mx, "t": t, "k": k, "fw": 9 - t if mx else 16 - t, "lw": words(k * t), "pw": words((HD - k) * 16)}
    g["sw"] = words(k * g["fw"])
    g["off"] = 64 * (5 if mx else 4)  # words of a tile before its fields
    g["spec"] = (g["off"] + 64 * g["sw"] + 63) // 64 * 64
    g["verif"] = (64 * (g["lw"] + g["pw"]) + 63) // 64 * 64
    return g


def _pack(fields, width, n):
    """[rows, m] fields of `width` bits as [rows, n] little-endian 32-bit words."""
    rows, m = fields.shape
    out = torch.zeros(rows, n + 1, dtype=torch.int64, device=fields.device)
    if m and width:
        bit = torch.arange(m, device=fields.device) * width
        v = fields << (bit % 32)
        at = (bit // 32).expand(rows, m)
        out.scatter_add_(1, at, v & 0xFFFFFFFF)
        out.scatter_add_(1, at + 1, v >> 32)
    return out[:, :n].to(torch.int32)


def _kept(bits, k):
    """Which of the 128 values are kept: the k largest magnitudes, ties to the lower channel."""
    at = torch.sort((bits & 0x7FFF).to(torch.int16), dim=1, descending=True, stable=True).indices[:, :k]
    return torch.zeros(bits.shape, dtype=torch.bool, device=bits.device).scatter_(1, at, True)


def _magnitudes(bits, mask):
    """Shared exponent per 32 values (over the kept ones) and the kept values' 8-bit magnitudes under it."""
    exp = (bits >> 7 & 0xFF).clamp(min=1)
    sig = (bits & 0x7F) | torch.where((bits >> 7 & 0xFF) > 0, 0x80, 0)
    shared = torch.where(mask, exp, 0).view(-1, 4, 32).amax(2)
    return shared, sig >> (shared.repeat_interleave(32, 1) - exp).clamp(0, 31)


def _encode(bits, g, spec, verif):
    """Writes vectors bits [tiles * 64, 128] (bf16 patterns, int32) into tiles spec / verif [tiles, words]."""
    n, t, k = bits.shape[0], g["t"], g["k"]
    mask = _kept(bits, k)
    kept = mask.nonzero()[:, 1].view(n, k)  # ascending channels of a vector
    rest = (~mask).nonzero()[:, 1].view(n, HD - k)
    low = (1 << t) - 1
    tiles = n // 64
    bitmap = (mask.view(n, 4, 32).long() << torch.arange(32, device=bits.device)).sum(2).to(torch.int32)
    spec[:, :256] = bitmap.view(tiles, 256)
    if g["mx"]:
        shared, mag = _magnitudes(bits, mask)
        spec[:, 256:320] = (shared.long() << torch.arange(0, 32, 8, device=bits.device)).sum(1).to(torch.int32).view(tiles, 64)
        hi, lo = (bits >> 15 & 1) << (8 - t) | mag >> t, mag & low
    else:
        hi, lo = bits >> t, bits & low
    spec[:, g["off"]:g["off"] + 64 * g["sw"]] = _pack(hi.gather(1, kept).long(), g["fw"], g["sw"]).view(tiles, -1)
    verif[:, :64 * g["lw"]] = _pack(lo.gather(1, kept).long(), t, g["lw"]).view(tiles, -1)
    verif[:, 64 * g["lw"]:64 * (g["lw"] + g["pw"])] = _pack(bits.gather(1, rest).long(), 16, g["pw"]).view(tiles, -1)


def _pools(bits, g):
    """Pools with vectors bits [pages, 2, heads, 64, 128]: flat buffers as the cache wants them, views [pages, 2, heads, words]."""
    pages, _, heads = bits.shape[:3]
    tiles = pages * 2 * heads
    flat = [torch.zeros(tiles * g[p] + 64, dtype=torch.int32, device="cuda") for p in ("spec", "verif")]
    spec, verif = (f[:tiles * g[p]].view(tiles, g[p]) for f, p in zip(flat, ("spec", "verif")))
    flatbits = bits.view(tiles, 64, HD)
    for a in range(0, tiles, 1024):
        _encode(flatbits[a:a + 1024].reshape(-1, HD), g, spec[a:a + 1024], verif[a:a + 1024])
    return flat, spec.view(pages, 2, heads, -1), verif.view(pages, 2, heads, -1)


def _unpack(words, index, width):
    """Field number `index` [rows, 128] of `width` bits out of [rows, n] words."""
    if width == 0:
        return torch.zeros_like(index)
    w = torch.nn.functional.pad(words.long() & 0xFFFFFFFF, (0, 1))
    bit = index * width
    two = w.gather(1, bit >> 5) | w.gather(1, ((bit >> 5) + 1).clamp(max=w.shape[1] - 1)) << 32
    return two >> (bit & 31) & ((1 << width) - 1)


def _decode(spec, verif, g, full):
    """K and V as fp32 [2, heads, pages * 64, 128] from tiles [pages, 2, heads, words]."""
    pages, _, heads = spec.shape[:3]
    t, n = g["t"], pages * 2 * heads * 64
    part = lambda x, a, w: x[..., a:a + 64 * w].reshape(n, w)  # noqa: E731
    shift = torch.arange(32, device=spec.device)
    mask = (part(spec, 0, 4).unsqueeze(2) >> shift & 1).view(n, HD).long()
    rank = mask.cumsum(1) - mask
    last = max(g["k"] - 1, 0)
    kept = _unpack(part(spec, g["off"], g["sw"]), rank.clamp(max=last), g["fw"]) if g["k"] else torch.zeros_like(rank)
    low = _unpack(part(verif, 0, g["lw"]), rank.clamp(max=last), t) if full and t and g["k"] else 0
    if g["mx"]:
        e = (part(spec, 256, 1) >> torch.arange(0, 32, 8, device=spec.device) & 0xFF).repeat_interleave(32, 1)
        mag = ((kept & ((1 << (8 - t)) - 1)) << t | low).float()
        value = torch.ldexp(torch.where((kept >> (8 - t)) > 0, -mag, mag), (e - 134).float())
    else:
        value = ((kept << t | low) << 16).to(torch.int32).view(torch.float32)
    if full and g["k"] < HD:
        other = torch.arange(HD, device=spec.device) - rank
        other = _unpack(part(verif, 64 * g["lw"], g["pw"]), other.clamp(max=HD - g["k"] - 1), 16)
        value = torch.where(mask > 0, value, (other << 16).to(torch.int32).view(torch.float32))
    else:
        value = torch.where(mask > 0, value, 0.0)
    return value.view(pages, 2, heads, 64, HD).permute(1, 2, 0, 3, 4).reshape(2, heads, pages * 64, HD)


# ---- inputs -----------------------------------------------------------------------------------
def _rng(seed):
    r = torch.Generator(device="cuda")
    r.manual_seed(seed)
    return r


def _normal(r, *shape, sigma=1.0):
    return (torch.randn(*shape, generator=r, device="cuda") * sigma).bfloat16()


def _vectors(r, pages, heads):
    """bf16 patterns (int32) of K and V, [pages, 2, heads, 64, 128]."""
    x = torch.randn(pages, 2, heads, 64, HD, generator=r, device="cuda")
    for h in range(heads):  # four outlier channels of a head
        x[:, 0, h, :, torch.randperm(HD, generator=r, device="cuda")[:4]] *= 10.0
    return x.bfloat16().view(torch.int16).to(torch.int32) & 0xFFFF


def _layout(c, seed):
    """Pages of a case, who has which, and the vectors in them."""
    r = _rng(seed)
    seqs, prefix = c.get("seqs", 1), c.get("prefix", 0)
    if c["kind"] == "shared":  # own positions behind the prefix: ragged
        tails = torch.randint(0, c["tail"] + 1, (seqs,), generator=r, device="cuda").tolist()
        tails[0] = c["tail"]
    else:
        tails = [c["len"]]
    lens = [prefix + t for t in tails]
    common = prefix // 64
    most = max((n + c["new"] + 63) // 64 for n in lens)
    mine = most - common  # pages that each sequence has for itself
    pages = common + seqs * mine
    place = torch.randperm(pages, generator=r, device="cuda")
    table = torch.cat([place[:common].expand(seqs, common), place[common:].view(seqs, mine)], 1)
    bits = _vectors(r, pages, c["n_kv"])
    if prefix % 64:  # the page in which the sequences part holds the same vectors up to there
        at = table[:, common]
        bits[at, :, :, :prefix % 64] = bits[at[:1], :, :, :prefix % 64]
    n_q = c["n_kv"] * c["grp"]
    return {"lens": lens, "table": table, "bits": bits, "pages": pages, "q": _normal(r, seqs, c["cols"], n_q, HD, sigma=0.35),
            "kn": _normal(r, seqs, c["new"], c["n_kv"], HD), "vn": _normal(r, seqs, c["new"], c["n_kv"], HD), "r": r}


def _start(c, seed):
    """The position that a table begins with: near the case's."""
    return c["pos0"] + int(torch.randint(0, 4096, (1,), generator=_rng(seed), device="cuda"))


def prepare(case, seed):
    c, kind = dict(case), case["kind"]
    if kind == "table":
        return {**c, "pos0": _start(c, seed)}
    if kind == "rope":
        r = _rng(seed)
        width = (c["n_q"] + 2 * c["n_kv"]) * c["dim"]
        x = torch.randn(c["tokens"], width + c["pad"], generator=r, device="cuda")
        start = int(torch.randint(0, c["table"], (1,), generator=r, device="cuda"))
        # documents one after the other: positions begin again in the middle of the batch
        pos = (torch.arange(c["tokens"], device="cuda", dtype=torch.int32) + start) % c["table"]
        table = _angles({"rot": c["rot"], "pos0": 0, "n": c["table"], "base": 10000.0, "scaling": PLAIN, "factor": 1.0, "trained": 4096})
        return {**c, "x": x if c["fp32"] else x.bfloat16(), "pos": pos, "angles": table}
    if kind == "evict":
        return _prepare_evict(c, seed)
    lay = _layout(c, seed)
    g = _geometry(c)
    flat, spec, verif = _pools(lay.pop("bits"), g)
    s = {**c, **lay, "g": g, "flat": flat, "spec": spec, "verif": verif, "table": lay["table"].to(torch.int32)}
    if kind == "weights":
        n = c["len"] + c["new"]
        s["score"] = torch.empty(c["n_kv"], n, device="cuda").exponential_(1.0, generator=s["r"])
    return s


def _prepare_evict(c, seed):
    """Streams of random words: an eviction moves them as they are.  Sequence 1's pages take what stays of sequence 0."""
    r, g = _rng(seed), _geometry(c)
    src, dst = (c["len"] + 63) // 64, (c["keep_n"] + 63) // 64
    pages, tiles = src + dst, c["layers"] * (src + dst) * 2 * c["n_kv"]
    place = torch.randperm(pages, generator=r, device="cuda").to(torch.int32)
    table = torch.zeros(2, max(src, dst), dtype=torch.int32, device="cuda")
    table[0, :src], table[1, :dst] = place[:src], place[src:]
    s = {**c, "g": g, "table": table, "pages": pages}
    s["flat"] = [torch.randint(-2**31, 2**31, (tiles * g[p] + 64,), generator=r, device="cuda", dtype=torch.int32) for p in ("spec", "verif")]
    s["spec"], s["verif"] = (f[:tiles * g[p]].view(c["layers"], pages, 2, c["n_kv"], g[p]) for f, p in zip(s["flat"], ("spec", "verif")))
    # sums of attention weights: few large ones, some positions that nothing looked at, some alike
    s["score"] = torch.empty(c["layers"], c["n_kv"], c["len"], device="cuda").exponential_(1.0, generator=r) ** 3
    s["score"][torch.rand(s["score"].shape, generator=r, device="cuda") < 0.05] = 0.0
    return s


# ---- the plain forms --------------------------------------------------------------------------
def _angles(c):
    """fp32 [n, rot / 2, 2]: cos and sin of the angles, formed in 64 bits."""
    i = torch.arange(c["rot"] // 2, dtype=torch.float64, device="cuda")
    base = c["base"] * c["factor"] ** (c["rot"] / (c["rot"] - 2)) if c["scaling"] == BASE else c["base"]
    f = base ** (-2.0 * i / c["rot"])
    if c["scaling"] == LINEAR:
        f = f / c["factor"]
    if c["scaling"] == BANDS:  # by how often a channel turns within the trained context: 1 and 32 times
        part = ((c["trained"] * f / (2 * math.pi) - 1.0) / 31.0).clamp(0.0, 1.0)
        f = f * part + f / c["factor"] * (1.0 - part)
    a = (torch.arange(c["n"], dtype=torch.float64, device="cuda") + c["pos0"])[:, None] * f
    m = _magnitude(c)
    return torch.stack([a.cos() * m, a.sin() * m], 2).float()


def _magnitude(c):
    return 0.1 * math.log(c["factor"]) + 1.0 if c["scaling"] == BANDS else 1.0


def _turned(x, cs, rot, layout):
    c, s = cs[:, None, :, 0], cs[:, None, :, 1]
    y = x.clone()
    if layout == HALF:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y[..., :rot // 2], y[..., rot // 2:rot] = a * c - b * s, b * c + a * s
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y[..., 0:rot:2], y[..., 1:rot:2] = a * c - b * s, b * c + a * s
    return y


def _heads(s):
    """q, k, v as [tokens, heads, dim] in the projection."""
    q, kv = s["n_q"] * s["dim"], s["n_kv"] * s["dim"]
    return [s["x"][:, a:a + w].unflatten(1, (-1, s["dim"])) for a, w in ((0, q), (q, kv), (q + kv, kv))]


def _run_rope(s):
    q, k, v = (h.bfloat16().float() for h in _heads(s))
    cs = s["angles"][s["pos"].long()]
    return [_turned(x, cs, s["rot"], s["layout"]).bfloat16() for x in (q, k)] + [v.bfloat16()]


def _run_shared(s):
    """The prefix as one product for the queries of all sequences, what follows it sequence by sequence in a batch."""
    S, C, G, H, N = s["seqs"], s["cols"], s["grp"], s["n_kv"], s["new"]
    K, V = (x.view(H, s["pages"], 64, HD) for x in _decode(s["spec"], s["verif"], s["g"], s["full"]))
    table, common = s["table"].long(), s["prefix"] // 64
    front = [x[:, table[0, :common]].reshape(H, -1, HD) for x in (K, V)]
    back = [x[:, table[:, common:]].permute(1, 0, 2, 3, 4).reshape(S, H, -1, HD) for x in (K, V)]
    new = [x.float().transpose(1, 2) for x in (s["kn"], s["vn"])]
    q = s["q"].float().view(S, C, H, G, HD).permute(0, 2, 1, 3, 4).reshape(S, H, C * G, HD) / math.sqrt(HD)
    qa = q.transpose(0, 1).reshape(H, S * C * G, HD)
    scores = [(qa @ front[0].transpose(1, 2)).view(H, S, C * G, -1).transpose(0, 1),
              q @ torch.cat([back[0], new[0]], 2).transpose(2, 3)]
    there = torch.arange(back[0].shape[2], device="cuda") + common * 64 < torch.tensor(s["lens"], device="cuda")[:, None]
    seen = torch.arange(N, device="cuda") <= torch.arange(C, device="cuda")[:, None] + N - C
    seen = seen.repeat_interleave(G, 0)[None, None].expand(S, 1, C * G, N)
    scores[1] = scores[1].masked_fill(~torch.cat([there[:, None, None, :].expand(S, 1, C * G, -1), seen], 3), -math.inf)
    p = torch.cat(scores, 3)
    p = (p - p.amax(3, keepdim=True)).exp()
    p = p / p.sum(3, keepdim=True)
    n = common * 64
    o = (p[..., :n].transpose(0, 1).reshape(H, S * C * G, n) @ front[1]).view(H, S, C * G, HD).transpose(0, 1)
    o = o + p[..., n:] @ torch.cat([back[1], new[1]], 2)
    return o.view(S, H, C, G, HD).permute(0, 2, 1, 3, 4).reshape(S, C, H * G, HD).bfloat16()


def _run_weights(s):
    C, G, H, N, n = s["cols"], s["grp"], s["n_kv"], s["new"], s["len"]
    K, V = _decode(s["spec"], s["verif"], s["g"], s["full"]).view(2, H, s["pages"], 64, HD)[:, :, s["table"][0].long()].reshape(2, H, -1, HD)
    K, V = (torch.cat([x[:, :n], y[0].float().transpose(0, 1)], 1) for x, y in ((K, s["kn"]), (V, s["vn"])))
    q = s["q"][0].float().view(C, H, G, HD).transpose(0, 1).reshape(H, C * G, HD)
    p = q @ K.transpose(1, 2) / math.sqrt(HD)
    seen = torch.arange(n + N, device="cuda") <= torch.arange(C, device="cuda")[:, None] + n + N - C
    p = p.masked_fill(~seen.repeat_interleave(G, 0), -math.inf)
    p = (p - p.amax(2, keepdim=True)).exp()
    p = p / p.sum(2, keepdim=True)
    o = (p @ V).view(H, C, G, HD).transpose(0, 1).reshape(C, H * G, HD).bfloat16()
    w = p.sum(1)
    w[:, :n] += s["score"][:, :n]
    return [o, w]


def _run_evict(s):
    L, H, n, k, a, b = s["layers"], s["n_kv"], s["len"], s["keep_n"], s["first"], s["last"]
    score = s["score"]
    rank = score.clone()  # the first and the last ones before all others
    rank[..., :a], rank[..., n - b:] = math.inf, math.inf
    index = torch.sort(rank, dim=2, descending=True, stable=True).indices[..., :k].sort(2).values
    table = s["table"].long()
    page, row = table[0][index // 64], index % 64
    to, at = table[1][torch.arange(k, device="cuda") // 64], torch.arange(k, device="cuda") % 64
    lay, kv, head = (torch.arange(x, device="cuda") for x in (L, 2, H))
    lay, kv, head = lay[:, None, None, None], kv[None, :, None, None], head[None, None, :, None]
    g = s["g"]
    _move(s["spec"], 0, 4, lay, kv, head, page, row, to, at)
    if g["mx"]:
        _move(s["spec"], 256, 1, lay, kv, head, page, row, to, at)
    _move(s["spec"], g["off"], g["sw"], lay, kv, head, page, row, to, at)
    _move(s["verif"], 0, g["lw"], lay, kv, head, page, row, to, at)
    _move(s["verif"], 64 * g["lw"], g["pw"], lay, kv, head, page, row, to, at)
    return [index.to(torch.int32), score.gather(2, index), *_evicted(s)]


def _move(pool, off, w, lay, kv, head, page, row, to, at):
    """One stream (w words of a vector from word `off` of a tile on) of the kept vectors to the front of the new pages."""
    if w:
        part = pool[..., off:off + 64 * w].unflatten(-1, (64, w))
        part[lay, to, kv, head, at] = part[lay, page[:, None], kv, head, row[:, None]]


def _evicted(s):
    """The tiles of the new pages, rows that nothing was written to included."""
    dst = s["table"][1, :(s["keep_n"] + 63) // 64].long()
    return [s["spec"][:, dst], s["verif"][:, dst]]


# ---- the framework's calls --------------------------------------------------------------------
def _handles(s, layers=1):
    """The context and the cache object that a program keeps, made on the first pass."""
    from paper_2605_26558_amd import binding as B
    if "ctx" not in s:
        size = 0
        if s["kind"] in ("shared", "weights", "evict"):
            s["ctx"] = B.Context()
            s["kv"] = B.KVCache(s["ctx"], layers, s["n_kv"], s["pages"], *s["table"].shape, keep_permille=s["keep"], trunc_bits=s["trunc"],
                                page_table=s["table"], exp_mode=B.CAS_EXP_SHARED if s["g"]["mx"] else B.CAS_EXP_RAW,
                                spec_pool=s["flat"][0], verif_pool=s["flat"][1])
            for i, n in enumerate(s.get("lens", [s.get("len")])):
                B.cas_kv_set_len(s["kv"], i, n)
            n_q = s["n_kv"] * s["grp"]
            if s["kind"] == "shared":
                size = B.cas_attention_shared_bytes(s["kv"], range(s["seqs"]), s["prefix"], [s["cols"]] * s["seqs"], n_q, [s["new"]] * s["seqs"])
            if s["kind"] == "weights":
                size = B.cas_attention_weights_bytes(s["kv"], 0, s["cols"], n_q, s["new"])
        s["ctx"] = B.Context(workspace=torch.empty(max(size, 256), dtype=torch.uint8, device="cuda"))
    return B, s["ctx"], s.get("kv")


def _own_table(s):
    B, ctx, _ = _handles(s)
    mode = (B.CAS_ROPE_PLAIN, B.CAS_ROPE_LINEAR, B.CAS_ROPE_BASE, B.CAS_ROPE_BANDS)[s["scaling"]]
    cfg = B.cas_rope_cfg(s["rot"], mode, s["base"], s["factor"], s["trained"], 1.0, 32.0, _magnitude(s))
    return B.cas_rope_table(ctx, cfg, s["pos0"], s["n"])


def _own_rope(s):
    B, ctx, _ = _handles(s)
    ys = B.cas_rope(ctx, s["angles"], _heads(s), pos=s["pos"], layout=(B.CAS_ROPE_HALF, B.CAS_ROPE_INTERLEAVED)[s["layout"]],
                    turn=(True, True, False))
    return [y.view(torch.bfloat16) for y in ys]


def _own_shared(s):
    B, ctx, kv = _handles(s)
    o = torch.empty_like(s["q"])
    B.cas_attention_shared(ctx, kv, 0, range(s["seqs"]), s["prefix"], s["full"], s["q"].unbind(0), s["kn"].unbind(0), s["vn"].unbind(0),
                           outs=o.unbind(0))
    return o


def _own_weights(s):
    B, ctx, kv = _handles(s)
    o, w = B.cas_attention_weights(ctx, kv, 0, 0, s["full"], s["q"][0], s["kn"][0], s["vn"][0], s["score"])
    return [o, w]


def _own_evict(s):
    B, ctx, kv = _handles(s, s["layers"])
    rows = s["score"].flatten(0, 1)
    kept = torch.empty(rows.shape[0], s["keep_n"], device="cuda")
    index = B.cas_kv_select(ctx, rows, s["len"], s["keep_n"], s["first"], s["last"], kept=kept)
    index = index.view(s["layers"], s["n_kv"], s["keep_n"])
    B.cas_kv_evict(ctx, kv, 0, s["layers"], 0, 1, index)
    return [index, kept.view(index.shape), *_evicted(s)]


def run(state):
    kind = state["kind"]
    if own:
        return {"table": _own_table, "rope": _own_rope, "shared": _own_shared, "weights": _own_weights, "evict": _own_evict}[kind](state)
    return {"table": _angles, "rope": _run_rope, "shared": _run_shared, "weights": _run_weights, "evict": _run_evict}[kind](state)


def work(case):
    c, kind = case, case["kind"]
    if kind == "table":
        n = c["n"] * c["rot"]
        return {"bytes": 4 * n, "flops": 3 * n}
    if kind == "rope":
        x = c["tokens"] * (c["n_q"] + 2 * c["n_kv"]) * c["dim"]
        turned = c["tokens"] * (c["n_q"] + c["n_kv"]) * c["rot"]
        return {"bytes": x * (6 if c["fp32"] else 4) + c["tokens"] * 4 + 4 * min(c["tokens"], c["table"]) * c["rot"], "flops": 3 * turned}
    g = _geometry(c)
    vector = 4 * (g["off"] // 64 + g["sw"] + g["lw"] + g["pw"])
    if kind == "evict":
        rows = c["layers"] * c["n_kv"]
        return {"bytes": rows * (4 * c["len"] + c["keep_n"] * (8 + 4 * vector)), "flops": 2 * rows * c["len"]}
    if not c["full"]:
        vector = 4 * (g["off"] // 64 + g["sw"])
    heads, rows = c["n_kv"], c["cols"] * c["grp"] * c["n_kv"]
    if kind == "weights":
        n = c["len"] + c["new"]
        return {"bytes": 2 * heads * (c["len"] * vector + c["new"] * 256) + rows * 512 + heads * (8 * c["len"] + 4 * c["new"]),
                "flops": rows * n * (4 * HD + 2)}
    tail = c["seqs"] * c["tail"] // 2  # on average
    return {"bytes": 2 * heads * ((c["prefix"] + tail) * vector + c["seqs"] * c["new"] * 256) + c["seqs"] * rows * 512,
            "flops": rows * (c["seqs"] * (c["prefix"] + c["new"]) + tail) * 4 * HD}


# ---- the operators' definitions in 64 bits ----------------------------------------------------
def _f64(bits):
    return (bits << 16).to(torch.int32).view(torch.float32).double()


def _dense(bits, c):
    """The values that the cache stands for, in 64 bits, from the vectors themselves: [pages, 2, heads, 64, 128]."""
    g = _geometry(c)
    flat = bits.reshape(-1, HD)
    mask = _kept(flat, g["k"])
    cut = 0 if c["full"] else (1 << g["t"]) - 1
    if g["mx"]:
        shared, mag = _magnitudes(flat, mask)
        v = (mag & ~cut).double() * 2.0 ** (shared.repeat_interleave(32, 1).double() - 134.0)
        v = torch.where(flat >> 15 > 0, -v, v)
    else:
        v = _f64(flat & ~cut)
    return torch.where(mask, v, _f64(flat) if c["full"] else 0.0).view(bits.shape)


def _exact_rope(case, seed):
    s = prepare(case, seed)
    f = 10000.0 ** (-2.0 * torch.arange(s["rot"] // 2, dtype=torch.float64, device="cuda") / s["rot"])
    z = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), s["pos"].double()[:, None] * f)[:, None]  # turns as complex numbers
    out = []
    for i, h in enumerate(_heads(s)):
        x = h.bfloat16().double()
        if i < 2:
            r = s["rot"]
            a = x[..., :r].unflatten(-1, (2, r // 2) if s["layout"] == HALF else (r // 2, 2))
            pair = -2 if s["layout"] == HALF else -1
            w = torch.complex(*a.unbind(pair)) * z
            x = torch.cat([torch.stack([w.real, w.imag], pair).flatten(-2), x[..., r:]], -1)
        out.append(x)
    return out


def _exact_table(case, seed):
    c = {**case, "pos0": _start(case, seed)}
    out = torch.empty(c["n"], c["rot"] // 2, 2, dtype=torch.float64, device="cuda")
    pos = torch.arange(c["pos0"], c["pos0"] + c["n"], dtype=torch.float64, device="cuda")
    base, m = c["base"], 1.0
    if c["scaling"] == BASE:
        base *= c["factor"] ** (c["rot"] / (c["rot"] - 2))
    if c["scaling"] == BANDS:
        m += 0.1 * math.log(c["factor"])
    for i in range(c["rot"] // 2):
        f = math.exp(-2.0 * i / c["rot"] * math.log(base))
        if c["scaling"] == LINEAR:
            f /= c["factor"]
        if c["scaling"] == BANDS:
            g = min(1.0, max(0.0, (c["trained"] * f / (2 * math.pi) - 1.0) / 31.0))
            f *= g + (1.0 - g) / c["factor"]
        w = m * torch.polar(torch.ones_like(pos), pos * f)
        out[:, i, 0], out[:, i, 1] = w.real, w.imag
    return out


def _exact_attention(case, seed):
    """Sequence by sequence and head by head, softmax in 64 bits."""
    c = case
    lay = _layout(c, seed)
    dense = _dense(lay["bits"], c)
    S, C, G, H, N = c.get("seqs", 1), c["cols"], c["grp"], c["n_kv"], c["new"]
    out = torch.empty(S, C, H * G, HD, dtype=torch.float64, device="cuda")
    weights = []
    for s in range(S):
        n = lay["lens"][s]
        kv = dense[lay["table"][s]]
        for h in range(H):
            k, v = (torch.cat([kv[:, i, h].reshape(-1, HD)[:n], lay[x][s, :, h].double()]) for i, x in ((0, "kn"), (1, "vn")))
            total = torch.zeros(n + N, dtype=torch.float64, device="cuda")
            for col in range(C):
                m = n + N - C + col + 1
                p = torch.softmax(lay["q"][s, col, h * G:(h + 1) * G].double() @ k[:m].T / HD ** 0.5, 1)
                out[s, col, h * G:(h + 1) * G] = p @ v[:m]
                total[:m] += p.sum(0)
            weights.append(total)
    if c["kind"] == "shared":
        return out
    w = torch.stack(weights)
    score = torch.empty(H, c["len"] + N, device="cuda").exponential_(1.0, generator=lay["r"]).double()
    w[:, :c["len"]] += score[:, :c["len"]]
    return [out[0], w]


def _exact_evict(case, seed):
    """The sums that stay; the rest are whole numbers and words that are moved as they are."""
    score = prepare(case, seed)["score"].double().cpu().numpy()
    n, a, b = case["len"], case["first"], case["last"]
    at = np.arange(n)
    middle = np.broadcast_to((at >= a) & (at < n - b), score.shape)
    order = np.lexsort((np.broadcast_to(at, score.shape), -score, middle), axis=-1)
    index = np.sort(order[..., :case["keep_n"]], axis=-1)
    return [None, torch.from_numpy(np.take_along_axis(score, index, -1)), None, None]


def exact(case, seed):
    if case["kind"] == "table":
        return _exact_table(case, seed)
    if case["kind"] == "rope":
        return _exact_rope(case, seed)
    if case["kind"] == "evict":
        return _exact_evict(case, seed)
    return _exact_attention(case, seed)
