"""Operators of one sampled speculative round over the compressed cache, as cases that can be timed and compared: appending
with the position rotation on the way, attention within a window with a few first tokens that stay visible, and the
verification of drafted tokens against the target's probabilities from given random numbers.

  append   q, k, v of some tokens of several sequences out of a projection: rounded to bf16, q and k turned to given
           positions, q written dense, k and v encoded into the pages of their sequences
  window   one decode step of several sequences of which a column sees the first few positions and the last `window`
  accept   per sequence, how many drafted tokens are kept and which token follows them: r <= p / q at a drafted token,
           and a draw from max(0, p - q) behind the first that is not kept, from p behind the last

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


# ---- cases ------------------------------------------------------------------------------------
def listed():
    return [
        # three accepted tokens of one conversation: the smallest call, once per layer of a round
        {"name": "append_round", "kind": "append", **_cache(8), "n_q": 32, "tokens": "3", "len": 8190, "rot": 128, "layout": HALF, "fp32": True},
        # a round of a serving batch: one to six tokens a sequence, a quarter of the channels turns, neighbours in pairs
        {"name": "append_batch", "kind": "append", **_cache(8, form="shared"), "n_q": 64, "tokens": _texts(1 + i * 7 % 6 for i in range(32)), "len": 5003,
         "rot": 32, "layout": INTERLEAVED, "fp32": True},
        # a long prompt that goes on behind 1021 positions
        {"name": "append_prompt", "kind": "append", **_cache(8), "n_q": 32, "tokens": "4099", "len": 1021, "rot": 128, "layout": HALF, "fp32": True},
        # prompts of several users, bf16 heads, no queries wanted (they are turned elsewhere)
        {"name": "append_prompts", "kind": "append", **_cache(8), "n_q": 0, "tokens": "1500 1 2049 64 900 3333 129", "len": 300, "rot": 96,
         "layout": HALF, "fp32": False},
        # one conversation, draft pass within a short window: latency
        {"name": "window_step", "kind": "window", **_cache(8), "grp": 4, "seqs": 1, "len": 20011, "window": 1024, "first": 4, "cols": 1, "new": 3,
         "full": False},
        # the verification of six drafts of one conversation
        {"name": "window_verify", "kind": "window", **_cache(8), "grp": 4, "seqs": 1, "len": 30011, "window": 4096, "first": 4, "cols": 7, "new": 7,
         "full": True},
        # a serving batch, draft pass, some sequences still shorter than the window
        {"name": "window_batch", "kind": "window", **_cache(8), "grp": 4, "seqs": 16, "len": 9000, "window": 4096, "first": 64, "cols": 1, "new": 2,
         "full": False},
        # the verification of four drafts of a batch, 64 query heads, cache with shared exponents
        {"name": "window_batch_verify", "kind": "window", **_cache(8, form="shared"), "grp": 8, "seqs": 16, "len": 60000, "window": 8192, "first": 128,
         "cols": 5, "new": 5, "full": True},
        # four drafts of one conversation, a small vocabulary: latency
        {"name": "accept_one", "kind": "accept", "vocab": 32000, "drafts": "4", "known": True, "cold": 0},
        # a serving batch, ragged drafts, every fifth sequence greedy
        {"name": "accept_batch", "kind": "accept", "vocab": 128256, "drafts": _texts(2 + i * 5 % 6 for i in range(32)), "known": True, "cold": 5},
        # no drafts: a token of each sequence drawn from its logits, as drafting by sampling does
        {"name": "accept_draw", "kind": "accept", "vocab": 128256, "drafts": _texts([0] * 64), "known": True, "cold": 0},
        # drafts looked up in the prompt, so certain; odd vocabulary
        {"name": "accept_lookup", "kind": "accept", "vocab": 50257, "drafts": _texts([7] * 8), "known": False, "cold": 0},
    ]


def _cache(n_kv, keep=600, trunc=4, form="raw"):
    return {"n_kv": n_kv, "keep": keep, "trunc": trunc, "form": form}


def _texts(numbers):
    return " ".join(str(n) for n in numbers)


def _numbers(c):
    """A case with its numbers of tokens or drafts, one for each sequence, as lists."""
    return {**c, **{x: [int(n) for n in c[x].split()] for x in ("tokens", "drafts") if x in c}}


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "window", "window", "accept"])
    if kind == "accept":
        seqs, known = _log(rng, 1, 64), rng.random() < 0.7
        vocab = rng.choice([_log(rng, 1000, 160000), _log(rng, 1000, 160000), 32000, 128256])
        most = rng.choice([0, 1, 4, 7, 12])
        drafts = [rng.randint(0, most) for _ in range(seqs)]
        while (sum(drafts) * (2 if known else 1) + len(drafts)) * vocab > 40_000_000:
            drafts = drafts[:len(drafts) // 2]
        return {"kind": kind, "vocab": vocab, "drafts": _texts(drafts), "known": known, "cold": rng.choice([0, 0, 2, 5])}
    n_kv, grp = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 5, 7, 8])
    keep, trunc = rng.choice([250, 400, 500, 600, 600, 600, 700, rng.randint(100, 1000)]), rng.choice([4, 4, 4, 0, 1, 2, 3, 5, 7])
    c = {"kind": kind, **_cache(n_kv, keep, trunc, rng.choice(["raw", "raw", "raw", "shared"]))}
    if kind == "append":
        total = _log(rng, 1, 6500)
        seqs = min(_log(rng, 1, 32), total)
        cuts = sorted(rng.randint(0, total) for _ in range(seqs - 1))  # of equal ones, a sequence without tokens
        c["tokens"] = _texts(b - a for a, b in zip([0] + cuts, cuts + [total]))
        c["n_q"] = rng.choice([0, n_kv * grp, n_kv * grp])
        c["len"] = rng.choice([0, _log(rng, 1, 30000)])
        c["rot"] = rng.choice([128, 128, 64, 32, 2 * rng.randint(1, 64)])
        c["layout"], c["fp32"] = rng.choice([HALF, INTERLEAVED]), rng.random() < 0.6
        return c
    c["grp"], c["full"] = grp, rng.random() < 0.5
    c["cols"] = 1 if not c["full"] and rng.random() < 0.8 else rng.randint(1, 8)
    c["new"] = c["cols"] + rng.choice([0, 0, 1, 3])
    c["seqs"] = _log(rng, 1, 32)
    c["len"] = rng.choice([_log(rng, 1, 100000), _log(rng, 1000, 100000)])
    c["first"] = rng.choice([0, 4, 64, _log(rng, 1, 300)])
    most = min(800_000 // (c["seqs"] * n_kv), 40_000_000 // (c["seqs"] * c["cols"] * grp * n_kv))
    c["window"] = min(rng.choice([_log(rng, 1, 8192), _log(rng, 256, 8192), 4096]), max(1, most - c["first"]))
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


def _streams(bits, g):
    """The streams of vectors bits [n, 128] (bf16 patterns, int32): bitmap, exponents, fields, dropped bits, other values."""
    n, t, k = bits.shape[0], g["t"], g["k"]
    mask = _kept(bits, k)
    kept = mask.nonzero()[:, 1].view(n, k)  # ascending channels of a vector
    rest = (~mask).nonzero()[:, 1].view(n, HD - k)
    low = (1 << t) - 1
    bitmap = (mask.view(n, 4, 32).long() << torch.arange(32, device=bits.device)).sum(2).to(torch.int32)
    exps = None
    if g["mx"]:
        shared, mag = _magnitudes(bits, mask)
        exps = (shared.long() << torch.arange(0, 32, 8, device=bits.device)).sum(1, keepdim=True).to(torch.int32)
        hi, lo = (bits >> 15 & 1) << (8 - t) | mag >> t, mag & low
    else:
        hi, lo = bits >> t, bits & low
    return (bitmap, exps, _pack(hi.gather(1, kept).long(), g["fw"], g["sw"]), _pack(lo.gather(1, kept).long(), t, g["lw"]),
            _pack(bits.gather(1, rest).long(), 16, g["pw"]))


def _rows(pool, off, w):
    """One stream of the tiles of a pool, w words of a vector from word `off` of a tile on: [..., 64, w]."""
    return pool[..., off:off + 64 * w].unflatten(-1, (64, w))


def _placed(g, spec, verif):
    """Where the streams that _streams gives lie in tiles."""
    return (_rows(spec, 0, 4), _rows(spec, 256, 1), _rows(spec, g["off"], g["sw"]), _rows(verif, 0, g["lw"]), _rows(verif, 64 * g["lw"], g["pw"]))


def _pools(tiles, g, fill=None):
    """Flat buffers as the cache wants them, and their tiles [tiles, words]: zeros, or random words of a generator."""
    flat = []
    for p in ("spec", "verif"):
        n = tiles * g[p] + 64
        flat.append(torch.zeros(n, dtype=torch.int32, device="cuda") if fill is None else
                    torch.randint(-2**31, 2**31, (n,), generator=fill, device="cuda", dtype=torch.int32))
    return flat, *(f[:tiles * g[p]].view(tiles, g[p]) for f, p in zip(flat, ("spec", "verif")))


def _encoded(bits, g):
    """Pools with vectors bits [pages, 2, heads, 64, 128]: flat buffers, and tiles [pages, 2, heads, words]."""
    pages, _, heads = bits.shape[:3]
    tiles = pages * 2 * heads
    flat, spec, verif = _pools(tiles, g)
    vectors = bits.view(tiles, 64, HD)
    for a in range(0, tiles, 2048):
        part = slice(a, min(a + 2048, tiles))
        for to, x in zip(_placed(g, spec[part], verif[part]), _streams(vectors[part].reshape(-1, HD), g)):
            if x is not None and x.numel():
                to.copy_(x.view(to.shape))
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
    """fp32 [tiles, 64, 128] from tiles [tiles, words]."""
    tiles = spec.shape[0]
    t, n = g["t"], tiles * 64
    bitmap, exps, fields, dropped, others = (x.reshape(n, x.shape[-1]) for x in _placed(g, spec, verif))
    shift = torch.arange(32, device=spec.device)
    mask = (bitmap.unsqueeze(2) >> shift & 1).view(n, HD).long()
    rank = mask.cumsum(1) - mask
    last = max(g["k"] - 1, 0)
    kept = _unpack(fields, rank.clamp(max=last), g["fw"]) if g["k"] else torch.zeros_like(rank)
    low = _unpack(dropped, rank.clamp(max=last), t) if full and t and g["k"] else 0
    if g["mx"]:
        e = (exps >> torch.arange(0, 32, 8, device=spec.device) & 0xFF).repeat_interleave(32, 1)
        mag = ((kept & ((1 << (8 - t)) - 1)) << t | low).float()
        value = torch.ldexp(torch.where((kept >> (8 - t)) > 0, -mag, mag), (e - 134).float())
    else:
        value = ((kept << t | low) << 16).to(torch.int32).view(torch.float32)
    if full and g["k"] < HD:
        other = torch.arange(HD, device=spec.device) - rank
        other = _unpack(others, other.clamp(max=HD - g["k"] - 1), 16)
        value = torch.where(mask > 0, value, (other << 16).to(torch.int32).view(torch.float32))
    else:
        value = torch.where(mask > 0, value, 0.0)
    return value.view(tiles, 64, HD)


# ---- inputs -----------------------------------------------------------------------------------
def _rng(seed):
    r = torch.Generator(device="cuda")
    r.manual_seed(seed)
    return r


def _normal(r, *shape, sigma=1.0):
    return (torch.randn(*shape, generator=r, device="cuda") * sigma).bfloat16()


def _lens(c):
    """Committed positions of the sequences of a case: the first has all, the others between half and all."""
    n = len(c["tokens"]) if c["kind"] == "append" else c["seqs"]
    return [c["len"] - i * 1237 % (c["len"] // 2 + 1) for i in range(n)]


def _tables(pages, ends, r):
    """A page table from each sequence's list of the pages that a call touches and its last position, and how many pages there
    are.  The other pages of a sequence have been given back: their entries name pages that are others' by now."""
    n = sum(len(p) for p in pages)
    place = torch.randperm(max(n, 1), generator=r, device="cuda").tolist()
    table = torch.zeros(len(pages), (max(ends) + 63) // 64 + 1, dtype=torch.int32)
    at = 0
    for s, mine in enumerate(pages):
        for p in mine:
            table[s, p] = place[at]
            at += 1
    return table.cuda(), max(n, 1)


def _angles(n, rot):
    """fp32 [n, rot / 2, 2]: cos and sin of the angles of n positions, formed in 64 bits."""
    f = 500000.0 ** (-2.0 * torch.arange(rot // 2, dtype=torch.float64, device="cuda") / rot)
    a = torch.arange(n, dtype=torch.float64, device="cuda")[:, None] * f
    return torch.stack([a.cos(), a.sin()], 2).float()


def _prepare_append(c, seed):
    r, g, lens = _rng(seed), _geometry(c), _lens(c)
    total = sum(c["tokens"])
    table, pages = _tables([range(a // 64, (a + n + 63) // 64 if n else a // 64) for a, n in zip(lens, c["tokens"])],
                           [a + n for a, n in zip(lens, c["tokens"])], r)
    flat, spec, verif = _pools(pages * 2 * c["n_kv"], g, r)
    # what a sequence has been through before may have been cut: positions run ahead of the places
    ahead = [int(x) for x in torch.randint(0, 500, (len(lens),), generator=r, device="cuda")]
    pos = torch.cat([torch.arange(n) + a + b for a, b, n in zip(lens, ahead, c["tokens"])]).to(torch.int32).cuda()
    x = torch.randn(total, c["n_q"] + 2 * c["n_kv"], HD, generator=r, device="cuda")
    for h in range(c["n_kv"]):  # four outlier channels of a head's keys
        x[:, c["n_q"] + h, torch.randperm(HD, generator=r, device="cuda")[:4]] *= 10.0
    x = x.view(total, -1)
    return {**c, "g": g, "lens": lens, "table": table, "pages": pages, "flat": flat, "spec": spec.view(pages, 2, c["n_kv"], -1),
            "verif": verif.view(pages, 2, c["n_kv"], -1), "pos": pos, "x": x if c["fp32"] else x.bfloat16(),
            "angles": _angles(max(lens) + max(c["tokens"]) + 500, c["rot"])}


def _visible(c, n):
    """Pages that some column of a sequence of n committed positions sees."""
    total = n + c["new"]
    lowest = max(0, total - c["cols"] - c["window"] + 1)
    return sorted(set(range(min((c["first"] + 63) // 64, (total + 63) // 64))) | set(range(lowest // 64, (total + 63) // 64)))


def _layout(c, seed):
    """Pages of a case, who has which, and the vectors in them."""
    r, lens = _rng(seed), _lens(c)
    seen = [_visible(c, n) for n in lens]
    table, pages = _tables(seen, [n + c["new"] for n in lens], r)
    x = torch.randn(pages, 2, c["n_kv"], 64, HD, generator=r, device="cuda")
    for h in range(c["n_kv"]):
        x[:, 0, h, :, torch.randperm(HD, generator=r, device="cuda")[:4]] *= 10.0
    S = c["seqs"]
    return {"lens": lens, "seen": seen, "table": table, "pages": pages, "bits": x.bfloat16().view(torch.int16).to(torch.int32) & 0xFFFF,
            "q": _normal(r, S, c["cols"], c["n_kv"] * c["grp"], HD, sigma=0.35), "kn": _normal(r, S, c["new"], c["n_kv"], HD),
            "vn": _normal(r, S, c["new"], c["n_kv"], HD)}


def _prepare_accept(c, seed):
    r, V, drafts = _rng(seed), c["vocab"], c["drafts"]
    n, S = sum(drafts), len(drafts)
    target = torch.randn(n + S, V, generator=r, device="cuda") * 2.5
    # what a grammar or a filter rules out; every row keeps some tokens
    target[torch.rand(n + S, V, generator=r, device="cuda") < 0.03] = -math.inf
    temp = torch.rand(S, generator=r, device="cuda") * 0.7 + 0.5
    if c["cold"]:
        temp[c["cold"] - 1::c["cold"]] = 0.0
    rows = _draft_rows(drafts)  # of the target, for each drafted token
    near = torch.empty(n, V, device="cuda")
    if n:  # the draft model's logits are the target's, a little off
        torch.randn(n, V, generator=r, device="cuda", out=near)
        near.mul_(0.5).add_(target[rows])
    t = temp.repeat_interleave(torch.tensor(drafts, device="cuda")).double()[:, None]
    tokens = torch.empty(0, dtype=torch.int32, device="cuda")
    if n:
        hot = torch.softmax(near.double() / t.clamp(min=1e-3), 1).float()
        tokens = torch.where(t[:, 0] > 0, torch.multinomial(hot, 1, generator=r)[:, 0], near.argmax(1)).to(torch.int32)
    return {**c, "target": target, "near": near if c["known"] else None, "tokens": tokens, "temp": temp,
            "r": torch.rand(n + S, generator=r, device="cuda", dtype=torch.float64)}


def _draft_rows(drafts):
    """Rows of the target's logits that judge the drafted tokens: a sequence's drafts, then one row behind the last."""
    return torch.tensor([i + s for s, i in zip([s for s, k in enumerate(drafts) for _ in range(k)], range(sum(drafts)))], dtype=torch.int64, device="cuda")


def prepare(case, seed):
    c = _numbers(case)
    if c["kind"] == "accept":
        return _prepare_accept(c, seed)
    if c["kind"] == "append":
        return _prepare_append(c, seed)
    lay = _layout(c, seed)
    g = _geometry(c)
    flat, spec, verif = _encoded(lay.pop("bits"), g)
    return {**c, **lay, "g": g, "flat": flat, "spec": spec, "verif": verif}


# ---- the plain forms --------------------------------------------------------------------------
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
    q, kv = s["n_q"] * HD, s["n_kv"] * HD
    return [s["x"][:, a:a + w].unflatten(1, (w // HD, HD)) for a, w in ((0, q), (q, kv), (q + kv, kv))]


def _run_append(s):
    q, k, v = (h.bfloat16().float() for h in _heads(s))
    cs = s["angles"][s["pos"].long()]
    q, k, v = _turned(q, cs, s["rot"], s["layout"]).bfloat16(), _turned(k, cs, s["rot"], s["layout"]).bfloat16(), v.bfloat16()
    vec = torch.stack([k, v], 1)  # [tokens, 2, heads, 128]
    bits = vec.view(torch.int16).to(torch.int32) & 0xFFFF
    place = torch.cat([torch.arange(n, device="cuda") + a for a, n in zip(s["lens"], s["tokens"])])
    seq = torch.repeat_interleave(torch.arange(len(s["tokens"]), device="cuda"), torch.tensor(s["tokens"], device="cuda"))
    page = s["table"][seq, place // 64].long()[:, None, None]
    kv, head = torch.arange(2, device="cuda")[None, :, None], torch.arange(s["n_kv"], device="cuda")[None, None, :]
    row = (place % 64)[:, None, None]
    for to, x in zip(_placed(s["g"], s["spec"], s["verif"]), _streams(bits.view(-1, HD), s["g"])):
        if x is not None and x.numel():
            to[page, kv, head, row] = x.view(*bits.shape[:3], -1)
    return [s["spec"], s["verif"]] + [q] * (s["n_q"] > 0)


def _run_window(s):
    """The pages that a sequence sees side by side, the shorter lists filled up; what a column does not see is masked."""
    S, C, G, H, N = s["seqs"], s["cols"], s["grp"], s["n_kv"], s["new"]
    kv = _decode(s["spec"].flatten(0, 2), s["verif"].flatten(0, 2), s["g"], s["full"]).view(s["pages"], 2, H, 64, HD)
    most = max(len(p) for p in s["seen"])
    pg = torch.tensor([p + [-1] * (most - len(p)) for p in s["seen"]], device="cuda")
    lens = torch.tensor(s["lens"], device="cuda")[:, None]
    at = s["table"].long().gather(1, pg.clamp(min=0))
    k, v = (kv[:, i][at].permute(0, 2, 1, 3, 4).reshape(S, H, -1, HD) for i in (0, 1))
    place = (pg[:, :, None] * 64 + torch.arange(64, device="cuda")).view(S, -1)
    there = (place >= 0) & (place < lens)
    place = torch.cat([place, lens + torch.arange(N, device="cuda")], 1)
    there = torch.cat([there, torch.ones(S, N, dtype=torch.bool, device="cuda")], 1)
    k, v = (torch.cat([x, y.float().transpose(1, 2)], 2) for x, y in ((k, s["kn"]), (v, s["vn"])))
    own_place = (lens + N - C + torch.arange(C, device="cuda"))[:, :, None]
    place = place[:, None, :]
    seen = there[:, None, :] & (place <= own_place) & ((place < s["first"]) | (place > own_place - s["window"]))
    q = s["q"].float().view(S, C, H, G, HD).permute(0, 2, 1, 3, 4).reshape(S, H, C * G, HD)
    p = q @ k.transpose(2, 3).contiguous() / math.sqrt(HD)
    p = p.masked_fill(~seen.repeat_interleave(G, 1)[:, None], -math.inf)
    p = (p - p.amax(3, keepdim=True)).exp()
    p = p / p.sum(3, keepdim=True)
    return (p @ v).view(S, H, C, G, HD).permute(0, 2, 1, 3, 4).reshape(S, C, H * G, HD).bfloat16()


def _probabilities(z, t):
    """[rows, vocab] in 64 bits at temperatures t [rows, 1]; at 0 all of it on the first of the largest."""
    z = z.double()
    w = torch.exp((z - z.amax(1, keepdim=True)) / torch.where(t > 0, t, 1.0))
    one = torch.zeros_like(w).scatter_(1, z.argmax(1, keepdim=True), 1.0)
    return torch.where(t > 0, w / w.sum(1, keepdim=True), one)


def _run_accept(s):
    """Sums over the vocabulary in 64 bits: which token a number falls on is decided between neighbours of them."""
    drafts, S, most = s["drafts"], len(s["drafts"]), max(s["drafts"])
    n = sum(drafts)
    ks = torch.tensor(drafts, device="cuda")
    temp = s["temp"].double()[:, None]
    p = _probabilities(s["target"], temp.repeat_interleave(ks + 1, 0))
    row0 = torch.cumsum(ks + 1, 0) - ks - 1  # a sequence's first row of the target
    out = torch.full((S, most + 1), -1, dtype=torch.int64, device="cuda")
    kept = torch.zeros(S, dtype=torch.int64, device="cuda")
    px = qx = torch.empty(0, device="cuda")
    q = None
    if n:
        seq = torch.repeat_interleave(torch.arange(S, device="cuda"), ks)
        i = torch.arange(n, device="cuda") - (row0 - torch.arange(S, device="cuda"))[seq]  # which of its sequence's drafts
        token = s["tokens"].long()
        pd = p[row0[seq] + i, token]
        if s["known"]:
            q = _probabilities(s["near"], temp.repeat_interleave(ks, 0))
            qd = q.gather(1, token[:, None])[:, 0]
        else:
            qd = torch.ones_like(pd)
        good = (pd > 0) & (s["r"][row0[seq] + i] <= pd / qd)
        all_good = torch.zeros(S, most, dtype=torch.int64, device="cuda")
        all_good[seq, i] = good.long()
        kept = torch.cumprod(all_good, 1).sum(1)
        drafted = torch.full((S, most + 1), -1, dtype=torch.int64, device="cuda")
        drafted[seq, i] = token
        px, qx = pd.float(), qd.float()
    w = p[row0 + kept]
    if n:  # behind the first draft that is not kept: what the target has beyond the draft
        cut = (kept < ks)[:, None]
        at = (row0 - torch.arange(S, device="cuda") + kept).clamp(max=n - 1)
        less = q[at] if q is not None else torch.zeros_like(w).scatter_(1, token[at][:, None], 1.0)
        rest = torch.where(cut, (w - less).clamp(min=0.0), w)
        w = torch.where(rest.sum(1, keepdim=True) > 0, rest, w)
    c = torch.cumsum(w, 1)
    over = (c > (s["r"][row0 + ks] * c[:, -1])[:, None]) & (w > 0)
    last = s["vocab"] - 1 - (w > 0).flip(1).to(torch.uint8).argmax(1)
    after = torch.where(over.any(1), over.to(torch.uint8).argmax(1), last)
    place = torch.arange(most + 1, device="cuda")
    if n:
        out = torch.where(place < kept[:, None], drafted, out)
    out = torch.where(place == kept[:, None], after[:, None], out)
    return [kept.to(torch.int32), out.to(torch.int32), px, qx]


# ---- the framework's calls --------------------------------------------------------------------
def _handles(s):
    """The context and the cache object that a program keeps, made on the first pass."""
    from paper_2605_26558_amd import binding as B
    if "ctx" not in s:
        size = 0
        if s["kind"] != "accept":
            s["ctx"] = B.Context()
            s["kv"] = B.KVCache(s["ctx"], 1, s["n_kv"], s["pages"], *s["table"].shape, keep_permille=s["keep"], trunc_bits=s["trunc"],
                                page_table=s["table"], exp_mode=B.CAS_EXP_SHARED if s["g"]["mx"] else B.CAS_EXP_RAW,
                                spec_pool=s["flat"][0], verif_pool=s["flat"][1])
            for i, n in enumerate(s["lens"]):
                B.cas_kv_set_len(s["kv"], i, n)
        if s["kind"] == "window":
            S = s["seqs"]
            size = B.cas_attention_window_bytes(s["kv"], range(S), s["first"], s["window"], [s["cols"]] * S, s["n_kv"] * s["grp"], [s["new"]] * S)
        if s["kind"] == "accept":
            size = B.cas_accept_tokens_bytes(s["drafts"], s["vocab"])
        s["ctx"] = B.Context(workspace=torch.empty(max(size, 256), dtype=torch.uint8, device="cuda"))
    return B, s["ctx"], s.get("kv")


def _own_append(s):
    B, ctx, kv = _handles(s)
    q, k, v = _heads(s)
    out = B.cas_kv_append_rope(ctx, kv, 0, range(len(s["tokens"])), s["tokens"], s["angles"], k, v, q=q if s["n_q"] else None, pos=s["pos"],
                               layout=(B.CAS_ROPE_HALF, B.CAS_ROPE_INTERLEAVED)[s["layout"]])
    return [s["spec"], s["verif"]] + ([out.view(torch.bfloat16)] if s["n_q"] else [])


def _own_window(s):
    B, ctx, kv = _handles(s)
    o = torch.empty_like(s["q"])
    B.cas_attention_window(ctx, kv, 0, range(s["seqs"]), s["first"], s["window"], s["full"], s["q"].unbind(0), s["kn"].unbind(0), s["vn"].unbind(0),
                           outs=o.unbind(0))
    return o


def _own_accept(s):
    B, ctx, _ = _handles(s)
    n, out, p, q = B.cas_accept_tokens(ctx, s["target"], s["near"], s["tokens"], s["drafts"], s["r"], temperature=s["temp"], probs=True)
    return [n, out, p, q]


def run(state):
    kind = state["kind"]
    if own:
        return {"append": _own_append, "window": _own_window, "accept": _own_accept}[kind](state)
    return {"append": _run_append, "window": _run_window, "accept": _run_accept}[kind](state)


def work(case):
    c, kind = _numbers(case), case["kind"]
    if kind == "accept":
        n, S = sum(c["drafts"]), len(c["drafts"])
        rows = n * (2 if c["known"] else 1) + S
        return {"bytes": 4 * rows * c["vocab"] + 12 * (n + S) + 12 * n + 8 * S, "flops": 4 * rows * c["vocab"]}
    g = _geometry(c)
    vector = 4 * (g["off"] // 64 + g["sw"] + g["lw"] + g["pw"])
    if kind == "append":
        n, size = sum(c["tokens"]), 4 if c["fp32"] else 2
        return {"bytes": n * ((c["n_q"] + 2 * c["n_kv"]) * HD * size + c["n_q"] * HD * 2 + 2 * c["n_kv"] * vector + 4 * c["rot"] + 4),
                "flops": n * (c["n_q"] + c["n_kv"]) * c["rot"] * 3}
    if not c["full"]:
        vector = 4 * (g["off"] // 64 + g["sw"])
    cells, places = 0, 0  # (column, position) pairs; committed positions that some column sees
    for n in _lens(c):
        total = n + c["new"]
        lowest = max(0, total - c["cols"] - c["window"] + 1)
        places += max(0, n - lowest) + min(c["first"], lowest, n)
        for col in range(c["cols"]):
            at = total - c["cols"] + col
            low = max(0, at - c["window"] + 1)
            cells += at - low + 1 + min(c["first"], low)
    heads, rows = c["n_kv"], c["cols"] * c["grp"] * c["n_kv"]
    return {"bytes": 2 * heads * (places * vector + c["seqs"] * c["new"] * 256) + c["seqs"] * rows * 512, "flops": cells * c["grp"] * heads * 4 * HD}


# ---- the operators' definitions in 64 bits ----------------------------------------------------
def _exact_append(case, seed):
    """The turned queries; the rest are bit fields."""
    if case["n_q"] == 0:
        return None
    s = prepare(case, seed)
    r = s["rot"]
    f = 500000.0 ** (-2.0 * torch.arange(r // 2, dtype=torch.float64, device="cuda") / r)
    z = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), s["pos"].double()[:, None] * f)[:, None]  # turns as complex numbers
    x = _heads(s)[0].bfloat16().double()
    a = x[..., :r].unflatten(-1, (2, r // 2) if s["layout"] == HALF else (r // 2, 2))
    pair = -2 if s["layout"] == HALF else -1
    w = torch.complex(*a.unbind(pair)) * z
    return [None, None, torch.cat([torch.stack([w.real, w.imag], pair).flatten(-2), x[..., r:]], -1)]


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


def _exact_window(case, seed):
    """Sequence by sequence, head by head and column by column over the positions that the column sees."""
    c = case
    lay = _layout(c, seed)
    dense = _dense(lay["bits"], c)
    G, N, C = c["grp"], c["new"], c["cols"]
    out = torch.empty(c["seqs"], C, c["n_kv"] * G, HD, dtype=torch.float64, device="cuda")
    for s, n in enumerate(lay["lens"]):
        pages = lay["table"][s].long()
        for col in range(C):
            me = n + N - C + col
            low = max(0, me - c["window"] + 1)
            at = torch.tensor([*range(min(c["first"], low)), *range(low, me + 1)], device="cuda")
            old, new = at[at < n], at[at >= n] - n
            for h in range(c["n_kv"]):
                k, v = (torch.cat([dense[pages[old // 64], i, h, old % 64], lay[x][s, new, h].double()]) for i, x in ((0, "kn"), (1, "vn")))
                q = lay["q"][s, col, h * G:(h + 1) * G].double()
                out[s, col, h * G:(h + 1) * G] = torch.softmax(q @ k.T / HD ** 0.5, 1) @ v
    return out


def _exact_accept(case, seed):
    """Draft by draft on the host, logarithms of the probabilities by log-sum-exp."""
    s = prepare(case, seed)
    tokens, r, temp = s["tokens"].tolist(), s["r"].cpu().numpy(), s["temp"].double().cpu().numpy()
    target, near = s["target"].cpu().numpy(), None if s["near"] is None else s["near"].cpu().numpy()

    def prob(z, t):
        z = z.astype(np.float64)
        if t == 0.0:
            return (np.arange(len(z)) == int(np.argmax(z))).astype(np.float64)
        z = z / t
        return np.exp(z - (z.max() + np.log(np.exp(z - z.max()).sum())))

    counts, outs, px, qx, d, row = [], [], [], [], 0, 0
    for i, k in enumerate(s["drafts"]):
        w, n = None, 0
        for j in range(k):
            p, x = prob(target[row + j], temp[i]), tokens[d + j]
            q = prob(near[d + j], temp[i]) if near is not None else (np.arange(s["vocab"]) == x).astype(np.float64)
            px.append(p[x])
            qx.append(q[x])
            if w is None:
                if p[x] > 0.0 and r[row + j] <= p[x] / q[x]:
                    n += 1
                else:
                    w = np.maximum(0.0, p - q)
                    w = w if w.sum() > 0.0 else p
        if w is None:
            w = prob(target[row + k], temp[i])
        c = np.cumsum(w)
        at = int(np.searchsorted(c, r[row + k] * c[-1], side="right"))
        after = at if at < len(w) else int(np.flatnonzero(w)[-1])
        counts.append(n)
        outs.append([*tokens[d:d + n], after] + [-1] * (max(s["drafts"]) - n))
        d, row = d + k, row + k + 1
    return [torch.tensor(counts, dtype=torch.int32), torch.tensor(outs, dtype=torch.int32), torch.tensor(px, dtype=torch.float64),
            torch.tensor(qx, dtype=torch.float64)]


def exact(case, seed):
    return {"append": _exact_append, "window": _exact_window, "accept": _exact_accept}[case["kind"]](case, seed)
