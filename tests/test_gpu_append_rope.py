"""cas_kv_append_rope against cas_rope followed by cas_kv_append, word by word of both pools, and against the rotation in 64 bits
of what the cache then holds: single tokens and prompts, ragged batches, partial heads, both layouts, types, strides, padding,
places that cross pages, bad page tables, pools beyond 32 bits, streams, captured calls, refusals."""
import ctypes as C

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2605_26558_amd import binding as B
    return torch, B, B.Context()


def _table(torch, n_pos, rot, seed=None):
    f = 10000.0 ** (-2.0 * torch.arange(rot // 2, dtype=torch.float64, device="cuda") / rot)
    a = torch.arange(n_pos, dtype=torch.float64, device="cuda")[:, None] * f
    return torch.stack([a.cos(), a.sin()], 2).float().contiguous()


def _caches(torch, B, ctx, n, n_kv, lens, toks, keep, t, mode, layers=2):
    """n caches alike, filled with the same random words."""
    most = max((a + b + 63) // 64 for a, b in zip(lens, toks)) + 1
    rng = np.random.Generator(np.random.Philox(3))
    place = rng.permutation(len(lens) * most + 3)[:len(lens) * most].astype(np.int32).reshape(len(lens), most)
    out = []
    for i in range(n):
        kv = B.KVCache(ctx, layers, n_kv, len(lens) * most + 3, len(lens), most, keep_permille=keep, trunc_bits=t, exp_mode=mode,
                       page_table=torch.from_numpy(place))
        g = torch.Generator(device="cuda").manual_seed(1)
        for pool in (kv.spec_pool, kv.verif_pool):
            pool.copy_(torch.randint(0, 256, pool.shape, generator=g, device="cuda", dtype=torch.uint8))
        for s, a in enumerate(lens):
            B.cas_kv_set_len(kv, s, a)
        out.append(kv)
    return out


def _heads(torch, n_tok, n_q, n_kv, fp32, seed, pad=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(n_tok, (n_q + 2 * n_kv) * 128 + pad, generator=g, device="cuda")
    x = x if fp32 else x.bfloat16()
    cut = lambda a, h: x[:, pad + a * 128:pad + (a + h) * 128].unflatten(1, (h, 128))  # noqa: E731
    return cut(0, n_q), cut(n_q, n_kv), cut(n_q + n_kv, n_kv)


def _apart(torch, B, ctx, kv, layer, toks, table, q, k, v, pos, layout, turn):
    """The two calls that the one stands for, sequence by sequence; padded tokens are left out one by one."""
    n_pos = table.shape[0]
    lens = [B.cas_kv_len(kv, s) for s in range(len(toks))]
    places = [a + i for a, n in zip(lens, toks) for i in range(n)]
    at = list(places) if pos is None else pos.tolist()
    p = torch.tensor(at, dtype=torch.int32, device="cuda")
    outs = [torch.full(x.shape, 9, dtype=torch.int16, device="cuda") for x in (q, k, v)]
    n_pos and B.cas_rope(ctx, table, [q, k, v], pos=p, layout=layout, turn=turn, outs=outs)
    i = 0
    for s, (a, n) in enumerate(zip(lens, toks)):
        j = 0
        while j < n:  # runs of tokens that are not padding
            e = j
            while e < n and 0 <= at[i + e] < n_pos:
                e += 1
            if e > j:
                B.cas_kv_set_len(kv, s, a + j)
                B.cas_kv_append(ctx, kv, layer, s, outs[1][i + j:i + e].contiguous(), outs[2][i + j:i + e].contiguous())
            j = e + 1
        B.cas_kv_set_len(kv, s, a)
        i += n
    return outs


CASES = [  # kv heads, query heads, lengths, tokens, keep, t, mode, channels that turn, layout, fp32
    (1, 1, [0], [1], 600, 4, 0, 128, 0, True),
    (8, 32, [8190], [3], 600, 4, 0, 128, 0, True),
    (2, 0, [63, 64, 0], [1, 1, 2], 600, 4, 2, 128, 1, False),
    (2, 6, [5, 0, 127, 9], [0, 70, 1, 0], 700, 3, 0, 64, 0, False),
    (3, 3, [31] * 32, [1 + i % 6 for i in range(32)], 500, 1, 2, 2, 1, True),
    (8, 8, [100], [300], 600, 4, 0, 128, 0, True),
    (8, 24, [1021], [1000], 600, 4, 0, 128, 0, True),
    (8, 3, [13, 0, 64, 200], [100, 1, 0, 150], 600, 4, 2, 96, 0, False),
    (8, 17, [13, 0, 64, 201], [130, 3, 64, 77], 400, 0, 0, 128, 1, True),
    (4, 4, [7, 1], [401, 3], 1000, 7, 0, 62, 0, True),           # halves that are no whole eights
    (4, 5, [7, 1], [401, 3], 0, 5, 0, 126, 1, False),
    (8, 0, [3] * 20, [17] * 20, 333, 2, 2, 32, 0, True),
    (16, 16, [250], [515], 600, 6, 0, 16, 0, False),
    (4, 70, [0], [900], 600, 4, 0, 6, 0, True),
    # sixteen vectors to a wave, from 24 for each CU (32 over shared exponents) on: every t, both forms, all kinds of partners
    (8, 3, [13, 0, 64, 200], [260, 1, 0, 259], 600, 4, 2, 96, 0, False),
    (8, 17, [13, 0, 64, 201], [330, 3, 64, 177], 400, 0, 0, 128, 1, True),
    (8, 17, [15, 0, 64, 201], [331, 3, 65, 176], 400, 0, 2, 128, 1, True),
    (8, 4, [7, 1], [601, 3], 1000, 7, 0, 62, 0, True),
    (8, 4, [7, 1], [601, 3], 1000, 7, 2, 126, 0, False),
    (8, 5, [7, 1], [601, 3], 0, 5, 0, 126, 1, False),
    (8, 5, [7, 1], [601, 3], 0, 5, 2, 128, 0, True),
    (8, 0, [3] * 20, [33] * 20, 333, 2, 2, 32, 0, True),
    (8, 1, [i for i in range(32)], [17 + i % 7 for i in range(32)], 333, 2, 0, 128, 0, False),
    (16, 2, [47], [400], 500, 1, 0, 2, 0, True),
    (16, 2, [47], [400], 8, 1, 2, 2, 1, True),
    (16, 0, [48], [400], 992, 3, 0, 64, 0, False),
    (16, 0, [48], [400], 700, 3, 2, 6, 1, False),
    (8, 8, [63], [641], 600, 5, 2, 64, 1, True),
    (8, 8, [63], [641], 600, 6, 2, 16, 0, True),
    (48, 8, [1], [130], 600, 2, 0, 30, 0, True),
]


@pytest.mark.parametrize("n_kv,n_q,lens,toks,keep,t,mode,rot,layout,fp32", CASES)
def test_words_are_those_of_the_two_calls(env, n_kv, n_q, lens, toks, keep, t, mode, rot, layout, fp32):
    torch, B, ctx = env
    print("case", n_kv, n_q, lens, toks, keep, t, mode, rot, layout, fp32, flush=True)
    n = sum(toks)
    table = _table(torch, max(a + b for a, b in zip(lens, toks)) + 50, rot)
    q, k, v = _heads(torch, n, n_q, n_kv, fp32, 5)
    rng = np.random.Generator(np.random.Philox(9))
    spread = rng.integers(0, table.shape[0], n).astype(np.int32)
    holes = spread.copy()
    holes[rng.random(n) < 0.3] = -1
    holes[rng.random(n) < 0.1] = table.shape[0]
    for what, pos in (("places", None), ("given", spread), ("padded", holes)):
        pos = None if pos is None else torch.from_numpy(pos).cuda()
        one, two = _caches(torch, B, ctx, 2, n_kv, lens, toks, keep, t, mode)
        outs = [torch.full(x.shape, 9, dtype=torch.int16, device="cuda") for x in (q, k, v)]
        given = B.cas_kv_append_rope(ctx, one, 1, range(len(lens)), toks, table, k, v, q=q if n_q else None, pos=pos, layout=layout, q_out=outs[0] if n_q else None,
                                     k_out=outs[1], v_out=outs[2])
        assert given is (outs[0] if n_q else None)
        want = _apart(torch, B, ctx, two, 1, toks, table, q, k, v, pos, layout, (True, True, False))
        for a, b, x in zip(outs, want, "qkv"):
            assert torch.equal(a, b), (what, x)
        assert torch.equal(one.spec_pool, two.spec_pool) and torch.equal(one.verif_pool, two.verif_pool), what
        assert [B.cas_kv_len(one, s) for s in range(len(lens))] == lens
        # no dense vectors wanted, queries through an output of the call's own: the same words
        three = _caches(torch, B, ctx, 1, n_kv, lens, toks, keep, t, mode)[0]
        alone = B.cas_kv_append_rope(ctx, three, 1, range(len(lens)), toks, table, k, v, q=q if n_q else None, pos=pos, layout=layout)
        if n_q and what != "padded":
            assert torch.equal(alone.view(torch.int16), want[0])
        assert torch.equal(three.spec_pool, two.spec_pool) and torch.equal(three.verif_pool, two.verif_pool), what


@pytest.mark.parametrize("n_kv,n_q,lens,toks,keep,t,mode,rot,layout,fp32", [  # few tokens each of many sequences, many heads: either side of the limit
    (64, 4, [7 * i for i in range(32)], [2] * 32, 600, 4, 0, 128, 0, True), (64, 4, [7 * i for i in range(32)], [7] * 32, 600, 4, 0, 128, 0, True),
    (32, 32, [5 * i for i in range(32)], [4] * 32, 600, 3, 2, 128, 1, False), (32, 32, [5 * i for i in range(32)], [11] * 32, 600, 3, 2, 128, 1, False),
    (16, 16, [16 * i for i in range(32)], [6] * 32, 500, 2, 0, 96, 0, False), (16, 16, [16 * i + 9 for i in range(32)], [15, 0] * 16, 500, 2, 2, 62, 0, True)])
def test_words_of_batches_with_many_heads(env, n_kv, n_q, lens, toks, keep, t, mode, rot, layout, fp32):
    test_words_are_those_of_the_two_calls(env, n_kv, n_q, lens, toks, keep, t, mode, rot, layout, fp32)


@pytest.mark.parametrize("mode", [0, 2])
@pytest.mark.parametrize("fp32", [False, True])
@pytest.mark.parametrize("rot,layout", [(128, 0), (128, 1), (96, 0), (96, 1), (62, 0), (16, 0), (2, 0)])
def test_special_values_turn_alike_whatever_the_call_holds(env, rot, layout, fp32, mode):
    """Infinities, NaN of both signs, zeros, subnormal and largest numbers as partners of each other, at angles among which sin or
    cos is 0: one call with few tokens, one with many, and the two calls they stand for.  Of two products that are both NaN
    either may come out, and infinity times 0 is one: a NaN has finite partners here."""
    torch, B, ctx = env
    n_kv, n_q, n_tok = 8, 8, 480   # 18 vectors a token: from 342 (over shared exponents 456) on sixteen to a wave
    special = [0x0000, 0x8000, 0x3F80, 0xBFC0, 0x7F80, 0xFF80, 0x7FC0, 0xFFC5, 0x7F81, 0xFFA3, 0x7F7F, 0xFF7F, 0x0001, 0x8003, 0x0080, 0x7F00]
    nan, large = (lambda w: w & 0x7FFF > 0x7F80), (lambda w: w & 0x7FFF >= 0x7F80)
    pairs = torch.tensor([(a, b) for a in special for b in special if not (nan(a) and large(b) or large(a) and nan(b))], dtype=torch.int32)
    g = torch.Generator().manual_seed(rot + layout)
    half = rot // 2
    x = torch.randint(0, 65536, (n_tok, n_q + 2 * n_kv, 128), generator=g, dtype=torch.int32)   # channels behind rot: anything
    a = torch.arange(half)
    ia, ib = (a, a + half) if layout == 0 else (2 * a, 2 * a + 1)
    p = pairs[torch.randint(0, len(pairs), (n_tok, n_q + 2 * n_kv, half), generator=g)]
    x[..., ia], x[..., ib] = p[..., 0], p[..., 1]
    x = x.to(torch.int16).cuda()
    if fp32:  # with bits below bf16: numbers that round up to infinity among them, and NaN that have nothing above
        low = torch.randint(0, 65536, x.shape, generator=g, dtype=torch.int32).cuda()
        x = ((x.int() << 16) | low).view(torch.float32)
        x = torch.where(torch.rand(x.shape, generator=g).cuda() < 0.5, x, (x.view(torch.int32) & -65536).view(torch.float32))
        # an infinity with bits below is a NaN, and the largest bf16 number with enough of them rounds to infinity
        rounded = x.bfloat16()
        one, other = rounded[..., ia.cuda()], rounded[..., ib.cuda()]
        both = torch.isnan(one) & ~torch.isfinite(other) | torch.isnan(other) & ~torch.isfinite(one)
        x[..., ia.cuda()] = torch.where(both, 1.0, x[..., ia.cuda()])
    q, k, v = x[:, :n_q], x[:, n_q:n_q + n_kv], x[:, n_q + n_kv:]
    table = torch.rand(40, half, 2, generator=g).cuda() * 2 - 1
    for i, cs in enumerate(((1.0, 0.0), (0.0, 1.0), (-1.0, -0.0), (-0.0, -1.0), (1.0, 1.0))):
        table[i] = torch.tensor(cs)
    pos = (torch.arange(n_tok, dtype=torch.int32) % 40).cuda()
    turn = (rot != 16, True, rot != 62)
    few, many, alone, two = _caches(torch, B, ctx, 4, n_kv, [7], [n_tok], 600, 4, mode)
    outs = [[torch.full(y.shape, 9, dtype=torch.int16, device="cuda") for y in (q, k, v)] for _ in range(2)]
    call = lambda kv, n, i, o: B.cas_kv_append_rope(ctx, kv, 1, [0], [n], table, k[i:i + n], v[i:i + n], q=q[i:i + n], pos=pos[i:i + n].contiguous(),  # noqa: E731
                                                    layout=layout, turn=turn, q_out=o[0][i:i + n], k_out=o[1][i:i + n], v_out=o[2][i:i + n])
    call(many, n_tok, 0, outs[0])
    for i in range(0, n_tok, 48):
        B.cas_kv_set_len(few, 0, 7 + i)
        call(few, 48, i, outs[1])
    want = _apart(torch, B, ctx, two, 1, [n_tok], table, q, k, v, pos, layout, turn)
    assert bool(((want[0] & 0x7FFF) > 0x7F80).any()) and bool(((want[0] & 0x7FFF) == 0x7F80).any())
    for kv, o, what in ((many, outs[0], "many"), (few, outs[1], "few")):
        for y, ref, part in zip(o, want, "qkv"):
            assert torch.equal(y, ref), (what, part)
        assert torch.equal(kv.spec_pool, two.spec_pool) and torch.equal(kv.verif_pool, two.verif_pool), what
    B.cas_kv_append_rope(ctx, alone, 1, [0], [n_tok], table, k, v, q=q, pos=pos, layout=layout, turn=turn)   # no dense keys and values
    assert torch.equal(alone.spec_pool, two.spec_pool) and torch.equal(alone.verif_pool, two.verif_pool)


@pytest.mark.parametrize("n_tok", [5, 700])
@pytest.mark.parametrize("layout", [0, 1])
def test_what_the_cache_holds_against_the_rotation_in_64_bits(env, n_tok, layout):
    torch, B, ctx = env
    n_kv, n_q, rot, start = 4, 8, 96, 30
    q, k, v = _heads(torch, n_tok, n_q, n_kv, True, 6)
    kv = _caches(torch, B, ctx, 1, n_kv, [start], [n_tok], 600, 4, 0)[0]
    pos = torch.randperm(5000, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))[:n_tok].int()
    out = B.cas_kv_append_rope(ctx, kv, 0, [0], [n_tok], _table(torch, 5000, rot), k, v, q=q, pos=pos, layout=layout)
    K, V = B.cas_kv_read(ctx, kv, 0, 0, start, n_tok, True)
    assert torch.equal(V.view(torch.bfloat16), v.bfloat16())
    f = 10000.0 ** (-2.0 * torch.arange(rot // 2, dtype=torch.float64, device="cuda") / rot)
    z = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), pos.double()[:, None] * f)[:, None]
    for got, x in ((out, q), (K, k)):
        x = x.bfloat16().double()
        a = x[..., :rot].unflatten(-1, (2, rot // 2) if layout == 0 else (rot // 2, 2))
        pair = -2 if layout == 0 else -1
        w = torch.complex(*a.unbind(pair)) * z
        ref = torch.cat([torch.stack([w.real, w.imag], pair).flatten(-2), x[..., rot:]], -1)
        # its rounding to bf16, and of what is added: two products, the sum, and the table's entries, 2^-24 each
        sums = torch.cat([torch.stack([w.abs(), w.abs()], pair).flatten(-2), x[..., rot:].abs()], -1)
        err = (got.view(torch.bfloat16).double() - ref).abs()
        assert bool((err <= 2.0 ** -8 * ref.abs() + 8 * 2.0 ** -24 * sums * 1.5).all()), float(err.max())


@pytest.mark.parametrize("n_tok", [3, 500])
def test_strides_types_and_places_in_memory(env, n_tok):
    """Rows any distance apart, from any element on, outputs in place: the words do not change."""
    torch, B, ctx = env
    n_kv, n_q = 8, 9
    table = _table(torch, 4000, 128)
    pos = torch.arange(n_tok, dtype=torch.int32, device="cuda") * 3
    for fp32 in (False, True):
        q, k, v = _heads(torch, n_tok, n_q, n_kv, fp32, 7)
        call = lambda kv, q, k, v, **how: B.cas_kv_append_rope(ctx, kv, 0, [0], [n_tok], table, k, v, q=q, pos=pos, **how)  # noqa: E731
        ref = _caches(torch, B, ctx, 1, n_kv, [70], [n_tok], 600, 4, 0)[0]
        want = call(ref, q, k, v).view(torch.int16)
        for pad in (1, 2, 3, 5, 8):
            moved = []
            for x in (q, k, v):
                wide = torch.zeros(n_tok, x.shape[1] * 128 + 11 * pad, dtype=x.dtype, device="cuda")
                part = wide[:, pad:pad + x.shape[1] * 128].unflatten(1, (x.shape[1], 128))
                part.copy_(x)
                moved.append(part)
            kv = _caches(torch, B, ctx, 1, n_kv, [70], [n_tok], 600, 4, 0)[0]
            out = torch.zeros(n_tok, n_q * 128 + 7 * pad, dtype=torch.int16, device="cuda")[:, pad:pad + n_q * 128].unflatten(1, (n_q, 128))
            assert torch.equal(call(kv, *moved, q_out=out), want)
            assert torch.equal(kv.spec_pool, ref.spec_pool) and torch.equal(kv.verif_pool, ref.verif_pool), pad
        if not fp32:  # in place
            kv = _caches(torch, B, ctx, 1, n_kv, [70], [n_tok], 600, 4, 0)[0]
            dense = B.cas_rope(ctx, table, [k], pos=pos)[0]
            assert torch.equal(call(kv, q, k, v, q_out=q, k_out=k, v_out=v).view(torch.int16), want) and torch.equal(k, dense)
            assert torch.equal(kv.spec_pool, ref.spec_pool) and torch.equal(kv.verif_pool, ref.verif_pool)


@pytest.mark.parametrize("n_tok", [40, 500])
def test_pages_outside_the_pool_are_not_written(env, n_tok):
    torch, B, ctx = env
    table = _table(torch, 4000, 128)
    q, k, v = _heads(torch, n_tok, 4, 8, True, 8)
    good = _caches(torch, B, ctx, 1, 8, [50], [n_tok], 600, 4, 0)[0]
    bad = _caches(torch, B, ctx, 1, 8, [50], [n_tok], 600, 4, 0)[0]
    before = bad.spec_pool.clone(), bad.verif_pool.clone()
    page = int(good.page_table[0, 1])
    for entry in (-1, bad.desc.n_pages, 2 ** 31 - 1, -2 ** 31):
        bad.spec_pool.copy_(before[0])
        bad.verif_pool.copy_(before[1])
        bad.page_table[0, 1] = entry
        a = B.cas_kv_append_rope(ctx, good, 0, [0], [n_tok], table, k, v, q=q)
        assert torch.equal(B.cas_kv_append_rope(ctx, bad, 0, [0], [n_tok], table, k, v, q=q), a)
        d = good.desc
        for got, want, old, tile in ((bad.spec_pool, good.spec_pool, before[0], d.tile_spec_bytes), (bad.verif_pool, good.verif_pool, before[1], d.tile_verif_bytes)):
            want, lo = want.clone(), page * 2 * d.n_kv_heads * tile
            want[lo:lo + 2 * d.n_kv_heads * tile] = old[lo:lo + 2 * d.n_kv_heads * tile]
            assert torch.equal(got, want), entry


@pytest.mark.parametrize("n_tok", [2, 500])
def test_pools_beyond_32_bits(env, n_tok):
    """The last pages of the last layer, tens of gigabytes into the pools."""
    torch, B, ctx = env
    n_pages, layers, n_kv = 12000, 6, 8
    kv = B.KVCache(ctx, layers, n_kv, n_pages, 1, 8, page_table=torch.arange(n_pages - 8, n_pages, dtype=torch.int32).view(1, 8))
    assert kv.desc.spec_pool_bytes > 1 << 33 and kv.desc.verif_pool_bytes > 1 << 33
    q, k, v = _heads(torch, n_tok, 4, n_kv, True, 9)
    table = _table(torch, 600, 128)
    B.cas_kv_append_rope(ctx, kv, layers - 1, [0], [n_tok], table, k, v)
    kb, vb = B.cas_rope(ctx, table, [k, v], turn=(True, False))
    K, V = B.cas_kv_read(ctx, kv, layers - 1, 0, 0, n_tok, True)
    assert torch.equal(K, kb) and torch.equal(V, vb)


@pytest.mark.parametrize("n_tok", [4, 500])
def test_streams_and_captured_calls(env, n_tok):
    """A captured call replayed over new heads and positions, with eager calls and waits between."""
    torch, B, _ = env
    stream = torch.cuda.Stream()
    table = _table(torch, 3000, 128)
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        ctx = B.Context()
        held, eager = _caches(torch, B, ctx, 2, 8, [60], [n_tok], 600, 4, 0)
        q, k, v = (x.contiguous() for x in _heads(torch, n_tok, 8, 8, True, 1))
        pos = torch.arange(n_tok, dtype=torch.int32, device="cuda")
        out = torch.empty(q.shape, dtype=torch.int16, device="cuda")
        call = lambda kv, q, k, v, pos, out=None: B.cas_kv_append_rope(ctx, kv, 1, [0], [n_tok], table, k, v, q=q, pos=pos, q_out=out)  # noqa: E731
        call(held, q, k, v, pos, out)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            call(held, q, k, v, pos, out)
        for seed in (2, 3, 4):
            fresh = _heads(torch, n_tok, 8, 8, True, seed)
            p = (pos * 7 + seed) % 3000
            for h, f in zip((q, k, v), fresh):
                h.copy_(f)
            held_pos = pos.clone()
            pos.copy_(p)
            graph.replay()
            want = call(eager, *fresh, p)
            stream.synchronize()
            assert torch.equal(out, want), seed
            assert torch.equal(held.spec_pool, eager.spec_pool) and torch.equal(held.verif_pool, eager.verif_pool), seed
            pos.copy_(held_pos)


@pytest.mark.parametrize("mode", [0, 2])
@pytest.mark.parametrize("t,keep,start,n_tok", [(0, 600, 5, 1301), (1, 700, 0, 1300), (2, 1000, 63, 1298), (3, 8, 64, 1216), (4, 600, 1, 1215), (5, 0, 16, 1297), (6, 992, 17, 1300),
                                                (7, 400, 31, 1300)])
def test_long_appends_are_their_pieces(env, t, keep, start, n_tok, mode):
    """cas_kv_append of enough vectors for sixteen to a wave, against appends of a few tokens each; infinities, NaN, equal
    magnitudes and zeros among them."""
    torch, B, ctx = env
    g = torch.Generator(device="cuda").manual_seed(t)
    k, v = (torch.randn(n_tok, 8, 128, generator=g, device="cuda").bfloat16() for _ in range(2))
    k[3::7] = k[3::7].round()                       # many equal magnitudes
    v[5::11] = 0
    v[6::11, :, ::2] = -0.0
    k[8::13, :, 5] = float("inf")
    k[9::13, :, 100:] = float("nan")
    k[10::13] *= 2.0 ** 100                         # exponents far apart
    k[11::13, :, :64] *= 2.0 ** -126                # subnormal numbers
    one, two = _caches(torch, B, ctx, 2, 8, [start], [n_tok], keep, t, mode)
    k, v = k.view(torch.int16), v.view(torch.int16)
    B.cas_kv_append(ctx, one, 1, 0, k, v)
    i = 0
    while i < n_tok:
        n = min(3 + i % 14, n_tok - i)
        B.cas_kv_set_len(two, 0, start + i)
        B.cas_kv_append(ctx, two, 1, 0, k[i:i + n].contiguous(), v[i:i + n].contiguous())
        i += n
    assert torch.equal(one.spec_pool, two.spec_pool) and torch.equal(one.verif_pool, two.verif_pool)


def test_refusals(env):
    torch, B, ctx = env
    lib, i32 = B._lib(), B._i32
    table = _table(torch, 100, 128)
    q, k, v = (x.contiguous() for x in _heads(torch, 3, 4, 2, True, 1))
    kv = _caches(torch, B, ctx, 1, 2, [60, 0], [3, 0], 600, 4, 0)[0]
    out = torch.zeros(3, 4, 128, dtype=torch.int16, device="cuda")
    part = lambda x, y, heads, ldx=None, ldy=None, fp32=1: B.cas_rope_part(x, y, ldx or heads * 128, ldy or heads * 128, heads, fp32, 1, 0)  # noqa: E731
    pq, pk, pv = part(q.data_ptr(), out.data_ptr(), 4), part(k.data_ptr(), None, 2), part(v.data_ptr(), None, 2)
    good = dict(ctx=ctx.h, kv=kv.h, layer=0, n=2, seqs=i32([0, 1]), toks=i32([3, 0]), table=table.data_ptr(), n_pos=100, rot=128, layout=0, pos=None,
                q=C.byref(pq), k=C.byref(pk), v=C.byref(pv))
    call = lambda **bad: lib.cas_kv_append_rope(*{**good, **bad}.values())  # noqa: E731
    before = kv.spec_pool.clone()
    ref = lambda p: C.byref(p)  # noqa: E731
    for bad in (dict(ctx=None), dict(kv=None), dict(layer=2), dict(layer=-1), dict(n=-1), dict(n=33), dict(seqs=None), dict(toks=None), dict(seqs=i32([0, 0])),
                dict(seqs=i32([0, 2])), dict(toks=i32([3, -1])), dict(table=None), dict(table=table.data_ptr() + 8), dict(n_pos=-1), dict(rot=0),
                dict(rot=127), dict(rot=130), dict(layout=2), dict(k=None), dict(v=None), dict(k=ref(part(k.data_ptr(), None, 1))), dict(k=ref(part(None, None, 2))),
                dict(k=ref(part(k.data_ptr() + 2, None, 2))), dict(k=ref(part(k.data_ptr(), None, 2, ldx=255))), dict(q=ref(part(q.data_ptr(), None, 4))),
                dict(q=ref(part(q.data_ptr(), q.data_ptr(), 4))), dict(q=ref(part(q.data_ptr(), out.data_ptr() + 1, 4))),
                dict(q=ref(part(q.data_ptr(), out.data_ptr(), 4, ldy=511)))):
        assert call(**bad) == B.CAS_EINVAL, bad
    assert call(toks=i32([3 * 64, 0])) == B.CAS_ENOMEM
    assert call(toks=i32([3, 1 << 30])) == B.CAS_ENOMEM
    torch.cuda.synchronize()
    assert torch.equal(kv.spec_pool, before) and not bool(out.any())   # nothing was launched
    assert call(toks=i32([0, 0])) == B.CAS_OK and call(n=0, seqs=None, toks=None) == B.CAS_OK and call(n_pos=0) == B.CAS_OK
    torch.cuda.synchronize()
    assert torch.equal(kv.spec_pool, before) and not bool(out.any())
    assert call() == B.CAS_OK
    torch.cuda.synchronize()
    assert not torch.equal(kv.spec_pool, before) and bool(out.any())
