"""cas_attention_shared and cas_attention_weights against attention in 64 bits on the vectors that cas_kv_read gives
(checked bit for bit elsewhere): formats, group sizes, lengths from nothing to long, prefixes that end inside pages,
masks, infinities in places that a column does not see, bad page tables, streams, captured calls, refusals."""
import math

import numpy as np
import pytest

import synth

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2605_26558_amd import binding as B
    return torch, B, B.Context(workspace=torch.empty(256 << 20, dtype=torch.uint8, device="cuda"))


def _bits(torch, a):
    return torch.from_numpy(np.ascontiguousarray(a).view(np.int16)).cuda()


def _cache(torch, B, ctx, n_kv, prefix, tails, keep=600, t=4, mode=0, layers=1, layer=0, new=64):
    """A cache whose sequences hold the same `prefix` positions, then `tails` of their own; pages of the prefix shared."""
    common = prefix // 64
    most = max((prefix + n + new + 63) // 64 for n in tails)
    mine, S = most - common, len(tails)
    rng = np.random.Generator(np.random.Philox(7))
    place = rng.permutation(common + S * mine).astype(np.int32)
    table = np.concatenate([np.broadcast_to(place[:common], (S, common)), place[common:].reshape(S, mine)], 1)
    kv = B.KVCache(ctx, layers, n_kv, len(place), S, most, keep_permille=keep, trunc_bits=t, exp_mode=mode,
                   page_table=torch.from_numpy(np.ascontiguousarray(table)))
    K = synth.kv_tensor(max(prefix, 1), n_kv, 128, seed=3)[:prefix]
    V = synth.kv_tensor(max(prefix, 1), n_kv, 128, seed=4, outlier_channels=0)[:prefix]
    for s, n in enumerate(tails):
        k = np.concatenate([K, synth.kv_tensor(max(n, 1), n_kv, 128, seed=20 + s)[:n]])
        v = np.concatenate([V, synth.kv_tensor(max(n, 1), n_kv, 128, seed=60 + s, outlier_channels=0)[:n]])
        if len(k):
            B.cas_kv_append(ctx, kv, layer, s, _bits(torch, k), _bits(torch, v))
        B.cas_kv_set_len(kv, s, prefix + n)
    return kv


def _inputs(torch, S, cols, news, nq, n_kv, seed=5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda n, h, s: (torch.randn(n, h, 128, device="cuda", generator=g) * s).bfloat16()  # noqa: E731
    return ([r(c, nq, 0.5) for c in cols], [r(n, n_kv, 1.0) for n in news], [r(n, n_kv, 1.0) for n in news])


def _reference(torch, B, ctx, kv, layer, s, full, q, kn, vn):
    """(output, its tolerance, weights per kv head and position, their tolerance) in 64 bits."""
    n, (C, nq), N, H = B.cas_kv_len(kv, s), q.shape[:2], kn.shape[0], kn.shape[1]
    G = nq // H
    k, v = kn.double(), vn.double()
    if n:
        kc, vc = B.cas_kv_read(ctx, kv, layer, s, 0, n, full)
        k, v = (torch.cat([a.view(torch.bfloat16).double(), b]) for a, b in ((kc, k), (vc, v)))
    qh = q.double().view(C, H, G, 128)
    k, v = k.transpose(0, 1), v.transpose(0, 1)                                    # [H, n + N, 128]
    sc = torch.matmul(qh.permute(1, 0, 2, 3).reshape(H, C * G, 128), k.transpose(1, 2).contiguous()) / math.sqrt(128.0)
    big = torch.matmul(qh.permute(1, 0, 2, 3).reshape(H, C * G, 128).abs(), k.abs().transpose(1, 2).contiguous()) / math.sqrt(128.0)
    seen = torch.arange(n + N, device="cuda") <= (torch.arange(C, device="cuda") + n + N - C).repeat_interleave(G)[:, None]
    sc = sc.masked_fill(~seen, -math.inf)
    p = torch.softmax(sc, 2)
    o, mean = torch.empty_like(p[..., :1]).expand(-1, -1, 128).clone(), torch.empty_like(p[..., :1]).expand(-1, -1, 128).clone()
    for i in range(C * G):  # row by row, so that what a row does not see is no factor of it
        row = torch.where(seen[i][:, None], v, 0.0)
        o[:, i] = (p[:, i, :, None] * row).sum(1)
        mean[:, i] = (p[:, i, :, None] * row.abs()).sum(1)
    # a weight's relative error: its score as 128 fp32 additions of exact products and a scaling, in the exponent, and the
    # rounding of the exponential (2^-23 each of these); the same once more through the sum it is divided by
    rel = 2.0 ** -23 * (70 * big.masked_fill(~seen, 0.0) + 8)
    rel = rel + (p * rel).sum(2, keepdim=True) + 2.0 ** -24 * (64 + (n + N) / 16)
    w, wt = p.sum(1), (p * rel).sum(1) + 2.0 ** -23 * p.sum(1) * C * G
    # an output: weights as a bf16 head and the bf16 rounding of the rest (2^-7 cut off, 2^-8 of that), its own rounding (2^-8),
    # fp32 additions
    tol = 2.0 ** -8 * o.abs() + (2.0 ** -15 + 2.0 ** -24 * (64 + (n + N) / 4) + rel.amax(2, keepdim=True)) * mean
    shape = lambda x: x.view(H, C, G, 128).transpose(0, 1).reshape(C, nq, 128)  # noqa: E731
    return shape(o), shape(tol), w, wt


def _check(torch, out, ref, tol, what):
    got = out.view(torch.bfloat16).double()
    finite = torch.isfinite(ref)
    assert torch.equal(torch.isnan(got), torch.isnan(ref)), what
    assert torch.equal(got[~finite & ~torch.isnan(ref)], ref[~finite & ~torch.isnan(ref)]), what
    err, tol = (got - ref).abs()[finite], tol[finite]
    assert bool((err <= tol).all()), (what, float((err / tol).max()))


SHARED = [  # n_kv, group, prefix, tails, columns, in flight, full, keep, t, mode
    (2, 2, 0, [0], [1], [1], False, 600, 4, 0),
    (2, 2, 0, [0, 1], [1, 2], [3, 2], True, 600, 4, 0),
    (1, 1, 64, [0, 63, 64], [1, 1, 1], [1, 1, 2], False, 600, 4, 0),
    (2, 4, 130, [5, 0], [1, 1], [2, 1], False, 600, 4, 0),
    (2, 4, 63, [1, 0], [5, 3], [5, 4], True, 600, 4, 0),
    (3, 5, 700, [70, 1, 0, 200], [3, 1, 2, 16], [3, 64, 2, 16], True, 600, 4, 0),
    (8, 4, 1029, [300, 12, 77], [1, 1, 1], [4, 1, 2], False, 600, 4, 2),
    (2, 8, 512, [9] * 9, [2] * 9, [2] * 9, True, 600, 4, 2),
    (1, 48, 200, [3, 100], [16, 1], [16, 1], True, 700, 3, 0),
    (4, 2, 256, [1] * 32, [1] * 32, [1] * 32, False, 250, 0, 0),
    (1, 7, 4100, [64, 0], [4, 4], [9, 4], False, 500, 7, 0),
    (2, 1, 128, [10, 20], [1, 7], [1, 7], True, 1000, 5, 0),
    (2, 4, 128, [10, 20], [1, 7], [1, 7], True, 0, 4, 0),
    (2, 4, 192, [40, 2], [2, 2], [2, 2], False, 1000, 1, 2),
    (2, 3, 320, [129, 2, 3], [6, 5, 4], [6, 5, 4], True, 333, 2, 0),
    (8, 8, 640, [50, 20, 0, 64], [5, 5, 5, 5], [5, 5, 5, 5], True, 600, 6, 0),
    (2, 8, 704, [9] * 9, [2] * 9, [2] * 9, False, 600, 4, 0),
    # runs of several pages: of three, of five with a page left over, and of ten for the sixteen waves of many rows
    (8, 4, 14117, [70, 3], [1, 1], [1, 2], False, 600, 4, 0),
    (8, 2, 19205, [1], [7], [7], True, 400, 2, 2),
    (8, 8, 19205, [70, 3, 130], [3, 2, 1], [3, 2, 4], True, 600, 4, 0),
    (8, 8, 12900, [5, 3, 0, 1], [5, 5, 5, 5], [5, 5, 5, 5], True, 600, 4, 2),
    (4, 8, 20000, [0, 100, 7], [6, 6, 6], [6, 6, 6], False, 500, 1, 0),
    (8, 4, 0, [9000, 100], [5, 1], [5, 1], True, 600, 4, 0),
    # behind the prefix: runs of two steps, of sixteen waves and of eight; more than 64 steps
    (8, 4, 100, [130, 300, 5] + [70] * 13, [5] * 16, [5] * 16, True, 600, 4, 0),
    (8, 2, 70, [500, 300, 5, 129] + [70] * 28, [1] * 32, [1] * 32, False, 600, 4, 0),
    (1, 2, 64, [8300, 10], [1, 2], [1, 2], False, 600, 4, 0),
    # 4096 query rows of a kv head; shared exponents at the other truncations
    (2, 8, 130, [1] * 31 + [40], [16] * 32, [16] * 32, False, 600, 4, 0),
    (2, 4, 128, [30, 7], [2, 3], [2, 3], True, 600, 0, 2), (2, 4, 128, [30, 7], [2, 3], [2, 3], False, 600, 3, 2),
    (2, 4, 128, [30, 7], [2, 3], [2, 3], True, 700, 6, 2), (2, 4, 128, [30, 7], [2, 3], [2, 3], True, 500, 7, 2),
]


@pytest.mark.parametrize("n_kv,grp,prefix,tails,cols,news,full,keep,t,mode", SHARED)
def test_shared_matches_64_bits(env, n_kv, grp, prefix, tails, cols, news, full, keep, t, mode):
    torch, B, ctx = env
    print(f"case {n_kv=} {grp=} {prefix=} {tails=} {cols=} {news=} {full=} {keep=} {t=} {mode=}", flush=True)
    kv = _cache(torch, B, ctx, n_kv, prefix, tails, keep, t, mode, layers=2, layer=1)
    Q, Kn, Vn = _inputs(torch, len(tails), cols, news, n_kv * grp, n_kv)
    seqs = list(range(len(tails)))
    outs = B.cas_attention_shared(ctx, kv, 1, seqs, prefix, full, Q, Kn, Vn)
    torch.cuda.synchronize()
    for s in seqs:
        ref, tol, _, _ = _reference(torch, B, ctx, kv, 1, s, full, Q[s], Kn[s], Vn[s])
        _check(torch, outs[s], ref, tol, s)
    # the same once more: no order of arrival in the results; and the other way round
    again = B.cas_attention_shared(ctx, kv, 1, seqs, prefix, full, Q, Kn, Vn)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, again))


def test_a_sequence_does_not_see_the_others(env):
    """Values (infinities among them) and lengths of the other sequences leave a sequence's bits alone."""
    torch, B, ctx = env
    tails, cols = [100, 30, 0], [2, 2, 2]
    kv = _cache(torch, B, ctx, 2, 400, tails)
    Q, Kn, Vn = _inputs(torch, 3, cols, cols, 8, 2)
    a = B.cas_attention_shared(ctx, kv, 0, [0, 1, 2], 400, True, Q, Kn, Vn)
    Q2, Kn2, Vn2 = ([x[0], y, z] for x, y, z in ((Q, Q[1] * math.inf, Q[2] * 0), (Kn, Kn[1] * math.nan, Kn[2]), (Vn, Vn[1] * math.inf, Vn[2])))
    B.cas_kv_set_len(kv, 2, 400)
    B.cas_kv_set_len(kv, 1, 410)
    b = B.cas_attention_shared(ctx, kv, 0, [0, 1, 2], 400, True, Q2, Kn2, Vn2)
    torch.cuda.synchronize()
    assert torch.equal(a[0], b[0])
    assert torch.isnan(b[1].float()).any()


def test_infinities_a_column_does_not_see(env):
    """In-flight vectors with infinities and NaN: the columns before them are as without, those that see them as in 64 bits."""
    torch, B, ctx = env
    kv = _cache(torch, B, ctx, 2, 64, [61, 5])
    cols = [4, 4]
    Q, Kn, Vn = _inputs(torch, 2, cols, [5, 4], 8, 2)
    clean = B.cas_attention_shared(ctx, kv, 0, [0, 1], 64, True, Q, Kn, Vn)
    Vn[0][3, 0, 17], Vn[0][4, 1, 100], Kn[0][4, 0, 3] = math.inf, math.nan, math.nan
    Vn[1][2, 1, 64], Vn[1][3, 1, 64] = -math.inf, math.inf
    outs = B.cas_attention_shared(ctx, kv, 0, [0, 1], 64, True, Q, Kn, Vn)
    torch.cuda.synchronize()
    for s in (0, 1):
        ref, tol, _, _ = _reference(torch, B, ctx, kv, 0, s, True, Q[s], Kn[s], Vn[s])
        _check(torch, outs[s], ref, tol, s)
    assert torch.equal(outs[0][:2], clean[0][:2]) and torch.equal(outs[1][:2], clean[1][:2])


def test_infinities_of_keys(env):
    """In-flight keys with infinities: NaN for the rows that see them (or weight 0), the other columns as without."""
    torch, B, ctx = env
    kv = _cache(torch, B, ctx, 2, 64, [61, 5])
    Q, Kn, Vn = _inputs(torch, 2, [4, 4], [5, 4], 8, 2)
    Q[0], Q[1] = Q[0].abs(), Q[1].abs()
    clean = B.cas_attention_shared(ctx, kv, 0, [0, 1], 64, True, Q, Kn, Vn)
    Kn[0][3, 0, 17], Kn[1][2, 1, 64] = math.inf, -math.inf      # scores of +inf and of -inf
    outs = B.cas_attention_shared(ctx, kv, 0, [0, 1], 64, True, Q, Kn, Vn)
    torch.cuda.synchronize()
    for s in (0, 1):
        ref, tol, _, _ = _reference(torch, B, ctx, kv, 0, s, True, Q[s], Kn[s], Vn[s])
        _check(torch, outs[s], ref, torch.where(torch.isfinite(tol), tol, 2.0 ** -6 * ref.abs() + 1e-2), s)
        assert torch.equal(outs[s][:2], clean[s][:2])
    assert bool(torch.isnan(outs[0][2:, :4].float()).all()) and bool(torch.isfinite(outs[1].float()).all())


def test_order_of_sequences_and_copies_of_the_prefix(env):
    """The prefix is read through the first sequence's pages: the others may have copies of it, or pages of nothing."""
    torch, B, ctx = env
    n_kv, P, tails = 2, 200, [40, 3, 100]
    kv = B.KVCache(ctx, 1, n_kv, 24, 3, 8, page_table=torch.randperm(24, dtype=torch.int32).view(3, 8))
    K, V = synth.kv_tensor(P, n_kv, 128, seed=1), synth.kv_tensor(P, n_kv, 128, seed=2, outlier_channels=0)
    for s, n in enumerate(tails):
        k = np.concatenate([K, synth.kv_tensor(n, n_kv, 128, seed=20 + s)])
        v = np.concatenate([V, synth.kv_tensor(n, n_kv, 128, seed=60 + s, outlier_channels=0)])
        B.cas_kv_append(ctx, kv, 0, s, _bits(torch, k), _bits(torch, v))
        B.cas_kv_set_len(kv, s, P + n)
    Q, Kn, Vn = _inputs(torch, 3, [2, 1, 3], [2, 1, 4], 8, n_kv)
    for order in ([0, 1, 2], [2, 0, 1], [1, 2], [2]):
        outs = B.cas_attention_shared(ctx, kv, 0, order, P, True, [Q[s] for s in order], [Kn[s] for s in order], [Vn[s] for s in order])
        torch.cuda.synchronize()
        for s, o in zip(order, outs):
            ref, tol, _, _ = _reference(torch, B, ctx, kv, 0, s, True, Q[s], Kn[s], Vn[s])
            _check(torch, o, ref, tol, (order, s))


def test_a_cache_beyond_32_bits(env):
    """Pools of more than 2^32 words: shared attention, weights and an eviction in the last layer, on the last pages."""
    torch, B, ctx = env
    layers, n_kv, pages = 190, 8, 1100
    kv = B.KVCache(ctx, layers, n_kv, pages, 3, 4, keep_permille=600, trunc_bits=4,
                   page_table=torch.tensor([[1099, 1090, 1098, 1], [1099, 1090, 1097, 2], [1095, 1094, 0, 3]], dtype=torch.int32))
    assert min(kv.desc.spec_pool_bytes, kv.desc.verif_pool_bytes) > 4 << 32
    layer, P, tails = layers - 1, 128, [30, 9]
    K, V = synth.kv_tensor(P, n_kv, 128, seed=1), synth.kv_tensor(P, n_kv, 128, seed=2, outlier_channels=0)
    for s, n in enumerate(tails):
        k = np.concatenate([K, synth.kv_tensor(n, n_kv, 128, seed=20 + s)])
        v = np.concatenate([V, synth.kv_tensor(n, n_kv, 128, seed=60 + s, outlier_channels=0)])
        B.cas_kv_append(ctx, kv, layer, s, _bits(torch, k), _bits(torch, v))
        B.cas_kv_set_len(kv, s, P + n)
    Q, Kn, Vn = _inputs(torch, 2, [2, 1], [2, 1], 16, n_kv)
    outs = B.cas_attention_shared(ctx, kv, layer, [0, 1], P, True, Q, Kn, Vn)
    o, w = B.cas_attention_weights(ctx, kv, layer, 0, False, Q[0], Kn[0], Vn[0])
    torch.cuda.synchronize()
    for s in (0, 1):
        ref, tol, _, _ = _reference(torch, B, ctx, kv, layer, s, True, Q[s], Kn[s], Vn[s])
        _check(torch, outs[s], ref, tol, s)
    ref, tol, want, wt = _reference(torch, B, ctx, kv, layer, 0, False, Q[0], Kn[0], Vn[0])
    _check(torch, o, ref, tol, "weights")
    assert bool(((w.double() - want).abs() <= wt).all())
    index = B.cas_kv_select(ctx, w, P + 30, 70, 4, 10).view(1, n_kv, 70)
    B.cas_kv_evict(ctx, kv, layer, 1, 0, 2, index)
    B.cas_kv_set_len(kv, 2, 70)
    a, b = B.cas_kv_read(ctx, kv, layer, 0, 0, P + 30, True), B.cas_kv_read(ctx, kv, layer, 2, 0, 70, True)
    torch.cuda.synchronize()
    for x, y in zip(a, b):
        for h in range(n_kv):
            assert torch.equal(y[:, h], x[index[0, h].long(), h])
    del kv
    torch.cuda.empty_cache()


def test_shared_agrees_with_attention_per_sequence(env):
    torch, B, ctx = env
    tails, cols = [200, 3], [5, 5]
    kv = _cache(torch, B, ctx, 4, 900, tails)
    Q, Kn, Vn = _inputs(torch, 2, cols, cols, 16, 4)
    outs = B.cas_attention_shared(ctx, kv, 0, [0, 1], 900, True, Q, Kn, Vn)
    for s in (0, 1):
        one = B.cas_attention(ctx, kv, 0, s, True, Q[s], Kn[s], Vn[s])
        torch.cuda.synchronize()
        _, tol, _, _ = _reference(torch, B, ctx, kv, 0, s, True, Q[s], Kn[s], Vn[s])
        assert bool(((one.double() - outs[s].double()).abs() <= 2 * tol).all())


WEIGHTS = [  # n_kv, group, len, columns, in flight, full, keep, t, mode
    (2, 2, 0, 1, 1, False, 600, 4, 0), (2, 2, 0, 3, 5, True, 600, 4, 0), (1, 1, 1, 1, 1, True, 600, 4, 0),
    (2, 4, 63, 1, 1, False, 600, 4, 0), (2, 4, 64, 5, 5, True, 600, 4, 0), (8, 4, 1000, 1, 3, False, 600, 4, 2),
    (4, 8, 2049, 7, 7, True, 600, 4, 0), (1, 48, 130, 16, 20, True, 500, 3, 0), (2, 5, 4000, 3, 3, False, 250, 0, 0),
    (8, 1, 515, 2, 64, True, 700, 5, 2), (2, 16, 300, 1, 1, False, 1000, 7, 0), (8, 4, 17001, 3, 3, True, 600, 4, 0),
    (8, 8, 12300, 5, 6, False, 600, 4, 2), (1, 4, 9000, 1, 2, True, 600, 4, 0), (2, 9, 600, 16, 16, True, 600, 4, 0),
]


@pytest.mark.parametrize("n_kv,grp,n,cols,new,full,keep,t,mode", WEIGHTS)
def test_weights_match_64_bits(env, n_kv, grp, n, cols, new, full, keep, t, mode):
    torch, B, ctx = env
    print(f"case {n_kv=} {grp=} {n=} {cols=} {new=} {full=} {keep=} {t=} {mode=}", flush=True)
    kv = _cache(torch, B, ctx, n_kv, 0, [3, n], keep, t, mode)
    (q,), (kn,), (vn,) = _inputs(torch, 1, [cols], [new], n_kv * grp, n_kv)
    total, ld = n + new, n + new + 5
    before = torch.rand(n_kv, ld, device="cuda")
    before[:, n:] = math.nan                                  # behind the committed length: not read
    after = torch.full((n_kv, ld), 9.0, device="cuda")
    o, _ = B.cas_attention_weights(ctx, kv, 0, 1, full, q, kn, vn, before, score_out=after)
    o2, fresh = B.cas_attention_weights(ctx, kv, 0, 1, full, q, kn, vn)
    same = before.clone()
    o3, _ = B.cas_attention_weights(ctx, kv, 0, 1, full, q, kn, vn, same, score_out=same)
    torch.cuda.synchronize()
    ref, tol, w, wt = _reference(torch, B, ctx, kv, 0, 1, full, q, kn, vn)
    for x in (o, o2, o3):
        _check(torch, x, ref, tol, "output")
    assert fresh.shape == (n_kv, total)
    err = (fresh.double() - w).abs()
    assert bool((err <= wt).all()), float((err / wt).max())
    want = w.clone()
    want[:, :n] += before[:, :n].double()
    err = (after[:, :total].double() - want).abs()
    assert bool((err <= wt + 2.0 ** -24 * want).all()), float((err / (wt + 2.0 ** -24 * want)).max())
    assert bool((after[:, total:] == 9.0).all())
    assert torch.equal(same[:, :total], after[:, :total]) and bool(torch.isnan(same[:, total:]).all())
    # every row's weights add up to one
    sums = fresh.double().sum(1)
    assert bool(((sums - cols * grp).abs() <= wt.sum(1)).all())


def test_a_bad_page_table_stays_in_the_pool(env):
    """Entries outside the pool are clamped into it: wrong values, no access outside (a page nothing needs is not looked at)."""
    torch, B, ctx = env
    kv = _cache(torch, B, ctx, 2, 128, [70, 1])
    Q, Kn, Vn = _inputs(torch, 2, [1, 1], [1, 1], 4, 2)
    clean = B.cas_attention_shared(ctx, kv, 0, [0, 1], 128, True, Q, Kn, Vn)
    torch.cuda.synchronize()
    table = kv.page_table
    table[0, 4:], table[1, 3:] = 2**31 - 1, -5                 # pages behind all positions
    again = B.cas_attention_shared(ctx, kv, 0, [0, 1], 128, True, Q, Kn, Vn)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(clean, again))
    table[1, :2] = 10**9                                       # the prefix is read through the first sequence's row
    again = B.cas_attention_shared(ctx, kv, 0, [0, 1], 128, True, Q, Kn, Vn)
    table[0, 0], table[1, 2] = -7, 10**9
    B.cas_attention_shared(ctx, kv, 0, [0, 1], 128, True, Q, Kn, Vn)
    B.cas_attention_weights(ctx, kv, 0, 0, False, Q[0], Kn[0], Vn[0])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(clean, again))


def test_captured_and_on_another_stream(env):
    torch, B, _ = env
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        ctx = B.Context(workspace=torch.empty(32 << 20, dtype=torch.uint8, device="cuda"))
        kv = _cache(torch, B, ctx, 2, 300, [100, 7])
        Q, Kn, Vn = _inputs(torch, 2, [2, 2], [2, 2], 8, 2)
        outs = B.cas_attention_shared(ctx, kv, 0, [0, 1], 300, True, Q, Kn, Vn)
        score = torch.zeros(2, 512, device="cuda")
        o, _ = B.cas_attention_weights(ctx, kv, 0, 0, True, Q[0], Kn[0], Vn[0], score, score_out=score)
        want = [x.clone() for x in (*outs, o, score)]
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        B.cas_attention_shared(ctx, kv, 0, [0, 1], 300, True, Q, Kn, Vn, outs=outs)
        B.cas_attention_weights(ctx, kv, 0, 0, True, Q[0], Kn[0], Vn[0], None, score_out=score, out=o)
    for i in range(3):
        for x in (*outs, o, score):
            x.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip((*outs, o, score), want):
            assert torch.equal(x, y), i
        with torch.cuda.stream(s):   # eager work on the same context between replays
            B.cas_attention(ctx, kv, 0, 1, True, Q[1], Kn[1], Vn[1])
        s.synchronize()


def test_two_streams_at_once(env):
    """Two contexts with workspaces of their own, on streams of their own, over the same cache."""
    torch, B, ctx = env
    kv = _cache(torch, B, ctx, 4, 2000, [100, 7])
    Q, Kn, Vn = _inputs(torch, 2, [3, 1], [3, 1], 16, 4)
    want = B.cas_attention_shared(ctx, kv, 0, [0, 1], 2000, True, Q, Kn, Vn)
    want_w = B.cas_attention_weights(ctx, kv, 0, 0, True, Q[0], Kn[0], Vn[0])
    torch.cuda.synchronize()
    streams, runs = [torch.cuda.Stream() for _ in range(2)], []
    for s in streams:
        with torch.cuda.stream(s):
            runs.append((B.Context(workspace=torch.empty(32 << 20, dtype=torch.uint8, device="cuda")), [], []))
    for _ in range(10):
        for s, (c, outs, ws) in zip(streams, runs):
            with torch.cuda.stream(s):
                outs.append(B.cas_attention_shared(c, kv, 0, [0, 1], 2000, True, Q, Kn, Vn))
                ws.append(B.cas_attention_weights(c, kv, 0, 0, True, Q[0], Kn[0], Vn[0]))
    torch.cuda.synchronize()
    for _, outs, ws in runs:
        for o, w in zip(outs, ws):
            assert all(torch.equal(x, y) for x, y in zip(o, want)) and all(torch.equal(x, y) for x, y in zip(w, want_w))


def test_refusals(env):
    torch, B, ctx = env
    kv = _cache(torch, B, ctx, 2, 100, [10, 20], new=8)
    Q, Kn, Vn = _inputs(torch, 2, [1, 1], [1, 1], 4, 2)

    def code(*a, **k):
        with pytest.raises(B.CasError) as e:
            B.cas_attention_shared(*a, **k)
        return e.value.code

    assert code(ctx, kv, 1, [0, 1], 100, True, Q, Kn, Vn) == B.CAS_EINVAL          # layer
    assert code(ctx, kv, 0, [0, 0], 100, True, Q, Kn, Vn) == B.CAS_EINVAL          # a sequence twice
    assert code(ctx, kv, 0, [0, 2], 100, True, Q, Kn, Vn) == B.CAS_EINVAL
    assert code(ctx, kv, 0, [0, 1], 111, True, Q, Kn, Vn) == B.CAS_EINVAL          # longer than a sequence
    assert code(ctx, kv, 0, [0, 1], -1, True, Q, Kn, Vn) == B.CAS_EINVAL
    assert code(B.Context(), kv, 0, [0, 1], 100, True, Q, Kn, Vn) == B.CAS_ENOMEM  # no workspace
    need = B.cas_attention_shared_bytes(kv, [0, 1], 100, [1, 1], 4, [1, 1])
    small = B.Context(workspace=torch.empty(need - 1, dtype=torch.uint8, device="cuda"))
    assert code(small, kv, 0, [0, 1], 100, True, Q, Kn, Vn) == B.CAS_ENOMEM
    exact = B.Context(workspace=torch.empty(need, dtype=torch.uint8, device="cuda"))
    B.cas_attention_shared(exact, kv, 0, [0, 1], 100, True, Q, Kn, Vn)
    many = torch.zeros(17, 4, 128, dtype=torch.bfloat16, device="cuda")
    new = torch.zeros(17, 2, 128, dtype=torch.bfloat16, device="cuda")
    assert code(ctx, kv, 0, [0], 100, True, [many], [new], [new]) == B.CAS_EINVAL  # columns
    assert code(ctx, kv, 0, [0], 100, True, [many[:2]], [new[:1]], [new[:1]]) == B.CAS_EINVAL
    assert code(ctx, kv, 0, [0], 100, True, [many[:1, :3].contiguous()], [new[:1]], [new[:1]]) == B.CAS_EINVAL
    big = torch.zeros(64, 2, 128, dtype=torch.bfloat16, device="cuda")
    B.cas_kv_set_len(kv, 0, 128)
    assert code(ctx, kv, 0, [0], 100, True, [many[:1]], [big], [big]) == B.CAS_ENOMEM   # no page for what is in flight
    B.cas_kv_set_len(kv, 0, 110)
    odd = torch.zeros(1 + 512, dtype=torch.bfloat16, device="cuda")[1:].view(1, 4, 128)
    assert code(ctx, kv, 0, [0], 100, True, [odd], [new[:1]], [new[:1]]) == B.CAS_EINVAL   # alignment
    score = torch.zeros(2, 200, device="cuda")
    lib, p = B._lib(), lambda t: t.data_ptr()  # noqa: E731

    def weights(layer=0, seq=0, cols=1, nq=4, n=1, o=p(Q[0]), out=p(score), ld=200, c=ctx):
        return lib.cas_attention_weights(c.h, kv.h, layer, seq, 1, p(many), cols, nq, p(new), p(new), n, o, None, out, ld)

    for bad in (dict(layer=-1), dict(seq=5), dict(cols=0), dict(cols=17, n=17), dict(nq=3), dict(nq=98), dict(n=0), dict(n=65), dict(o=None),
                dict(out=None), dict(ld=110), dict(o=p(Q[0]) + 16)):
        assert weights(**bad) == B.CAS_EINVAL, bad
    assert weights(c=B.Context()) == B.CAS_ENOMEM
    assert weights(ld=111, o=p(torch.empty_like(many))) == B.CAS_OK
    torch.cuda.synchronize()


@pytest.mark.parametrize("prefix,own,other", [(0, 790, (790, 3000, 200)), (703, 90, (90, 4000)), (130, 500, (64, 5000))])
def test_lengths_of_the_others_leave_the_bits(env, prefix, own, other):
    """The same call with another sequence that is short, or so long that a row of it has more partial results than the one looked at."""
    torch, B, ctx = env
    cols = [16, 1]
    kv = _cache(torch, B, ctx, 8, prefix, [own, max(other)])
    for seed in range(4):   # a sum in another order shows in some 6 of 100000 values, of which a call has 131072
        Q, Kn, Vn = _inputs(torch, 2, cols, cols, 64, 8, seed=seed)
        outs = []
        for n in other:
            B.cas_kv_set_len(kv, 1, prefix + n)
            outs.append(B.cas_attention_shared(ctx, kv, 0, [0, 1], prefix, True, Q, Kn, Vn)[0])
        torch.cuda.synchronize()
        for n, o in zip(other, outs):
            assert torch.equal(o, outs[0]), (seed, n, int((o != outs[0]).sum()))


def test_scores_of_one_kv_head_in_other_tensors(env):
    """Sums of a single kv head read from and written to rows of tensors of different widths."""
    torch, B, ctx = env
    kv = _cache(torch, B, ctx, 1, 0, [300])
    (q,), (kn,), (vn,) = _inputs(torch, 1, [2], [3], 4, 1)
    before, after = torch.rand(5, 320, device="cuda"), torch.full((3, 400), 9.0, device="cuda")
    _, want = B.cas_attention_weights(ctx, kv, 0, 0, True, q, kn, vn, before[2:3, :303].contiguous())
    _, got = B.cas_attention_weights(ctx, kv, 0, 0, True, q, kn, vn, before[2:3, :303], score_out=after[1:2, 7:310])
    _, third = B.cas_attention_weights(ctx, kv, 0, 0, True, q, kn, vn, before[2].expand(1, 320))
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(third[:, :303], want)
    after[1, 7:310] = 9.0
    assert bool((after == 9.0).all())
