"""Eviction through the C ABI: the selection against a stable sort, the moved vectors bit for bit, in place and to other
pages, over formats and odd sizes; and the operators around the cache together: rotate, append, attend with sums, select, evict,
go on."""
import math

import numpy as np
import pytest

import synth

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2605_26558_amd import binding as B
    return torch, B, B.Context(workspace=torch.empty(64 << 20, dtype=torch.uint8, device="cuda"))


def _bits(torch, a):
    return torch.from_numpy(np.ascontiguousarray(a).view(np.int16)).cuda()


def _selected(row, n, keep, first, last):
    """Plain selection of one row: descending by (not NaN, value), ties to the lower position."""
    key = np.where(np.isnan(row[:n]), np.inf, row[:n].astype(np.float64))
    nan = np.isnan(row[:n])
    at = np.arange(first, n - last)
    order = at[np.lexsort((at, -key[at], ~nan[at]))]
    mid = order[:keep - first - last]
    return np.sort(np.concatenate([np.arange(first), mid, np.arange(n - last, n)])).astype(np.int32)


KINDS = {
    "spread": lambda r, s: r.exponential(1.0, s) ** 3,
    "ties": lambda r, s: r.integers(0, 4, s).astype(float),
    "equal": lambda r, s: np.full(s, 0.25),
    "signs": lambda r, s: np.where(r.random(s) < 0.3, np.where(r.random(s) < 0.5, 0.0, -0.0), r.standard_normal(s)),
    "special": lambda r, s: r.choice([math.nan, math.inf, -math.inf, -1e-45, 0.0, 3e38, -3e38, 1e-40, -math.nan], s),
    "close": lambda r, s: 1.0 + r.integers(0, 3, s) * 2.0 ** -23,
}


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("n,keep,first,last,rows", [
    (1, 1, 0, 0, 3), (1, 1, 1, 0, 1), (5, 2, 0, 0, 2), (64, 63, 4, 8, 5), (1000, 1000, 10, 10, 2), (1025, 512, 0, 512, 2), (2049, 100, 4, 95, 9),
    (8192, 2048, 4, 512, 3), (8193, 1, 0, 0, 2), (8193, 8192, 0, 0, 1), (32768, 5000, 1, 7, 2), (32769, 32000, 0, 0, 2), (70001, 777, 3, 0, 1),
    (300, 20, 20, 0, 2), (300, 20, 0, 20, 2), (300, 20, 13, 7, 2),
    (4096, 4000, 0, 3, 2), (20000, 300, 100, 200, 2), (65536, 40000, 3, 1000, 2), (65537, 9, 0, 0, 1), (50000, 17, 9, 8, 2), (70001, 70001, 0, 0, 1),
])
def test_selection_is_that_of_a_stable_sort(env, kind, n, keep, first, last, rows):
    torch, B, ctx = env
    print(f"case {kind=} {n=} {keep=} {first=} {last=} {rows=}", flush=True)
    r = np.random.Generator(np.random.Philox(n))
    score = KINDS[kind](r, (rows, n + 3)).astype(np.float32)
    dev = torch.from_numpy(score).cuda()
    kept = torch.full((rows, keep + 2), 5.0, device="cuda")
    index = B.cas_kv_select(ctx, dev, n, keep, first, last, kept=kept)
    own = dev.clone()
    again = B.cas_kv_select(ctx, own, n, keep, first, last, kept=own)
    torch.cuda.synchronize()
    want = np.stack([_selected(row, n, keep, first, last) for row in score])
    np.testing.assert_array_equal(index.cpu().numpy(), want)
    assert torch.equal(index, again)
    vals = np.take_along_axis(score, want.astype(np.int64), 1)
    np.testing.assert_array_equal(kept.cpu().numpy()[:, :keep].view(np.uint32), vals.view(np.uint32))
    assert bool((kept[:, keep:] == 5.0).all())
    np.testing.assert_array_equal(own.cpu().numpy()[:, :keep].view(np.uint32), vals.view(np.uint32))
    np.testing.assert_array_equal(own.cpu().numpy()[:, keep:].view(np.uint32), score[:, keep:].view(np.uint32))


def _filled(torch, B, ctx, layers, n_kv, lens, keep, t, mode, extra=0):
    pages = [(n + 63) // 64 + extra for n in lens]
    most = max(max(pages), 1)
    rng = np.random.Generator(np.random.Philox(9))
    table = rng.permutation(len(lens) * most).astype(np.int32).reshape(len(lens), most)
    kv = B.KVCache(ctx, layers, n_kv, len(lens) * most, len(lens), most, keep_permille=keep, trunc_bits=t, exp_mode=mode,
                   page_table=torch.from_numpy(table))
    kv.spec_pool.fill_(0xA5)
    kv.verif_pool.fill_(0x5A)
    for s, n in enumerate(lens):
        for l in range(layers):
            if n:
                B.cas_kv_append(ctx, kv, l, s, _bits(torch, synth.kv_tensor(n, n_kv, 128, seed=10 * s + l)),
                                _bits(torch, synth.kv_tensor(n, n_kv, 128, seed=100 + 10 * s + l, outlier_channels=0)))
        B.cas_kv_set_len(kv, s, n)
    return kv


def _streams(kv):
    """The four or five streams of a cache's pools as [tile][64 tokens][words], and the words of tiles behind them."""
    d = kv.desc
    sp, vf = (p.cpu().numpy()[:n].view("<u4") for p, n in ((kv.spec_pool, kv.desc.spec_pool_bytes - 256), (kv.verif_pool, kv.desc.verif_pool_bytes - 256)))
    sp = sp.reshape(-1, d.tile_spec_bytes // 4)
    vf = vf.reshape(len(sp), -1)                     # no words at all where everything is kept and nothing truncated
    out, at = [], 0
    for w in (4, 1 if d.fmt.exp_mode else 0, d.sw):
        out.append(sp[:, at:at + 64 * w].reshape(len(sp), 64, w))
        at += 64 * w
    rest = [sp[:, at:]]
    at = 0
    for w in (d.lw, d.pw):
        out.append(vf[:, at:at + 64 * w].reshape(len(sp), 64, w))
        at += 64 * w
    return out, rest + [vf[:, at:]]


def _moved(kv, before, layers, layer0, seq, dst, index):
    """What the streams have to be after an eviction, vector by vector from those before."""
    d, table = kv.desc, kv.page_table.cpu().numpy()
    after = [s.copy() for s in before]
    tile = lambda l, page, k, h: ((l * d.n_pages + page) * 2 + k) * d.n_kv_heads + h  # noqa: E731
    for l in range(layers):
        for h in range(d.n_kv_heads):
            p = index[l, h]
            i = np.arange(len(p))
            for k in (0, 1):
                src, to = tile(layer0 + l, table[seq][p // 64], k, h), tile(layer0 + l, table[dst][i // 64], k, h)
                for a, b in zip(after, before):
                    if b.shape[2]:
                        a[to, i % 64] = b[src, p % 64]
    return after


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("layers,layer0,n_layers,n_kv,n,n_keep,keep,t,mode", [
    (1, 0, 1, 1, 1, 1, 600, 4, 0), (1, 0, 1, 2, 64, 64, 600, 4, 0), (2, 1, 1, 2, 200, 63, 600, 4, 0), (3, 0, 3, 2, 1000, 511, 600, 4, 0),
    (1, 0, 1, 8, 1300, 65, 600, 4, 2), (2, 0, 2, 3, 321, 320, 250, 0, 0), (1, 0, 1, 1, 700, 300, 1000, 7, 0), (1, 0, 1, 2, 300, 129, 0, 4, 0),
    (2, 0, 1, 1, 130, 1, 333, 5, 2), (1, 0, 1, 2, 500, 400, 1000, 0, 0), (1, 0, 1, 2, 129, 128, 8, 1, 0), (1, 0, 1, 1, 260, 200, 992, 3, 2),
])
def test_vectors_move_bit_for_bit(env, in_place, layers, layer0, n_layers, n_kv, n, n_keep, keep, t, mode):
    torch, B, ctx = env
    print(f"case {in_place=} {layers=} {n_kv=} {n=} {n_keep=} {keep=} {t=} {mode=}", flush=True)
    kv = _filled(torch, B, ctx, layers, n_kv, [n, n_keep], keep, t, mode)
    rng = np.random.Generator(np.random.Philox(n_keep))
    index = np.stack([[np.sort(rng.permutation(n)[:n_keep]) for _ in range(n_kv)] for _ in range(n_layers)]).astype(np.int32)
    if not in_place:   # any order, and one more than once
        index[0, 0] = rng.permutation(index[0, 0])
        index[0, 0, -1] = index[0, 0, 0]
    dst = 0 if in_place else 1
    before, rest = _streams(kv)
    want = _moved(kv, before, n_layers, layer0, 0, dst, index)
    B.cas_kv_evict(ctx, kv, layer0, n_layers, 0, dst, torch.from_numpy(index).cuda())
    torch.cuda.synchronize()
    got, rest_after = _streams(kv)
    for a, b in zip(got, want):
        np.testing.assert_array_equal(a, b)
    for a, b in zip(rest_after, rest):
        np.testing.assert_array_equal(a, b)
    assert B.cas_kv_len(kv, 0) == n and B.cas_kv_len(kv, 1) == n_keep


def test_bad_pages_and_indices_stay_in_the_pool(env):
    torch, B, ctx = env
    kv = _filled(torch, B, ctx, 1, 2, [200, 130], 600, 4, 0)
    before, _ = _streams(kv)
    table = kv.page_table.clone()
    kv.page_table[1, 1] = 10**9                      # a destination outside the pool: nothing is written there
    index = torch.arange(130, dtype=torch.int32, device="cuda").expand(1, 2, 130).contiguous()
    B.cas_kv_evict(ctx, kv, 0, 1, 0, 1, index)
    torch.cuda.synchronize()
    after, _ = _streams(kv)
    t = table.cpu().numpy()
    for a, b in zip(after, before):
        for h in (0, 1):
            for k in (0, 1):
                tile = lambda s, i: (int(t[s, i]) * 2 + k) * 2 + h  # noqa: E731
                np.testing.assert_array_equal(a[tile(1, 0)], b[tile(0, 0)])
                np.testing.assert_array_equal(a[tile(1, 1)], b[tile(1, 1)])
                np.testing.assert_array_equal(a[tile(1, 2), :2], b[tile(0, 2), :2])
                np.testing.assert_array_equal(a[tile(1, 2), 2:], b[tile(1, 2), 2:])
    kv.page_table[:] = table
    kv.page_table[0, 1] = -3                         # a source outside: some page of the pool is read
    wild = torch.full((1, 2, 130), 2**31 - 1, dtype=torch.int32, device="cuda")
    wild[0, 1] = -2**31
    B.cas_kv_evict(ctx, kv, 0, 1, 0, 1, wild)        # clamped to the last and the first position
    torch.cuda.synchronize()
    kv.page_table[:] = table
    a, _ = B.cas_kv_read(ctx, kv, 0, 1, 0, 130, True)
    b, _ = B.cas_kv_read(ctx, kv, 0, 0, 0, 200, True)
    torch.cuda.synchronize()
    assert bool((a[:, 0] == b[199, 0]).all()) and bool((a[:, 1] == b[0, 1]).all())


def test_captured_eviction(env):
    torch, B, _ = env
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        ctx = B.Context()
        kv = _filled(torch, B, ctx, 2, 2, [300, 100], 600, 4, 0)
        score = torch.rand(4, 300, device="cuda")
        index = torch.zeros(4, 100, dtype=torch.int32, device="cuda")
        kept = torch.zeros(4, 100, device="cuda")
        B.cas_kv_select(ctx, score, 300, 100, 4, 30, kept=kept, index=index)
        B.cas_kv_evict(ctx, kv, 0, 2, 0, 1, index.view(2, 2, 100))
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        B.cas_kv_select(ctx, score, 300, 100, 4, 30, kept=kept, index=index)
        B.cas_kv_evict(ctx, kv, 0, 2, 0, 1, index.view(2, 2, 100))
    for i in range(3):
        score.copy_(torch.rand(4, 300, device="cuda"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = np.stack([_selected(r, 300, 100, 4, 30) for r in score.cpu().numpy()])
        np.testing.assert_array_equal(index.cpu().numpy(), want)
        for l in (0, 1):
            with torch.cuda.stream(s):
                a, b = B.cas_kv_read(ctx, kv, l, 1, 0, 100, True), B.cas_kv_read(ctx, kv, l, 0, 0, 300, True)
            s.synchronize()
            for x, y in zip(a, b):
                for h in (0, 1):
                    assert torch.equal(x[:, h], y[index[2 * l + h].long(), h]), (i, l, h)


def test_refusals(env):
    torch, B, ctx = env
    lib, score = B._lib(), torch.zeros(2, 100, device="cuda")
    index = torch.zeros(2, 100, dtype=torch.int32, device="cuda")

    def select(score_p=score.data_ptr(), ld=100, rows=2, n=100, keep=10, first=0, last=0, idx=index.data_ptr(), kept=None, ldk=0):
        return lib.cas_kv_select(ctx.h, score_p, ld, rows, n, keep, first, last, idx, kept, ldk)

    assert select() == B.CAS_OK
    for bad in (dict(score_p=None), dict(ld=99), dict(rows=-1), dict(n=-1), dict(keep=101), dict(keep=-1), dict(first=-1), dict(last=-1),
                dict(first=6, last=5), dict(idx=None), dict(kept=index.data_ptr(), ldk=9), dict(kept=score.data_ptr(), ldk=50),
                dict(first=2**31 - 1, last=2**31 - 1)):
        assert select(**bad) == B.CAS_EINVAL, bad
    assert select(n=(1 << 30) + 1, ld=1 << 40) == B.CAS_ENOTSUP
    assert select(rows=0, score_p=None, idx=None) == B.CAS_OK and select(keep=0, score_p=None, idx=None) == B.CAS_OK
    assert select(n=0, keep=0) == B.CAS_OK
    kv = _filled(torch, B, ctx, 2, 1, [100, 50], 600, 4, 0)

    def evict(layer0=0, layers=2, seq=0, dst=1, idx=index.data_ptr(), keep=50):
        return lib.cas_kv_evict(ctx.h, kv.h, layer0, layers, seq, dst, idx, keep)

    assert evict() == B.CAS_OK
    for bad in (dict(layer0=-1), dict(layers=3), dict(layer0=1), dict(layers=-1), dict(seq=2), dict(seq=-1), dict(dst=2), dict(dst=-1), dict(idx=None),
                dict(keep=101), dict(keep=-1), dict(seq=1, keep=51), dict(layer0=2**31 - 1, layers=2)):
        assert evict(**bad) == B.CAS_EINVAL, bad
    assert evict(layers=0, idx=None) == B.CAS_OK and evict(keep=0, idx=None) == B.CAS_OK
    torch.cuda.synchronize()


def test_operators_together(env):
    """Two conversations behind one prompt: positions turned one by one, appended, attended with a shared prefix; one of
    them decoded with sums, cut to its most looked-at positions, and decoded on at its true positions."""
    torch, B, ctx = env
    n_kv, grp, P, steps = 2, 4, 192, 6
    nq = n_kv * grp
    g = torch.Generator(device="cuda").manual_seed(11)
    table = B.cas_rope_table(ctx, B.cas_rope_cfg(128, B.CAS_ROPE_BANDS, 10000.0, 8.0, 512, 1.0, 32.0, 1.0), 0, 1024)
    pages = torch.tensor([[5, 1, 7, 2, 9], [5, 1, 7, 0, 4]], dtype=torch.int32)
    kv = B.KVCache(ctx, 1, n_kv, 10, 2, 5, page_table=pages)
    draw = lambda n: torch.randn(n, (nq + 2 * n_kv) * 128, device="cuda", generator=g)  # noqa: E731

    def split(y, pos):
        at = [y[:, a * 128:b * 128].unflatten(1, (b - a, 128)) for a, b in ((0, nq), (nq, nq + n_kv), (nq + n_kv, nq + 2 * n_kv))]
        return B.cas_rope(ctx, table, at, pos=torch.tensor(pos, dtype=torch.int32, device="cuda"), turn=(True, True, False))

    _, K, V = split(draw(P), list(range(P)))
    B.cas_kv_append(ctx, kv, 0, 0, K, V)                      # one copy, named by both page tables
    for s in (0, 1):
        B.cas_kv_set_len(kv, s, P)
    from tests.test_gpu_shared_attention import _check, _reference
    for step in range(steps):                                  # both go on, each with its own tokens
        qkv = [split(draw(1), [P + step]) for _ in (0, 1)]
        outs = B.cas_attention_shared(ctx, kv, 0, [0, 1], P, True, [x[0] for x in qkv], [x[1] for x in qkv], [x[2] for x in qkv])
        for s in (0, 1):
            q, k, v = (x.view(torch.bfloat16) for x in qkv[s])
            ref, tol, _, _ = _reference(torch, B, ctx, kv, 0, s, True, q, k, v)
            torch.cuda.synchronize()
            _check(torch, outs[s], ref, tol, (step, s))
            B.cas_kv_append(ctx, kv, 0, s, qkv[s][1], qkv[s][2])
            B.cas_kv_set_len(kv, s, P + step + 1)
    score = torch.zeros(n_kv, 5 * 64, device="cuda")
    want = torch.zeros(n_kv, 5 * 64, dtype=torch.float64, device="cuda")
    n, bound = P + steps, 0.0
    for step in range(4):
        q, k, v = (x.view(torch.bfloat16) for x in split(draw(1), [n]))
        B.cas_attention_weights(ctx, kv, 0, 1, True, q, k, v, score, score_out=score)
        _, _, w, wt = _reference(torch, B, ctx, kv, 0, 1, True, q, k, v)
        want[:, :n + 1] += w
        bound = bound + float(wt.max()) + 2.0 ** -22
        B.cas_kv_append(ctx, kv, 0, 1, k, v)
        n += 1
        B.cas_kv_set_len(kv, 1, n)
    torch.cuda.synchronize()
    assert float((score.double() - want).abs().max()) <= bound
    held = 100
    index = B.cas_kv_select(ctx, score, n, held, 4, 16, kept=score)
    a = [x.clone() for x in B.cas_kv_read(ctx, kv, 0, 1, 0, n, True)]
    other = [x.clone() for x in B.cas_kv_read(ctx, kv, 0, 0, P, steps, True)]
    # the prefix's pages belong to both conversations, so the first is over before the second is cut in place
    B.cas_kv_evict(ctx, kv, 0, 1, 1, 1, index.view(1, n_kv, held))
    B.cas_kv_set_len(kv, 1, held)
    b = B.cas_kv_read(ctx, kv, 0, 1, 0, held, True)
    after = B.cas_kv_read(ctx, kv, 0, 0, P, steps, True)
    torch.cuda.synchronize()
    for x, y in zip(a, b):
        for h in range(n_kv):
            assert torch.equal(y[:, h], x[index[h].long(), h])
    assert all(torch.equal(x, y) for x, y in zip(other, after))     # what only the first names is as it was
    q, k, v = (x.view(torch.bfloat16) for x in split(draw(2), [n, n + 1]))   # true positions, not the cache's length
    o, s2 = B.cas_attention_weights(ctx, kv, 0, 1, True, q, k, v, score, score_out=score)
    ref, tol, w, wt = _reference(torch, B, ctx, kv, 0, 1, True, q, k, v)
    torch.cuda.synchronize()
    _check(torch, o, ref, tol, "after the eviction")
    assert bool(torch.isfinite(s2).all())


@pytest.mark.parametrize("in_place", [False, True])
def test_sums_go_on_behind_an_eviction(env, in_place):
    """The sums of the positions that stay are carried on at their new places, those of new positions begin at nothing."""
    torch, B, ctx = env
    from tests.test_gpu_shared_attention import _cache, _inputs, _reference
    n_kv, n, held = 2, 300, 117
    kv = _cache(torch, B, ctx, n_kv, 0, [n, n])
    dst = 0 if in_place else 1
    (q,), (k,), (v,) = _inputs(torch, 1, [3], [3], 8, n_kv)
    _, score = B.cas_attention_weights(ctx, kv, 0, 0, True, q, k, v)
    before = score.clone()
    index = B.cas_kv_select(ctx, score, n, held, 4, 16, kept=score)
    B.cas_kv_evict(ctx, kv, 0, 1, 0, dst, index.view(1, n_kv, held))
    B.cas_kv_set_len(kv, dst, held)
    torch.cuda.synchronize()
    assert torch.equal(score[:, :held], before.gather(1, index.long())) and torch.equal(score[:, held:], before[:, held:])
    (q,), (k,), (v,) = _inputs(torch, 1, [2], [2], 8, n_kv, seed=6)
    after = torch.full_like(score, 9.0)
    B.cas_attention_weights(ctx, kv, 0, dst, True, q, k, v, score, score_out=after)
    _, _, w, wt = _reference(torch, B, ctx, kv, 0, dst, True, q, k, v)
    torch.cuda.synchronize()
    want = w.clone()
    want[:, :held] += score[:, :held].double()
    err = (after[:, :held + 2].double() - want).abs()     # the sum's own rounding beside the weights' tolerance
    assert bool((err <= wt + 2.0 ** -24 * want).all()), float((err / wt).max())
    assert bool((after[:, held + 2:] == 9.0).all())


def test_as_many_rows_as_a_launch_has(env):
    torch, B, ctx = env
    rows = 1 << 22
    score = torch.arange(rows, dtype=torch.float32, device="cuda").view(rows, 1)
    index = torch.full((rows, 1), 7, dtype=torch.int32, device="cuda")
    with pytest.raises(B.CasError) as e:
        B.cas_kv_select(ctx, score, 1, 1, index=index)
    assert e.value.code == B.CAS_ENOTSUP
    torch.cuda.synchronize()
    assert bool((index == 7).all())
    kept = torch.zeros(rows, 1, device="cuda")
    B.cas_kv_select(ctx, score[1:], 1, 1, index=index[1:], kept=kept[1:])
    torch.cuda.synchronize()
    assert int(index[0]) == 7 and bool((index[1:] == 0).all()) and torch.equal(kept[1:], score[1:])
