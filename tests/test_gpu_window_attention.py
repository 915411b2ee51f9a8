"""cas_attention_window against attention in 64 bits over the positions that each column sees, on the vectors that cas_kv_read
gives (checked bit for bit elsewhere): windows from one position to more than there are, first positions from none to all, edges
inside pages, formats, group sizes, lengths from nothing to far ones, infinities where a column does not see them, pages that were
given back, streams, captured calls, refusals."""
import math

import numpy as np
import pytest

import synth

pytestmark = pytest.mark.gpu

MOST = 2 ** 31 - 1


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2605_26558_amd import binding as B
    return torch, B, B.Context(workspace=torch.empty(256 << 20, dtype=torch.uint8, device="cuda"))


def _bits(torch, a):
    return torch.from_numpy(np.ascontiguousarray(a).view(np.int16)).cuda()


def _cache(torch, B, ctx, n_kv, lens, keep=600, t=4, mode=0, layers=1, layer=0, plant=None):
    """plant(s, k, v): changes the vectors (bit patterns) of a sequence before they are appended."""
    most = max((n + 64 + 63) // 64 for n in lens)
    rng = np.random.Generator(np.random.Philox(7))
    place = rng.permutation(len(lens) * most).astype(np.int32).reshape(len(lens), most)
    kv = B.KVCache(ctx, layers, n_kv, place.size, len(lens), most, keep_permille=keep, trunc_bits=t, exp_mode=mode, page_table=torch.from_numpy(place))
    for s, n in enumerate(lens):
        k = synth.kv_tensor(max(n, 1), n_kv, 128, seed=20 + s)[:n]
        v = synth.kv_tensor(max(n, 1), n_kv, 128, seed=60 + s, outlier_channels=0)[:n]
        if plant:
            k, v = k.copy(), v.copy()
            plant(s, k, v)
        if n:
            B.cas_kv_append(ctx, kv, layer, s, _bits(torch, k), _bits(torch, v))
        B.cas_kv_set_len(kv, s, n)
    return kv


def _inputs(torch, cols, news, nq, n_kv, seed=5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda n, h, s: (torch.randn(n, h, 128, device="cuda", generator=g) * s).bfloat16()  # noqa: E731
    return [r(c, nq, 0.5) for c in cols], [r(n, n_kv, 1.0) for n in news], [r(n, n_kv, 1.0) for n in news]


def _reference(torch, k, v, place, own, q, first, window):
    """(output, its tolerance) in 64 bits.  k, v: [positions, heads, 128] at the places `place`; own: the columns' places."""
    (C, nq), H = q.shape[:2], k.shape[1]
    G = nq // H
    k, v = k.double().transpose(0, 1), v.double().transpose(0, 1)
    qh = q.double().view(C, H, G, 128).permute(1, 0, 2, 3).reshape(H, C * G, 128)
    sc = torch.matmul(qh, k.transpose(1, 2).contiguous()) / math.sqrt(128.0)
    big = torch.matmul(qh.abs(), k.abs().transpose(1, 2).contiguous()) / math.sqrt(128.0)
    own = own.repeat_interleave(G)[:, None]
    seen = (place <= own) & ((place < first) | (place > own - window))
    sc = sc.masked_fill(~seen, -math.inf)
    p = torch.softmax(sc, 2)
    o, mean = torch.empty(H, C * G, 128, dtype=torch.float64, device="cuda"), torch.empty(H, C * G, 128, dtype=torch.float64, device="cuda")
    for i in range(C * G):  # row by row, so that what a row does not see is no factor of it
        row = torch.where(seen[i][:, None], v, 0.0)
        o[:, i] = (p[:, i, :, None] * row).sum(1)
        mean[:, i] = (p[:, i, :, None] * row.abs()).sum(1)
    # as for attention over a shared prefix: scores as 128 fp32 additions of exact products and a scaling, in the exponent; the
    # exponential's rounding; the sum they are divided by; weights as a bf16 head and the rounding of the rest; the output's rounding
    n = place.numel()
    rel = 2.0 ** -23 * (70 * big.masked_fill(~seen, 0.0) + 8)
    rel = rel + (p * rel).sum(2, keepdim=True) + 2.0 ** -24 * (64 + n / 16)
    tol = 2.0 ** -8 * o.abs() + (2.0 ** -15 + 2.0 ** -24 * (64 + n / 4) + rel.amax(2, keepdim=True)) * mean
    shape = lambda x: x.view(H, C, G, 128).transpose(0, 1).reshape(C, nq, 128)  # noqa: E731
    return shape(o), shape(tol)


def _of_sequence(torch, B, ctx, kv, layer, s, full, q, kn, vn, first, window):
    n = B.cas_kv_len(kv, s)
    k, v = kn.double(), vn.double()
    if n:
        kc, vc = B.cas_kv_read(ctx, kv, layer, s, 0, n, full)
        k, v = (torch.cat([a.view(torch.bfloat16).double(), b]) for a, b in ((kc, k), (vc, v)))
    total, C = n + kn.shape[0], q.shape[0]
    return _reference(torch, k, v, torch.arange(total, device="cuda"), torch.arange(total - C, total, device="cuda"), q, first, window)


def _check(torch, out, ref, tol, what):
    got = out.view(torch.bfloat16).double()
    finite = torch.isfinite(ref)
    assert torch.equal(torch.isnan(got), torch.isnan(ref)), what
    assert torch.equal(got[~finite & ~torch.isnan(ref)], ref[~finite & ~torch.isnan(ref)]), what
    err, tol = (got - ref).abs()[finite], tol[finite]
    assert bool((err <= tol).all()), (what, float((err / tol).max()))


CASES = [  # kv heads, group, lengths, columns, in flight, full, keep, t, mode
    (2, 2, [0], [1], [1], False, 600, 4, 0),
    (2, 4, [150, 0, 64], [1, 1, 1], [1, 3, 2], False, 600, 4, 0),
    (2, 4, [333, 128, 127], [5, 7, 1], [5, 9, 64], True, 600, 4, 0),
    (3, 5, [700, 65, 1], [16, 3, 2], [16, 3, 40], True, 600, 4, 0),
    (8, 4, [1029, 500, 3, 64], [1] * 4, [4, 1, 2, 1], False, 600, 4, 2),
    (2, 8, [512] * 9, [2] * 9, [2] * 9, True, 600, 4, 2),
    (1, 48, [200, 321], [16, 1], [16, 1], True, 700, 3, 0),        # more rows than a workgroup takes
    (1, 16, [400], [16], [20], False, 700, 3, 2),                  # sixteen tiles, two pages a step
    (1, 1, [3100], [1], [1], False, 500, 7, 0),
    (4, 2, [130 + i for i in range(32)], [1] * 32, [1] * 32, False, 250, 0, 0),
    (2, 1, [300, 290], [1, 7], [1, 7], True, 1000, 5, 0),
    (2, 4, [192, 70], [2, 16], [2, 16], False, 0, 1, 2),
    (2, 3, [449], [6], [6], True, 333, 2, 0),
    (1, 7, [2500], [9], [30], True, 600, 6, 2),
]
WINDOWS = [(0, 1), (1, 1), (0, 2), (4, 16), (4, 64), (0, 63), (63, 65), (64, 100), (65, 130), (200, 37), (4, 256), (0, 1000), (MOST, 5), (0, MOST), (MOST, MOST)]


@pytest.mark.parametrize("n_kv,grp,lens,cols,news,full,keep,t,mode", CASES)
def test_outputs_against_64_bits(env, n_kv, grp, lens, cols, news, full, keep, t, mode):
    torch, B, ctx = env
    kv = _cache(torch, B, ctx, n_kv, lens, keep, t, mode, layers=2, layer=1)
    q, kn, vn = _inputs(torch, cols, news, n_kv * grp, n_kv)
    for first, window in WINDOWS:
        print("case", n_kv, grp, lens, cols, news, full, keep, t, mode, first, window, flush=True)
        outs = B.cas_attention_window(ctx, kv, 1, range(len(lens)), first, window, full, q, kn, vn)
        for s in range(len(lens)):
            ref, tol = _of_sequence(torch, B, ctx, kv, 1, s, full, q[s], kn[s], vn[s], first, window)
            _check(torch, outs[s], ref, tol, (s, first, window))


def test_a_long_cache_in_many_runs(env):
    torch, B, ctx = env
    for full, mode, cols in ((False, 0, 1), (True, 2, 7)):
        lens = [20011, 9000]
        kv = _cache(torch, B, ctx, 2, lens, mode=mode)
        q, kn, vn = _inputs(torch, [cols, 1], [cols + 2, 3], 8, 2)
        for first, window in ((4, 4096), (1000, 6001), (0, 19000)):
            outs = B.cas_attention_window(ctx, kv, 0, [0, 1], first, window, full, q, kn, vn)
            for s in range(2):
                ref, tol = _of_sequence(torch, B, ctx, kv, 0, s, full, q[s], kn[s], vn[s], first, window)
                _check(torch, outs[s], ref, tol, (full, s, first, window))


def test_positions_near_the_end_of_32_bits(env):
    """A table of 17 million pages of which the last hold the window, the first the first positions, and the rest was given back."""
    torch, B, ctx = env
    length, n_kv, first, window, cols = (1 << 30) + 37, 2, 70, 200, 5
    pages = (length + 64 + 63) // 64
    table = torch.full((1, pages), -7, dtype=torch.int32)
    table[0, :2] = torch.tensor([3, 9])
    start = (length - 300) // 64
    table[0, start:] = torch.tensor([1, 4, 0, 2, 8, 5, 7, 6][:pages - start])
    kv = B.KVCache(ctx, 1, n_kv, 10, 1, pages, page_table=table)
    g = torch.Generator(device="cuda").manual_seed(3)
    rnd = lambda n: torch.randn(n, n_kv, 128, generator=g, device="cuda").bfloat16()  # noqa: E731
    front, back = [rnd(128) for _ in range(2)], [rnd(length - start * 64) for _ in range(2)]
    for at, (k, v) in ((0, front), (start * 64, back)):
        B.cas_kv_set_len(kv, 0, at)
        B.cas_kv_append(ctx, kv, 0, 0, k, v)
    B.cas_kv_set_len(kv, 0, length)
    q, kn, vn = _inputs(torch, [cols], [cols + 1], 8, n_kv)
    assert B.cas_attention_window_bytes(kv, [0], first, window, [cols], 8, [cols + 1]) < 1 << 20
    out = B.cas_attention_window(ctx, kv, 0, [0], first, window, True, q, kn, vn)[0]
    total = length + cols + 1
    place = torch.cat([torch.arange(128, device="cuda"), torch.arange(start * 64, total, device="cuda")])
    k, v = (torch.cat([a, b, c]) for a, b, c in zip(front, back, (kn[0], vn[0])))
    ref, tol = _reference(torch, k, v, place, torch.arange(total - cols, total, device="cuda"), q[0], first, window)
    _check(torch, out, ref, tol, "far")


@pytest.mark.parametrize("full,mode", [(True, 0), (False, 0), (True, 2), (False, 2)])
def test_what_a_column_does_not_see_does_not_reach_it(env, full, mode):
    """Infinities and NaN below the window, at its lower edge (where the first columns see them), and in flight."""
    torch, B, ctx = env
    INF, NINF, NAN = 0x7F80, 0xFF80, 0x7FC0
    for length, cols, new, first, window in ((400, 9, 9, 4, 100), (333, 16, 16, 0, 64), (333, 16, 20, 70, 77), (130, 3, 3, 0, 2), (70, 5, 60, 1, 30),
                                             (64, 16, 16, 0, 16), (255, 16, 16, 0, 17)):
        total = length + new
        lowest = total - cols + 1 - window
        edge = [p for p in range(max(lowest, first), min(lowest + cols - 1, length))]

        def plant(s, k, v):
            for p in range(first, max(first, min(lowest, length))):  # nobody sees these
                k[p], v[p] = (INF, NAN) if p % 2 else (NAN, NINF)
            for i, p in enumerate(edge):
                if i % 3 != 1:
                    v[p, :, i::17] = INF if i % 2 else NINF
                if i == 5:
                    v[p, :, 3] = NAN

        kv = _cache(torch, B, ctx, 2, [length], mode=mode, plant=plant)
        q, kn, vn = _inputs(torch, [cols], [new], 6, 2)
        for at in (new - 1, new - cols + 1):  # in flight: seen by the last columns only
            vn[0][at, :, 11 + at] = math.inf
        hidden = max(0, min(lowest - length, new))
        if first <= length:
            kn[0][:hidden], vn[0][:hidden] = math.nan, math.inf
        out = B.cas_attention_window(ctx, kv, 0, [0], first, window, full, q, kn, vn)[0]
        kc, vc = B.cas_kv_read(ctx, kv, 0, 0, 0, length, full)
        k, v = (torch.cat([a.view(torch.bfloat16), b[0]]) for a, b in ((kc, kn), (vc, vn)))
        bad = torch.isnan(k).any(2).any(1) | torch.isinf(k).any(2).any(1)
        k = torch.where(bad[:, None, None], 0.0, k)  # in the scores of positions that are masked
        ref, tol = _reference(torch, k, v, torch.arange(total, device="cuda"), torch.arange(total - cols, total, device="cuda"), q[0], first, window)
        _check(torch, out, ref, tol, (length, cols, new, first, window))


@pytest.mark.parametrize("full,mode", [(True, 0), (False, 0), (True, 2), (False, 2)])
@pytest.mark.parametrize("grp", [1, 4, 8, 16, 48])
def test_edges_of_windows_in_every_kind_of_workgroup(env, grp, full, mode):
    """2, 4, 8 and 16 tiles of rows, and several workgroups for the rows of a sequence (48): infinities and NaN among the positions
    that only some of sixteen columns see, in one page, over the border of two, in the last pages and far from them."""
    torch, B, ctx = env
    for length, new, first, window in ((333, 16, 0, 64), (333, 20, 70, 77), (255, 16, 0, 17), (2000, 16, 5, 910), (2000, 40, 0, 1000), (1100, 16, 0, 600)):
        cols, total = 16, length + new
        lowest = total - cols + 1 - window
        edge = [p for p in range(max(lowest, first), min(lowest + cols - 1, length))]

        def plant(s, k, v):
            for p in range(max(first, lowest - 70), max(first, min(lowest, length))):  # nobody sees these
                k[p], v[p] = (0x7F80, 0x7FC0) if p % 2 else (0x7FC0, 0xFF80)
            for i, p in enumerate(edge):
                if i % 4 != 1:
                    v[p, i % 2, i::19] = 0x7F80 if i % 2 else 0xFF80
                if i % 7 == 5:
                    v[p, :, 3 * i] = 0x7FC0

        print("case", grp, full, mode, length, new, first, window, flush=True)
        kv = _cache(torch, B, ctx, 2, [length, 90], mode=mode, plant=lambda s, k, v: plant(s, k, v) if s == 0 else None)
        q, kn, vn = _inputs(torch, [cols, 1], [new, 1], 2 * grp, 2)
        out = B.cas_attention_window(ctx, kv, 0, [1, 0], first, window, full, q[::-1], kn[::-1], vn[::-1])[1]
        kc, vc = B.cas_kv_read(ctx, kv, 0, 0, 0, length, full)
        k, v = (torch.cat([a.view(torch.bfloat16), b[0]]) for a, b in ((kc, kn), (vc, vn)))
        bad = ~torch.isfinite(k).all(2).all(1)
        k = torch.where(bad[:, None, None], 0.0, k)  # in the scores of positions that are masked
        ref, tol = _reference(torch, k, v, torch.arange(total, device="cuda"), torch.arange(total - cols, total, device="cuda"), q[0], first, window)
        # infinities and NaN are the largest magnitudes of their vectors, so they are kept, and in a draft too
        assert bool((~torch.isfinite(ref)).any()) and bool(torch.isfinite(ref).any())
        _check(torch, out, ref, tol, (grp, length, new, first, window))


@pytest.mark.parametrize("n_kv,grp,lens,cols,news,full,keep,t,mode", [
    (1, 16, [400, 3000], [16, 9], [16, 20], True, 600, 4, 2), (1, 48, [700], [16], [16], True, 700, 3, 2), (2, 17, [1500], [15], [15], True, 600, 6, 2),
    (1, 20, [900, 64], [13, 16], [13, 64], True, 500, 5, 0)])
def test_many_rows_exact(env, n_kv, grp, lens, cols, news, full, keep, t, mode):
    test_outputs_against_64_bits(env, n_kv, grp, lens, cols, news, full, keep, t, mode)


@pytest.mark.parametrize("full,mode", [(True, 0), (False, 0), (True, 2), (False, 2)])
def test_an_infinity_that_every_column_sees_stays_in_its_channel(env, full, mode):
    """(Under a shared exponent the other values of its 32 channels lose their bits; they are what cas_kv_read gives.)"""
    torch, B, ctx = env

    def plant(s, k, v):
        v[250, :, 7], v[260, 0, 40], v[2, 1, 90] = 0x7F80, 0xFF80, 0x7FC0
    for mode_cols in (1, 3, 16):
        kv = _cache(torch, B, ctx, 2, [300], mode=mode, plant=plant)
        q, kn, vn = _inputs(torch, [mode_cols], [mode_cols], 12, 2)
        out = B.cas_attention_window(ctx, kv, 0, [0], 4, 100, full, q, kn, vn)[0].double()
        ref, tol = _of_sequence(torch, B, ctx, kv, 0, 0, full, q[0], kn[0], vn[0], 4, 100)
        touched = ~torch.isfinite(ref)
        assert torch.equal(touched, ~torch.isfinite(out)) and int(touched.sum()) == mode_cols * (12 + 6 + 6)
        assert bool(((out - ref).abs() <= tol)[~touched].all())


@pytest.mark.parametrize("full", [False, True])
def test_pages_behind_the_window_may_be_given_back(env, full):
    torch, B, ctx = env
    lens, cols = [1000, 700, 90], [4, 1, 2]
    kv = _cache(torch, B, ctx, 2, lens)
    q, kn, vn = _inputs(torch, cols, cols, 8, 2)
    for first, window in ((4, 100), (65, 64), (0, 1), (0, 300)):
        want = B.cas_attention_window(ctx, kv, 0, [0, 1, 2], first, window, full, q, kn, vn)
        table = kv.page_table.clone()
        for s, (n, c) in enumerate(zip(lens, cols)):
            low = max(0, n + c - c + 1 - window) // 64
            for p in range((first + 63) // 64, low):
                kv.page_table[s, p] = (-1, 2 ** 31 - 1, kv.desc.n_pages, -2 ** 31)[p % 4]
            kv.page_table[s, (n + 63) // 64:] = -3   # pages of in-flight positions alone need none yet
        got = B.cas_attention_window(ctx, kv, 0, [0, 1, 2], first, window, full, q, kn, vn)
        for a, b in zip(got, want):
            assert torch.equal(a, b), (first, window)
        kv.page_table.copy_(table)
    kv.page_table[0, 14:] = 2 ** 31 - 1              # one that is needed: wrong values, no access outside the pools
    out = B.cas_attention_window(ctx, kv, 0, [0], 4, 100, full, q[:1], kn[:1], vn[:1])
    torch.cuda.synchronize()
    assert out[0].shape == q[0].shape


def test_a_sequences_values_do_not_depend_on_the_others(env):
    torch, B, ctx = env
    cols, new = [2, 2, 2], [2, 2, 2]
    kv = _cache(torch, B, ctx, 2, [900, 333, 20, 3000, 64, 1500])
    q, kn, vn = _inputs(torch, cols, new, 8, 2)
    a = B.cas_attention_window(ctx, kv, 0, [0, 1, 2], 4, 500, True, q, kn, vn)
    b = B.cas_attention_window(ctx, kv, 0, [0, 3, 4], 4, 500, True, [q[0], q[2], q[1]], [kn[0], kn[2], kn[1]], [vn[0], vn[2], vn[1]])
    c = B.cas_attention_window(ctx, kv, 0, [5, 4, 0], 4, 500, True, [q[2], q[1], q[0]], [kn[2], kn[1], kn[0]], [vn[2], vn[1], vn[0]])
    assert torch.equal(a[0], b[0]) and torch.equal(a[0], c[2])


def test_streams_and_two_captured_calls_side_by_side(env):
    """Two captured calls, each with a context and a workspace of its own, replayed together over new inputs."""
    torch, B, _ = env
    lens, cols = [500, 90], [3, 1]
    kv = _cache(torch, B, B.Context(), 2, lens)
    torch.cuda.synchronize()
    sides = []
    for window in (100, 300):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            size = B.cas_attention_window_bytes(kv, [0, 1], 4, window, cols, 8, cols)
            ctx = B.Context(workspace=torch.empty(size, dtype=torch.uint8, device="cuda"))
            held = _inputs(torch, cols, cols, 8, 2)
            outs = [torch.empty_like(x) for x in held[0]]
            B.cas_attention_window(ctx, kv, 0, [0, 1], 4, window, True, *held, outs=outs)
            stream.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                B.cas_attention_window(ctx, kv, 0, [0, 1], 4, window, True, *held, outs=outs)
        sides.append((window, stream, ctx, held, outs, graph))
    eager = B.Context(workspace=torch.empty(1 << 24, dtype=torch.uint8, device="cuda"))
    for seed in range(2, 7):
        fresh = _inputs(torch, cols, cols, 8, 2, seed)
        torch.cuda.synchronize()
        for window, stream, ctx, held, outs, graph in sides:
            with torch.cuda.stream(stream):
                for hs, fs in zip(held, fresh):
                    for h, f in zip(hs, fs):
                        h.copy_(f)
                graph.replay()
        for window, stream, ctx, held, outs, graph in sides:
            want = B.cas_attention_window(eager, kv, 0, [0, 1], 4, window, True, *fresh)
            torch.cuda.synchronize()
            for a, b in zip(outs, want):
                assert torch.equal(a, b), (window, seed)


def test_refusals(env):
    torch, B, ctx = env
    kv = _cache(torch, B, ctx, 2, [100, 20])
    q, kn, vn = _inputs(torch, [2, 1], [2, 1], 8, 2)
    lib, i32 = B._lib(), B._i32
    out = [torch.zeros_like(x) for x in q]
    import ctypes as C
    ptr = lambda ts: (C.c_void_p * len(ts))(*[t if t is None or isinstance(t, int) else t.data_ptr() for t in ts])  # noqa: E731
    good = dict(ctx=ctx.h, kv=kv.h, layer=0, n=2, seqs=i32([0, 1]), first=4, window=50, full=1, q=ptr(q), cols=i32([2, 1]), heads=8, k=ptr(kn),
                v=ptr(vn), new=i32([2, 1]), o=ptr(out))
    call = lambda **bad: lib.cas_attention_window(*{**good, **bad}.values())  # noqa: E731
    for bad in (dict(ctx=None), dict(kv=None), dict(layer=1), dict(layer=-1), dict(n=0), dict(n=33), dict(seqs=i32([0, 0])), dict(seqs=i32([0, 2])),
                dict(seqs=None), dict(first=-1), dict(window=0), dict(window=-5), dict(cols=i32([17, 1]), new=i32([17, 1])), dict(cols=i32([0, 1])),
                dict(new=i32([1, 1])), dict(new=i32([65, 1])), dict(heads=7), dict(heads=2 * 49), dict(q=None), dict(k=ptr([kn[0], None])),
                dict(v=ptr([vn[0].data_ptr() + 2, vn[1]])), dict(o=None)):
        assert call(**bad) == B.CAS_EINVAL, bad
    need = B.cas_attention_window_bytes(kv, [0, 1], 4, 50, [2, 1], 8, [2, 1])
    small = B.Context(workspace=torch.empty(need - 1, dtype=torch.uint8, device="cuda"))
    assert call(ctx=small.h) == B.CAS_ENOMEM and call(ctx=B.Context().h) == B.CAS_ENOMEM
    B.cas_kv_set_len(kv, 0, kv.desc.max_pages_per_seq * 64)
    assert call() == B.CAS_ENOMEM
    B.cas_kv_set_len(kv, 0, 100)
    torch.cuda.synchronize()
    assert not any(bool(o.any()) for o in out)
    assert B.cas_attention_window_bytes(kv, [0, 1], -1, 50, [2, 1], 8, [2, 1]) == 0 == B.cas_attention_window_bytes(kv, [0, 1], 4, 0, [2, 1], 8, [2, 1])
    assert call() == B.CAS_OK
