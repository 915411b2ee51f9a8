"""cas_accept_tokens against the definition in 64 bits on the host: vocabularies from one token to large and odd ones, ragged
drafts, greedy sequences, rows with nothing or infinities in them, numbers at the ends of their range, strides, the distribution
of the tokens, captured calls, refusals."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2605_26558_amd import binding as B
    return torch, B, B.Context(workspace=torch.empty(64 << 20, dtype=torch.uint8, device="cuda"))


def _probabilities(z, t):
    """Softmax of a row at temperature t; NaN counts as -inf, of rows with +inf these alike, greedy on the first of the largest."""
    z = np.where(np.isnan(z), -np.inf, z.astype(np.float64))
    top = z.max()
    if top == -np.inf:
        return np.zeros(len(z))
    if not t > 0:
        return (np.arange(len(z)) == int(np.argmax(z))).astype(np.float64)
    with np.errstate(invalid="ignore", over="ignore"):
        w = np.where(z == top, 1.0, np.where(z == -np.inf, 0.0, np.exp((z - top) / np.float64(t))))
    w = np.where(np.isnan(w), 0.0, w)
    return w / w.sum()


def _reference(target, draft, tokens, ks, r, temp):
    """Per sequence (drafts kept, token behind them), and p, q of the drafted tokens."""
    V = target.shape[1]
    got, px, qx, d, row = [], [], [], 0, 0
    for s, k in enumerate(ks):
        t, w, n = 1.0 if temp is None else temp[s], None, 0
        for j in range(k):
            x = int(tokens[d + j])
            p = _probabilities(target[row + j], t)
            inside = 0 <= x < V
            q = (np.arange(V) == x).astype(np.float64) if draft is None else _probabilities(draft[d + j], t)
            px.append(p[x] if inside else 0.0)
            qx.append(q[x] if inside else 0.0)
            if w is None:
                with np.errstate(divide="ignore", invalid="ignore"):
                    good = inside and p[x] > 0 and r[row + j] <= p[x] / q[x]
                if good:
                    n += 1
                else:
                    w = np.maximum(0.0, p - q)
                    w = w if w.sum() > 0 else p
        if w is None:
            w = _probabilities(target[row + k], t)
        there = np.flatnonzero(w)
        token = -1
        if len(there):
            c = np.cumsum(w)
            over = np.flatnonzero((c > r[row + k] * c[-1]) & (w > 0))
            token = int(over[0] if len(over) else there[-1])
        got.append((n, token))
        d, row = d + k, row + k + 1
    return got, np.array(px), np.array(qx)


def _case(torch, vocab, ks, known=True, seed=1, sigma=2.5, off=0.5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n, S = sum(ks), len(ks)
    target = torch.randn(n + S, vocab, generator=g, device="cuda") * sigma
    rows = [i + s for s, i in zip([s for s, k in enumerate(ks) for _ in range(k)], range(n))]
    near = target[rows] + off * torch.randn(n, vocab, generator=g, device="cuda")
    tokens = torch.multinomial(torch.softmax(near, 1), 1, generator=g)[:, 0].int() if n else torch.empty(0, dtype=torch.int32, device="cuda")
    r = torch.rand(n + S, generator=g, device="cuda", dtype=torch.float64)
    temp = torch.rand(S, generator=g, device="cuda") + 0.4
    return target, near if known else None, tokens, r, temp


def _host(x):
    return None if x is None else x.cpu().numpy()


def _check(torch, B, ctx, target, near, tokens, ks, r, temp, what, **how):
    n, out, p, q = B.cas_accept_tokens(ctx, target, near, tokens, ks, r, temperature=temp, probs=True, **how)
    want, px, qx = _reference(_host(target), _host(near), _host(tokens), ks, _host(r), _host(temp))
    n, out, tokens, d = n.tolist(), out.tolist(), tokens.tolist(), 0
    for s, k in enumerate(ks):
        kept, token = want[s]
        assert n[s] == kept, (what, s, n[s], kept)
        assert out[s] == tokens[d:d + kept] + [token] + [-1] * (len(out[s]) - kept - 1), (what, s, out[s], token)
        d += k
    # 64-bit probabilities, rounded to fp32 once; smallest fp32 numbers keep fewer bits
    for got, ref in ((p, px), (q, qx)):
        assert np.all(np.abs(got.cpu().numpy() - ref) <= 2.0 ** -23 * ref + 2.0 ** -149), what


CASES = [  # vocabulary, drafts, known
    (1, [0], True), (1, [1, 0, 2], True), (2, [3], True), (3, [1, 1], False), (63, [2, 0, 5], True), (64, [64], True), (65, [0, 0, 0], True),
    (1000, [4], True), (4095, [3, 1], True), (4096, [2, 2], False), (4097, [5, 0, 1], True), (8193, [1] * 40, True), (32000, [4, 7], True),
    (50257, [7, 0, 3], False), (128256, [5, 6, 0, 2], True), (128256, [0] * 8, True), (262145, [2], True), (700000, [1, 0], False), (11, [1] * 256, True)]


@pytest.mark.parametrize("vocab,ks,known", CASES)
def test_tokens_against_the_definition(env, vocab, ks, known):
    torch, B, ctx = env
    for seed in (1, 2, 3):
        target, near, tokens, r, temp = _case(torch, vocab, ks, known, seed)
        _check(torch, B, ctx, target, near, tokens, ks, r, temp, (vocab, ks, known, seed))
        _check(torch, B, ctx, target, near, tokens, ks, r, None, (vocab, ks, known, seed, "no temperature"))
        temp[::2] = 0.0
        _check(torch, B, ctx, target, near, tokens, ks, r, temp, (vocab, ks, known, seed, "greedy"))


def test_far_apart_models_leave_the_draw_to_the_rest(env):
    """Drafts of a model that has little to do with the target: nearly all are dropped, and the rest p - q decides."""
    torch, B, ctx = env
    for vocab in (17, 5000, 128256):
        for seed in range(4):
            target, near, tokens, r, temp = _case(torch, vocab, [3] * 20, True, seed, off=6.0)
            _check(torch, B, ctx, target, near, tokens, [3] * 20, r, temp, (vocab, seed))


def test_rows_with_nothing_or_infinities(env):
    torch, B, ctx = env
    inf, nan, ks = math.inf, math.nan, [2] * 9
    for vocab in (9, 4099):
        target, near, tokens, r, temp = _case(torch, vocab, ks, True, 7)
        target[0] = -inf                       # no token in the first row
        near[2] = -inf                         # none in a draft's
        target[6:9] = -inf                     # none in all rows of a sequence
        target[9, 3:] = nan                    # NaN are no tokens
        near[6, ::2] = nan
        target[12, [2, 5]] = inf               # infinite ones are all there is
        near[8, [2, 7]] = inf
        tokens[8] = 5
        target[15], near[10] = -inf, -inf
        target[15, 4], near[10, 4], tokens[10] = 1.5, -3.0, 4    # one token in both
        target[18, :] = target[18, 0]          # all alike
        near[12, :] = near[12, 0]
        target[21, tokens[14].long()] = -inf   # a draft that the target rules out
        r[21] = 0.0
        near[16] = target[24]                  # equal rows: never dropped
        for t in (temp, None, torch.zeros_like(temp)):
            _check(torch, B, ctx, target, near, tokens, ks, r, t, (vocab, t is None))
            _check(torch, B, ctx, target, None, tokens, ks, r, t, (vocab, t is None, "certain"))


def test_numbers_at_the_ends(env):
    """0, the largest below 1, and numbers out of range, which take the first or the last token that has a weight."""
    torch, B, ctx = env
    ks = [2] * 8
    for vocab in (5, 5000):
        target, near, tokens, r, temp = _case(torch, vocab, ks, True, 5)
        target[:, 0], target[:, -1] = -math.inf, -math.inf
        for u in (0.0, 1.0 - 2.0 ** -53, 1.0, 2.5, -0.5):
            for v in (0.0, 0.5, 1.0 - 2.0 ** -53, 1.5):
                x = r.clone().view(-1, 3)
                x[:, 2], x[:, :2] = u, v
                _check(torch, B, ctx, target, near, tokens, ks, x.view(-1), temp, (vocab, u, v))
        near[:] = target.view(8, 3, -1)[:, :2].reshape(16, -1)   # p = q and a number above 1: nothing is left of p - q
        x = r.clone().view(-1, 3)
        x[:, :2] = 1.5
        _check(torch, B, ctx, target, near, tokens, ks, x.view(-1), temp, (vocab, "equal"))


@pytest.mark.parametrize("where", ["first", "middle", "last"])
@pytest.mark.parametrize("vocab", [8192, 12289])
def test_a_chunk_whose_tokens_are_all_below_the_smallest_number_is_not_drawn(env, vocab, where):
    """4096 tokens 740 below the others: exp(-740) / n is 0 in 64 bits (the smallest number is exp(-744.4)), 4096 times that
    is not.  The definition gives them no weight, whatever the number; 735 below they have one."""
    torch, B, ctx = env
    low = {"first": slice(0, 4096), "middle": slice(4096, 8192), "last": slice(vocab - (vocab % 4096 or 4096), vocab)}[where]
    for below, t in ((740.0, 1.0), (7.4, 0.01), (735.0, 1.0)):  # numbers away from the steps of the sums by more than their roundings
        row = torch.zeros(vocab, device="cuda")
        row[low] = -below
        temp = torch.full((6,), t, device="cuda")
        for u in (0.0, 0.3, 1.0 - 2.0 ** -40, 1.0):
            r = torch.tensor([u] * 6, dtype=torch.float64, device="cuda")
            z = row.expand(6, -1).contiguous()
            none = torch.empty(0, dtype=torch.int32, device="cuda")
            _check(torch, B, ctx, z, None, none, [0] * 6, r, temp, (vocab, where, below, u, "no drafts"))
            # a draft that is kept, and one that is not where nothing is left of p - q
            tokens = torch.full((3,), 8191 if where == "first" else 0, dtype=torch.int32, device="cuda")
            for v in (0.0, 1.5):
                r = torch.tensor([v, u] * 3, dtype=torch.float64, device="cuda")
                _check(torch, B, ctx, z, z[:3], tokens, [1] * 3, r, temp[:3], (vocab, where, below, u, v))


@pytest.mark.parametrize("vocab", [1048577, (1 << 22) - 3, 1 << 22])
def test_vocabularies_of_more_than_256_chunks(env, vocab):
    """More chunks (4096 tokens) and pieces (2048) than a workgroup of the draw has threads: the token in the first of them, in
    later rounds and at the very end, out of p, of p - q with known drafts, and of p behind a certain draft."""
    torch, B, ctx = env
    g = torch.Generator(device="cuda").manual_seed(vocab)
    flat = torch.randn(3, vocab, generator=g, device="cuda") * 0.5
    high = flat.clone()
    high[:, vocab - 3000:] += 16.0      # nearly all of it in the last chunk or two
    low = flat.clone()
    low[:, 5:9] += 20.0
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    f64 = lambda *v: torch.tensor(v, dtype=torch.float64, device="cuda")  # noqa: E731
    for z, what in ((flat, "flat"), (high, "high"), (low, "low")):
        for us in ((0.0, 0.2503, 1.0 - 2.0 ** -30), (0.51, 0.7507, 0.99)):
            _check(torch, B, ctx, z, None, none, [0, 0, 0], f64(*us), None, (vocab, what, us, "draw"))
        for u in (0.0, 0.3001, 0.6002, 0.9995):
            tokens = torch.tensor([vocab - 2], dtype=torch.int32, device="cuda")
            near = torch.randn(1, vocab, generator=g, device="cuda") * 0.5
            for r in (1.0, 0.0):   # dropped (r above p / q unless the target is much the surer), kept
                _check(torch, B, ctx, z[:2], near, tokens, [1], f64(r, u), None, (vocab, what, u, r, "known"))
                _check(torch, B, ctx, z[:2], None, tokens, [1], f64(r, u), None, (vocab, what, u, r, "certain"))
    # greedy: the first of the largest, in a late chunk
    flat[0, vocab - 5] = flat[0, vocab - 2] = 60.0
    flat[1, 1048576 - 1] = 70.0
    for r in (1.0, 0.0):
        tokens = torch.tensor([vocab - 5], dtype=torch.int32, device="cuda")
        _check(torch, B, ctx, flat[:2], None, tokens, [1], f64(r, 0.5), torch.zeros(1, device="cuda"), (vocab, "greedy", r))
    _check(torch, B, ctx, flat, None, none, [0, 0, 0], f64(0.1, 0.5, 0.9), torch.zeros(3, device="cuda"), (vocab, "greedy draw"))


def test_drafted_tokens_outside_the_vocabulary_are_not_kept(env):
    torch, B, ctx = env
    target, near, tokens, r, temp = _case(torch, 301, [3] * 6, True, 3)
    tokens[0], tokens[4], tokens[8], tokens[9] = -1, 301, 2 ** 31 - 1, -2 ** 31
    r[::4] = 0.0
    _check(torch, B, ctx, target, near, tokens, [3] * 6, r, temp, "known")
    _check(torch, B, ctx, target, None, tokens, [3] * 6, r, temp, "certain")


def test_temperatures_from_nothing_to_infinity(env):
    torch, B, ctx = env
    temps = [0.0, -1.0, math.nan, 1e-45, 1e-30, 1e-3, 1.0, 50.0, 1e30, math.inf]
    ks = [2] * len(temps)
    for vocab in (40, 9000):
        target, near, tokens, r, _ = _case(torch, vocab, ks, True, 6)
        target[:, 5], near[:, 5] = -math.inf, -math.inf
        t = torch.tensor(temps, device="cuda")
        # exponents (z - max) / 1e30 and the like differ in the last bits of 64, which no token here lies within
        _check(torch, B, ctx, target, near, tokens, ks, r, t, vocab)


def test_rows_any_distance_apart_and_at_any_alignment(env):
    torch, B, ctx = env
    ks = [3, 0, 5]
    for vocab in (4100, 1001):
        target, near, tokens, r, temp = _case(torch, vocab, ks, True, 8)
        want = [x.cpu() for x in B.cas_accept_tokens(ctx, target, near, tokens, ks, r, temperature=temp, probs=True)]
        for pad in (1, 2, 3, 4, 61):
            wide = [torch.full((x.shape[0], vocab + pad), math.nan, device="cuda") for x in (target, near)]
            for w, x in zip(wide, (target, near)):
                w[:, pad:] = x
            out = torch.full((3, 9 + pad), 77, dtype=torch.int32, device="cuda")
            got = B.cas_accept_tokens(ctx, wide[0][:, pad:], wide[1][:, pad:], tokens, ks, r, temperature=temp, probs=True, out=out)
            assert torch.equal(got[0].cpu(), want[0]) and torch.equal(got[1].cpu()[:, :6], want[1]) and bool((got[1][:, 6:] == -1).all())
            assert torch.equal(got[2].cpu(), want[2]) and torch.equal(got[3].cpu(), want[3])


def test_tokens_come_out_with_the_targets_probabilities(env):
    """One draft each of 256 sequences, drawn from q: the first token out is distributed as p whatever q is."""
    torch, B, ctx = env
    V, S, rounds = 12, 256, 60
    g = torch.Generator(device="cuda").manual_seed(11)
    z = torch.randn(2, V, generator=g, device="cuda") * 1.5
    target, near = z[0].expand(2 * S, V).contiguous(), z[1].expand(S, V).contiguous()
    counts = torch.zeros(V, dtype=torch.int64)
    for _ in range(rounds):
        drawn = B.cas_accept_tokens(ctx, near, None, None, [0] * S, torch.rand(S, generator=g, device="cuda", dtype=torch.float64))[1][:, 0]
        out = B.cas_accept_tokens(ctx, target, near, drawn.contiguous(), [1] * S, torch.rand(2 * S, generator=g, device="cuda", dtype=torch.float64))[1]
        counts += torch.bincount(out[:, 0].cpu().long(), minlength=V)
    n, p = S * rounds, torch.softmax(z[0].double(), 0).cpu()
    # 5 standard deviations of each count: one of 12 is beyond by chance once in 10^5 seeds
    assert bool(((counts - n * p).abs() <= 5 * (n * p * (1 - p)).sqrt() + 1).all()), (counts, n * p)


def test_streams_and_captured_calls(env):
    """A context on a stream of its own; a captured call replayed over new inputs, with eager calls between, gives the eager tokens."""
    torch, B, _ = env
    ks, vocab = [4, 0, 2, 7], 20000
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        size = B.cas_accept_tokens_bytes(ks, vocab)
        ctx, eager = (B.Context(workspace=torch.empty(size, dtype=torch.uint8, device="cuda")) for _ in range(2))
        held = [x.clone() for x in _case(torch, vocab, ks, True, 1)]
        n, out = torch.empty(4, dtype=torch.int32, device="cuda"), torch.empty((4, 8), dtype=torch.int32, device="cuda")
        call = lambda c, xs, **how: B.cas_accept_tokens(c, xs[0], xs[1], xs[2], ks, xs[3], temperature=xs[4], **how)  # noqa: E731
        call(ctx, held, n_accepted=n, out=out)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            call(ctx, held, n_accepted=n, out=out)
        for seed in (2, 3, 4, 5):
            fresh = _case(torch, vocab, ks, True, seed)
            for h, f in zip(held, fresh):
                h.copy_(f)
            graph.replay()
            want = call(eager, fresh)
            stream.synchronize()
            assert torch.equal(n, want[0]) and torch.equal(out, want[1]), seed


def test_refusals(env):
    torch, B, ctx = env
    target, near, tokens, r, temp = _case(torch, 50, [2, 1], True, 1)
    lib, i32 = B._lib(), B._i32
    n, out = torch.empty(2, dtype=torch.int32, device="cuda"), torch.full((2, 4), 5, dtype=torch.int32, device="cuda")
    good = dict(ctx=ctx.h, S=2, ks=i32([2, 1]), vocab=50, target=target.data_ptr(), ldt=50, draft=near.data_ptr(), ldd=50, tokens=tokens.data_ptr(),
                temp=temp.data_ptr(), r=r.data_ptr(), n=n.data_ptr(), out=out.data_ptr(), ld_out=4, p=None, q=None)
    call = lambda **bad: lib.cas_accept_tokens(*{**good, **bad}.values())  # noqa: E731
    for bad in (dict(ctx=None), dict(S=-1), dict(ks=None), dict(ks=i32([2, -1])), dict(vocab=0), dict(target=None), dict(ldt=49), dict(ldd=49),
                dict(tokens=None), dict(r=None), dict(n=None), dict(out=None), dict(ld_out=2), dict(target=good["target"] + 2), dict(r=good["r"] + 4),
                dict(out=good["out"] + 1)):
        assert call(**bad) == B.CAS_EINVAL, bad
    for bad in (dict(ks=i32([65, 1]), ld_out=66), dict(vocab=(1 << 22) + 1, ldt=1 << 23, ldd=1 << 23), dict(S=257, ks=i32([0] * 257))):
        assert call(**bad) == B.CAS_ENOTSUP, bad
    small = B.Context(workspace=torch.empty(B.cas_accept_tokens_bytes([2, 1], 50) - 1, dtype=torch.uint8, device="cuda"))
    assert call(ctx=small.h) == B.CAS_ENOMEM and call(ctx=B.Context().h) == B.CAS_ENOMEM
    torch.cuda.synchronize()
    assert bool((out == 5).all())   # nothing was launched
    assert call(S=0, ks=None, target=None, r=None, n=None, out=None) == B.CAS_OK
    assert call() == B.CAS_OK
