"""Sampled speculative rounds of a one-layer windowed model out of the stand-alone calls, as a program would run them: drafts
drawn by cas_accept_tokens from the draft product's logits, cas_attention_window in both forms, verification by
cas_accept_tokens, and what was kept appended by cas_kv_append_rope."""
import numpy as np
import pytest

from test_gpu_accept import _reference as accept_reference
from test_gpu_window_attention import _check, _of_sequence

pytestmark = pytest.mark.gpu

HIDDEN, VOCAB, N_Q, N_KV, FIRST, WINDOW, K = 512, 1000, 4, 2, 4, 70, 3


class Windowed:
    """Embedding -> q, k, v -> attention within the window -> output head, for some sequences of one cache."""

    def __init__(self, torch, B, lens, keep, t, seed=1):
        self.torch, self.B = torch, B
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.ctx = ctx = B.Context(workspace=torch.empty(32 << 20, dtype=torch.uint8, device="cuda"))
        rnd = lambda *shape, sigma=1.0: (torch.randn(*shape, generator=g, device="cuda") * sigma).bfloat16()  # noqa: E731
        self.embed = rnd(VOCAB, HIDDEN)
        self.wqkv = B.cas_encode_weight(ctx, rnd((N_Q + 2 * N_KV) * 128, HIDDEN, sigma=HIDDEN ** -0.5), keep, t)
        self.head = B.cas_encode_weight(ctx, rnd(VOCAB, N_Q * 128, sigma=0.2), keep, t)
        S, pages = len(lens), 6
        self.kv = B.KVCache(ctx, 1, N_KV, S * pages, S, pages, keep_permille=keep, trunc_bits=t)
        cfg = B.cas_rope_cfg(128, B.CAS_ROPE_PLAIN, 10000.0, 1.0, 0, 0.0, 0.0, 1.0)
        self.angles = B.cas_rope_table(ctx, cfg, 0, 1024)
        self.prompts = [torch.randint(0, VOCAB, (n,), generator=g, device="cuda", dtype=torch.int32) for n in lens]
        self.extend(range(S), self.prompts)

    def project(self, tokens, exact):
        x = self.embed[tokens.long()]
        f = self.B.cas_gemm_verify if exact else self.B.cas_gemv_draft
        step = 16 if exact else 4
        y = self.torch.cat([f(self.ctx, self.wqkv, x[i:i + step].contiguous()) for i in range(0, len(x), step)])
        return y.unflatten(1, (-1, 128)).split((N_Q, N_KV, N_KV), 1)

    def extend(self, seqs, tokens):
        """Appends the exact keys and values of the tokens, all sequences at once."""
        B, counts = self.B, [len(t) for t in tokens]
        _, k, v = self.project(self.torch.cat(tokens), True)
        B.cas_kv_append_rope(self.ctx, self.kv, 0, seqs, counts, self.angles, k, v)
        for s, n in zip(seqs, counts):
            B.cas_kv_set_len(self.kv, s, B.cas_kv_len(self.kv, s) + n)

    def step(self, seqs, tokens, flight, exact, check=False):
        """Logits of the sequences' tokens (a column each, the last of those in flight); flight: per sequence the (k, v) before."""
        torch, B, ctx = self.torch, self.B, self.ctx
        cols = [len(t) for t in tokens]
        start = [B.cas_kv_len(self.kv, s) + (0 if f is None else len(f[0])) for s, f in zip(seqs, flight)]
        pos = torch.cat([torch.arange(a, a + c, dtype=torch.int32) for a, c in zip(start, cols)]).cuda()
        q, k, v = B.cas_rope(ctx, self.angles, self.project(torch.cat(tokens), exact), pos=pos, turn=(True, True, False))
        q, k, v = ([x.contiguous() for x in y.split(cols)] for y in (q, k, v))
        new = [(a, b) if f is None else (torch.cat([f[0], a]), torch.cat([f[1], b])) for f, a, b in zip(flight, k, v)]
        out = B.cas_attention_window(ctx, self.kv, 0, seqs, FIRST, WINDOW, exact, q, [n[0] for n in new], [n[1] for n in new])
        if check:
            for i, s in enumerate(seqs):
                kn, vn = (x.view(torch.bfloat16) for x in new[i])
                ref, tol = _of_sequence(torch, B, ctx, self.kv, 0, s, exact, q[i].view(torch.bfloat16), kn, vn, FIRST, WINDOW)
                _check(torch, out[i], ref, tol, (s, exact))
        x = torch.cat(out).flatten(1)
        f, n = (B.cas_gemm_verify, 16) if exact else (B.cas_gemv_draft, 4)
        return torch.cat([f(ctx, self.head, x[i:i + n].contiguous()) for i in range(0, len(x), n)]), new

    def round(self, seqs, pending, r, temp, check=False):
        """K drafts of every sequence, one verification; returns per sequence the tokens that follow the pending one."""
        torch, B, S = self.torch, self.B, len(seqs)
        flight, last, drafted, near = [None] * S, pending, [], []
        for i in range(K):
            logits, flight = self.step(seqs, [t.view(1) for t in last], flight, False, check)
            drawn = B.cas_accept_tokens(self.ctx, logits, None, None, [0] * S, r[:, i].contiguous(), temperature=temp)[1][:, 0]
            last = list(drawn)
            drafted.append(drawn)
            near.append(logits)
        drafted, near = torch.stack(drafted, 1), torch.stack(near, 1)
        columns = [torch.cat([p.view(1), d]) for p, d in zip(pending, drafted)]
        target, _ = self.step(seqs, columns, [None] * S, True, check)
        numbers = r[:, K:].contiguous().view(-1)
        tokens = drafted.reshape(-1).contiguous()
        n, out = B.cas_accept_tokens(self.ctx, target, near.flatten(0, 1), tokens, [K] * S, numbers, temperature=temp)
        if check:
            want = accept_reference(target.cpu().numpy(), near.flatten(0, 1).cpu().numpy(), tokens.cpu().numpy(), [K] * S, numbers.cpu().numpy(), temp.cpu().numpy())[0]
            assert [(a, o[a]) for a, o in zip(n.tolist(), out.tolist())] == [tuple(w) for w in want]
        n = n.tolist()
        self.extend(seqs, [c[:a + 1] for c, a in zip(columns, n)])
        return [o[:a + 1] for o, a in zip(out, n)]


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2605_26558_amd import binding as B
    return torch, B


def _run(torch, m, seqs, rounds, check, seed=3):
    g = torch.Generator(device="cuda").manual_seed(seed)
    temp = torch.tensor([0.8, 1.0, 0.0][:len(seqs)], device="cuda")
    streams = [[int(m.prompts[s][-1])] for s in seqs]
    kept = 0
    for _ in range(rounds):
        r = torch.rand(len(seqs), 2 * K + 1, generator=g, device="cuda", dtype=torch.float64)
        pending = [torch.tensor(s[-1], dtype=torch.int32, device="cuda") for s in streams]
        for s, t in zip(streams, m.round(seqs, pending, r, temp, check)):
            s.extend(t.tolist())
            kept += len(t) - 1
    return streams, kept


def test_rounds_of_a_batch(env):
    """Every step against its definition, and the cache of the rounds against one that was given the same tokens at once."""
    torch, B = env
    lens, rounds = [60, 130, 3], 6
    m = Windowed(torch, B, lens, 600, 4)
    streams, kept = _run(torch, m, [0, 1, 2], rounds, True)
    assert 0 < kept < 3 * K * rounds            # both ends of a verification were met
    again = Windowed(torch, B, lens, 600, 4)
    again.extend([0, 1, 2], [torch.tensor(s[:-1], dtype=torch.int32, device="cuda") for s in streams])
    for s in range(3):
        n = B.cas_kv_len(m.kv, s)
        assert n == B.cas_kv_len(again.kv, s) == lens[s] + len(streams[s]) - 1
        for a, b in zip(B.cas_kv_read(m.ctx, m.kv, 0, s, 0, n, True), B.cas_kv_read(m.ctx, again.kv, 0, s, 0, n, True)):
            assert torch.equal(a, b)


def test_a_draft_model_that_is_the_target_is_kept(env):
    """Nothing pruned, nothing cut off: p and q differ by the order of fp32 sums, and a draft is dropped once in some 10^5."""
    torch, B = env
    m = Windowed(torch, B, [40, 77], 1000, 0)
    streams, kept = _run(torch, m, [0, 1], 8, False)
    assert kept == 2 * K * 8


def test_graphs_of_one_context_in_turn(env):
    """A captured appending, attention and verification that share a context and its workspace, replayed in changing order over
    new inputs, give what a context of its own gives eagerly."""
    torch, B = env
    ks, vocab, lens, toks = [3, 0, 5], 9001, [200, 64, 1], [3, 1, 2]
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        size = max(B.cas_accept_tokens_bytes(ks, vocab), 1 << 22)
        shared, own = (B.Context(workspace=torch.empty(size, dtype=torch.uint8, device="cuda")) for _ in range(2))
        caches = [B.KVCache(c, 1, 2, 15, 3, 5) for c in (shared, own)]
        table = torch.randn(400, 64, 2, device="cuda").contiguous()

        def inputs(seed):
            g = torch.Generator(device="cuda").manual_seed(seed)
            rnd = lambda *s, **k: torch.randn(*s, generator=g, device="cuda", **k)  # noqa: E731
            heads = [rnd(sum(toks), h, 128) for h in (8, 2, 2)]
            flight = [rnd(t, h, 128).bfloat16().view(torch.int16) for h in (8, 2, 2) for t in toks]
            logits = [rnd(sum(ks) + 3, vocab), rnd(sum(ks), vocab)]
            tokens = torch.randint(0, vocab, (sum(ks),), generator=g, device="cuda", dtype=torch.int32)
            return heads, flight, logits, tokens, torch.rand(sum(ks) + 3, generator=g, device="cuda", dtype=torch.float64)

        def calls(ctx, kv, x):
            (q, k, v), f, (t, d), tokens, r = x
            return [lambda: [B.cas_kv_append_rope(ctx, kv, 0, [0, 1, 2], toks, table, k, v, q=q)],
                    lambda: B.cas_attention_window(ctx, kv, 0, [0, 1, 2], 4, 100, True, f[:3], f[3:6], f[6:]),
                    lambda: list(B.cas_accept_tokens(ctx, t, d, tokens, ks, r)[:2])]

        for kv in caches:
            for pool in (kv.spec_pool, kv.verif_pool):
                pool.zero_()
            for s, n in enumerate(lens):
                k = torch.randn(n, 2, 128, generator=torch.Generator(device="cuda").manual_seed(s), device="cuda").bfloat16().view(torch.int16)
                B.cas_kv_set_len(kv, s, 0)
                B.cas_kv_append(shared if kv is caches[0] else own, kv, 0, s, k, k)
                B.cas_kv_set_len(kv, s, n)
        held, graphs = inputs(1), []
        for f in calls(shared, caches[0], held):
            f()
            stream.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=stream):
                out = f()
            graphs.append((g, out))
        flat = lambda x: [t for p in x for t in (p if isinstance(p, list) else [p])]  # noqa: E731
        for seed, order in ((2, (0, 1, 2)), (3, (2, 1, 0)), (4, (1, 2, 0)), (5, (2, 0, 1))):
            fresh = inputs(seed)
            for h, f in zip(flat(held), flat(fresh)):
                h.copy_(f)
            eager = calls(own, caches[1], fresh)
            for i in order:
                graphs[i][0].replay()
                want = eager[i]()
                stream.synchronize()
                for a, b in zip(graphs[i][1], want):
                    assert torch.equal(a, b), (seed, i)
            assert torch.equal(caches[0].spec_pool, caches[1].spec_pool) and torch.equal(caches[0].verif_pool, caches[1].verif_pool), seed
