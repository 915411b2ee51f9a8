"""Host parts of cas_kv_append_rope, cas_attention_window and cas_accept_tokens: refusals and sizes that need no device, and what
the wrappers take."""
import ctypes as C
import math
import types

import pytest


def _kv(B, n_kv=2, pages=8, seqs=3, per_seq=8):
    """A cache object without memory behind it: nothing here reaches a launch."""
    d = B.cas_kv_desc()
    d.n_layers, d.n_kv_heads, d.head_dim, d.page_tokens, d.n_pages, d.max_seqs, d.max_pages_per_seq = 1, n_kv, 128, 64, pages, seqs, per_seq
    d.fmt = B.cas_fmt(600, 4, 0)
    assert B._lib().cas_kv_desc_init(C.byref(d)) == B.CAS_OK
    h = C.c_void_p()
    assert B._lib().cas_kv_create(C.byref(d), 4096, 4096, 4096, C.byref(h)) == B.CAS_OK
    return types.SimpleNamespace(h=h, desc=d)


def test_refusals_without_a_device():
    from paper_2605_26558_amd import binding as B
    lib, one = B._lib(), (C.c_int32 * 1)(1)
    assert lib.cas_kv_append_rope(None, None, 0, 1, one, one, None, 4, 64, 0, None, None, None, None) == B.CAS_EINVAL
    assert lib.cas_attention_window(None, None, 0, 1, one, 0, 8, 1, None, one, 8, None, None, one, None) == B.CAS_EINVAL
    assert lib.cas_accept_tokens(None, 1, one, 10, None, 10, None, 0, None, None, None, None, None, 2, None, None) == B.CAS_EINVAL
    assert lib.cas_attention_window_bytes(None, 1, one, 0, 8, one, 8, one) == 0


def test_sizes_of_the_verification():
    from paper_2605_26558_amd import binding as B
    size = B.cas_accept_tokens_bytes
    assert size([], 100) == 0 and size([0], 1) > 0
    # 16 bytes a chunk of 4096 tokens and row, 8 a piece of 2048 and sequence, 40 a sequence, each rounded up to 256
    assert size([4], 128256) == (9 * 32 * 16 + 255) // 256 * 256 + 512 + 256
    assert size([64] * 256, 1 << 22) == (2 * 64 + 1) * 256 * 1024 * 16 + 256 * 2048 * 8 + 256 * 40
    for ks, vocab in (([65], 10), ([-1], 10), ([0] * 257, 10), ([1], 0), ([1], (1 << 22) + 1)):
        assert size(ks, vocab) == 0, (ks, vocab)


def test_workspace_of_a_window_goes_by_what_is_seen():
    from paper_2605_26558_amd import binding as B
    kv = _kv(B, pages=8, per_seq=1 << 20)
    at = lambda length, first, window, cols=1: (B.cas_kv_set_len(kv, 0, length), B.cas_attention_window_bytes(kv, [0], first, window, [cols], 8, [cols]))[1]  # noqa: E731
    whole = at(1000, 0, 2 ** 31 - 1)
    assert whole == at(1000, 2 ** 31 - 1, 1) == at(1000, 0, 1001) and whole > at(1000, 0, 100)
    assert at(1000, 4, 100) == at(60_000_000 // 64 * 64 + 1000 % 64, 4, 100)   # a far end costs nothing
    assert at(1000, 4, 100) == at(1064, 4, 100)
    for first, window, cols, new, heads in ((-1, 5, 1, 1, 8), (0, 0, 1, 1, 8), (0, -3, 1, 1, 8), (0, 5, 17, 17, 8), (0, 5, 2, 1, 8), (0, 5, 1, 65, 8), (0, 5, 1, 1, 7)):
        assert B.cas_attention_window_bytes(kv, [0], first, window, [cols], heads, [new]) == 0
    assert B.cas_attention_window_bytes(kv, [0, 0], 0, 5, [1, 1], 8, [1, 1]) == 0
    B._lib().cas_kv_destroy(kv.h)


def test_lengths_stay_below_32_bits():
    """A page table that would reach past 2^31 positions: no call takes a length whose sums with what it adds would not fit."""
    from paper_2605_26558_amd import binding as B
    lib, room = B._lib(), 2 ** 31 - 256
    kv = _kv(B, per_seq=1 << 27)
    for length in (2 ** 31 - 1, 2 ** 31 - 64, room + 1):
        assert lib.cas_kv_set_len(kv.h, 0, length) == B.CAS_ENOMEM, length
    ctx, data = C.create_string_buffer(4096), 4096   # looked at before a launch only, which no call here reaches
    one = lambda *v: (C.c_int32 * len(v))(*v)  # noqa: E731
    part = C.byref(B.cas_rope_part(data, data, 256, 256, 2, 0, 0, 0))
    append = lambda seq, n, n_pos=0: lib.cas_kv_append_rope(ctx, kv.h, 0, 1, one(seq), one(n), data, n_pos, 64, 0, None, None, part, part)  # noqa: E731
    ptr = (C.c_void_p * 1)(data)
    window = lambda new: lib.cas_attention_window(ctx, kv.h, 0, 1, one(0), 0, 8, 1, ptr, one(1), 2, ptr, ptr, one(new), ptr)  # noqa: E731
    for short in (0, 1, 63):
        assert lib.cas_kv_set_len(kv.h, 0, room - short) == B.CAS_OK
        assert B.cas_attention_window_bytes(kv, [0], 4, 100, [1], 8, [short + 1]) == 0 and window(short + 1) == B.CAS_ENOMEM
        assert B.cas_attention_shared_bytes(kv, [0], 0, [1], 8, [short + 1]) == 0
        assert append(0, short + 1) == append(0, 2 ** 31 - 1) == B.CAS_ENOMEM
        assert lib.cas_kv_append(ctx, kv.h, 0, 0, data, data, short + 1) == lib.cas_kv_append(ctx, kv.h, 0, 0, data, data, 2 ** 31 - 1) == B.CAS_ENOMEM
        assert lib.cas_kv_read(ctx, kv.h, 0, 0, room - short, short + 1, 1, data, data) == B.CAS_EINVAL
        if short:  # what fits: as much workspace as at any other length, and no refusal
            assert append(0, short) == B.CAS_OK
            here = B.cas_attention_window_bytes(kv, [0], 4, 100, [1], 8, [short])
            B.cas_kv_set_len(kv, 1, (room - short) % 64 + 6400)
            assert here == B.cas_attention_window_bytes(kv, [1], 4, 100, [1], 8, [short]) > 0
    lib.cas_kv_destroy(kv.h)


def test_numbers_of_tokens_near_the_end_of_32_bits_are_refused():
    """A commit of 2^31 - 1 accepted drafts, and passes of as many columns: refused before anything is launched, lengths as they were."""
    from paper_2605_26558_amd import binding as B
    lib, kv, data, most = B._lib(), _kv(B, n_kv=1), 4096, 2 ** 31 - 1
    cfg = B.cas_model_cfg(256, 1, 1, 1, 128, 256, 300, 8, 512, 1e-5, 2)
    size = C.c_size_t()
    assert lib.cas_model_act_bytes(C.byref(cfg), C.byref(size)) == B.CAS_OK

    def tensor(rows, cols):
        t = B.cas_tensor()
        t.desc.rows, t.desc.cols, t.d_spec, t.d_verif = rows, cols, data, data
        return t
    layers = (B.cas_layer_weights * 1)(B.cas_layer_weights(tensor(384, 256), tensor(256, 128), tensor(512, 256), tensor(256, 256), data, data))
    w, m = B.cas_model_weights(layers, tensor(300, 256), data, data, data), C.c_void_p()
    assert lib.cas_model_create(C.byref(cfg), C.byref(w), data, size.value, C.byref(m)) == B.CAS_OK
    ctx, n, one = C.create_string_buffer(4096), C.c_int32(), lambda *v: (C.c_int32 * len(v))(*v)
    out = one(*[0] * 64)
    B.cas_kv_set_len(kv, 0, 5)
    for big in (most, most - 1, 8):
        assert lib.cas_commit(ctx, m, kv.h, 0, big) == B.CAS_EINVAL
        assert B.cas_kv_len(kv, 0) == 5
        assert lib.cas_draft_step(ctx, m, kv.h, 0, data, big, data, None) == B.CAS_EINVAL
        assert lib.cas_verify_step(ctx, m, kv.h, 0, data, big, data, None) == B.CAS_EINVAL
        assert lib.cas_verify_step_multi(ctx, m, kv.h, 2, one(0, 1), one(big, 1), data, data) == B.CAS_EINVAL
        assert lib.cas_spec_round(ctx, m, kv.h, 0, 1, big, out, C.byref(n)) == B.CAS_EINVAL
        assert lib.cas_spec_round_multi(ctx, m, kv.h, 2, one(0, 1), one(1, 1), big, out, out) == B.CAS_EINVAL
    lib.cas_model_destroy(m)
    lib.cas_kv_destroy(kv.h)


@pytest.fixture
def wrappers(monkeypatch):
    """The binding with tensors that say they are on the GPU and a context that is none: a call whose arguments the wrapper takes
    comes back from the library as CAS_EINVAL, one that it does not take raises AssertionError."""
    import torch
    from paper_2605_26558_amd import binding as B

    class OnGpu(torch.Tensor):
        is_cuda = True

    def check(rc, what):
        if rc != B.CAS_OK:
            raise B.CasError(rc, what)

    ctx = types.SimpleNamespace(_torch=torch, h=None, _check=check)
    kv = types.SimpleNamespace(h=None, desc=types.SimpleNamespace(n_kv_heads=2, head_dim=128))
    return torch, B, ctx, kv, lambda *shape, dtype=torch.bfloat16: torch.zeros(*shape, dtype=dtype).as_subclass(OnGpu)


def _taken(B, call):
    with pytest.raises((B.CasError, AssertionError)) as e:
        call()
    return isinstance(e.value, B.CasError) and e.value.code == B.CAS_EINVAL


def test_types_that_the_wrappers_take(wrappers):
    torch, B, ctx, kv, t = wrappers
    bits = (torch.bfloat16, torch.int16, torch.uint16)
    f32 = lambda *shape: t(*shape, dtype=torch.float32)  # noqa: E731
    table = f32(4, 64, 2)
    for dtype in (*bits, torch.float32, torch.float16, torch.float64, torch.int32):
        for i in range(3):
            x = [t(3, 4, 128), t(3, 2, 128), t(3, 2, 128)]
            x[i] = x[i].to(dtype).as_subclass(type(table))
            assert _taken(B, lambda: B.cas_kv_append_rope(ctx, kv, 0, [0], [3], table, x[1], x[2], q=x[0])) == (dtype in bits or dtype == torch.float32)
            y = [None, None, None]
            y[i] = t(*x[i].shape, dtype=dtype)
            assert _taken(B, lambda: B.cas_kv_append_rope(ctx, kv, 0, [0], [3], table, t(3, 2, 128), t(3, 2, 128), q=t(3, 4, 128), q_out=y[0], k_out=y[1],
                                                          v_out=y[2])) == (dtype in bits)
        for i in range(4):
            a = [t(1, 4, 128), t(1, 2, 128), t(1, 2, 128), t(1, 4, 128)]
            a[i] = a[i].to(dtype).as_subclass(type(table))
            assert _taken(B, lambda: B.cas_attention_window(ctx, kv, 0, [0], 4, 9, True, [a[0]], [a[1]], [a[2]], outs=[a[3]])) == (dtype in bits)
        target, near, tokens, r, temp = f32(3, 50), f32(2, 50), t(2, dtype=torch.int32), t(3, dtype=torch.float64), f32(1)
        accept = lambda a=target, b=near, c=tokens, d=r, e=temp, **how: B.cas_accept_tokens(ctx, a, b, c, [2], d, temperature=e, **how)  # noqa: E731
        assert _taken(B, accept) and _taken(B, lambda: accept(b=None)) and _taken(B, lambda: accept(e=None))
        assert _taken(B, lambda: accept(a=t(3, 50, dtype=dtype))) == (dtype == torch.float32) == _taken(B, lambda: accept(b=t(2, 50, dtype=dtype)))
        assert _taken(B, lambda: accept(c=t(2, dtype=dtype))) == (dtype == torch.int32) == _taken(B, lambda: accept(out=t(1, 3, dtype=dtype)))
        assert _taken(B, lambda: accept(d=t(3, dtype=dtype))) == (dtype == torch.float64)
        assert _taken(B, lambda: accept(e=t(1, dtype=dtype))) == (dtype == torch.float32)


def test_shapes_that_the_wrappers_do_not_take(wrappers):
    torch, B, ctx, kv, t = wrappers
    table = t(4, 64, 2, dtype=torch.float32)
    append = lambda q=t(3, 4, 128), k=t(3, 2, 128), v=t(3, 2, 128), toks=[3], **how: B.cas_kv_append_rope(ctx, kv, 0, [0], toks, table, k, v, q=q, **how)  # noqa: E731,B006
    assert _taken(B, append) and _taken(B, lambda: append(q=None))
    for bad in (dict(k=t(3, 3, 128)), dict(v=t(2, 2, 128)), dict(q=t(3, 4, 64)), dict(toks=[2]), dict(toks=[1, 2]), dict(k=t(3, 128, 2).transpose(1, 2)),
                dict(q=t(4, 3, 128).transpose(0, 1)), dict(pos=t(2, dtype=torch.int32)), dict(pos=t(3, dtype=torch.int64)), dict(q_out=t(3, 3, 128)),
                dict(k_out=t(3, 2, 64))):
        assert not _taken(B, lambda: append(**bad)), bad
    f32 = lambda *shape: t(*shape, dtype=torch.float32)  # noqa: E731
    accept = lambda a=f32(3, 50), b=f32(2, 50), c=t(2, dtype=torch.int32), d=t(3, dtype=torch.float64), **how: B.cas_accept_tokens(ctx, a, b, c, [2], d, **how)  # noqa: E731
    assert _taken(B, accept)
    for bad in (dict(a=f32(2, 50)), dict(b=f32(3, 50)), dict(b=f32(2, 51)), dict(c=t(3, dtype=torch.int32)), dict(c=None), dict(d=t(2, dtype=torch.float64)),
                dict(a=f32(50, 3).T), dict(temperature=f32(2)), dict(out=t(2, 3, dtype=torch.int32)), dict(n_accepted=t(2, dtype=torch.int32))):
        assert not _taken(B, lambda: accept(**bad)), bad
    for tensors in ((t(1, 4, 128), t(1, 3, 128), t(1, 3, 128)), (t(1, 4, 64), t(1, 2, 128), t(1, 2, 128)), (t(1, 4, 128), t(2, 2, 128), t(1, 2, 128))):
        assert not _taken(B, lambda: B.cas_attention_window(ctx, kv, 0, [0], 4, 9, True, *([x] for x in tensors), outs=[t(1, 4, 128)]))


def test_exponential_of_the_verification_in_64_bits():
    """exp2_64 of accept.hip, operation by operation: within 4e-14 of 2^y where that is a normal number, 1 at 0."""
    import os
    import re
    from decimal import Decimal, getcontext
    from fractions import Fraction
    import numpy as np
    import paper_2605_26558_amd as P
    getcontext().prec = 40
    text = open(os.path.join(os.path.dirname(P.__file__), "csrc", "accept.hip"), encoding="utf-8").read()
    body = text[text.index("constexpr double kPoly[] = {"):]
    steps = [float(x) for x in re.findall(r"[0-9][0-9.e+-]+", body[body.index("{"):body.index("}")])]
    assert len(steps) == 10

    def fma(a, b, c):
        return float(Fraction(a) * Fraction(b) + Fraction(c))
    rng = np.random.Generator(np.random.Philox(2))
    for y in [0.0, -1e-300, -1e-9, -0.5, -0.49999999999999994, -0.5000000000000001, -1.0, -1.5, -1021.9, *(-rng.exponential(30.0, 400)), *(-rng.random(400))]:
        y = float(y)
        m = y + 6755399441055744.0
        n = int(m - 6755399441055744.0)
        f = y - (m - 6755399441055744.0)
        assert abs(f) <= 0.5 and (int(np.float64(m).view(np.int64)) & 0xFFFFFFFF) == n & 0xFFFFFFFF
        e = steps[0]
        for c in steps[1:]:
            e = fma(e, f, c)
        got = math.ldexp(e, n)
        want = Decimal(2) ** Decimal(y)
        assert abs(Decimal(got) - want) <= Decimal(4e-14) * want, y
        assert y != 0.0 or got == 1.0
