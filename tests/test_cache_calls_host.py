"""Host parts of the calls around the cache: frequencies of rotary positions, and refusals that need no device."""
import ctypes as C
import math

import pytest


def close(got, want):
    return len(got) == len(want) and all(math.isclose(a, b, rel_tol=1e-13) for a, b in zip(got, want))


def _cfg(B, rot=128, scaling=0, base=10000.0, factor=1.0, trained=0, low=0.0, high=0.0, magnitude=1.0):
    return B.cas_rope_cfg(rot, scaling, base, factor, trained, low, high, magnitude)


def test_frequencies_of_every_scaling():
    from paper_2605_26558_amd import binding as B
    for rot in (2, 6, 64, 128, 256):
        plain = [500000.0 ** (-2.0 * i / rot) for i in range(rot // 2)]
        assert close(B.cas_rope_freqs(_cfg(B, rot, base=500000.0, factor=7.0)), plain)
        assert close(B.cas_rope_freqs(_cfg(B, rot, 1, 500000.0, 8.0)), [f / 8 for f in plain])
        if rot > 2:  # the slowest pair ends up as far as with squeezed positions, the fastest stays
            got = B.cas_rope_freqs(_cfg(B, rot, 2, 500000.0, 8.0))
            assert got[0] == 1.0 and math.isclose(got[-1], plain[-1] / 8, rel_tol=1e-12)
        got = B.cas_rope_freqs(_cfg(B, rot, 3, 500000.0, 8.0, 8192, 1.0, 32.0))
        for f, g in zip(plain, got):
            turns = 8192 * f / (2 * math.pi)
            assert f / 8 * (1 - 1e-12) <= g <= f * (1 + 1e-12)
            if turns >= 32:
                assert math.isclose(g, f, rel_tol=1e-13)
            if turns <= 1:
                assert math.isclose(g, f / 8, rel_tol=1e-13)


def test_refusals_without_a_device():
    from paper_2605_26558_amd import binding as B
    lib = B._lib()
    for bad in (dict(rot=0), dict(rot=5), dict(rot=258), dict(scaling=4), dict(base=0.0), dict(base=math.nan), dict(scaling=1, factor=0.5),
                dict(rot=2, scaling=2), dict(scaling=3, trained=0, high=1.0), dict(scaling=3, trained=9, low=1.0, high=1.0), dict(magnitude=0.0)):
        with pytest.raises(B.CasError) as e:
            B.cas_rope_freqs(_cfg(B, **bad))
        assert e.value.code == B.CAS_EINVAL, bad
    cfg, one = _cfg(B), (C.c_int32 * 1)(1)
    assert lib.cas_rope_freqs(C.byref(cfg), None) == B.CAS_EINVAL and lib.cas_rope_freqs(None, None) == B.CAS_EINVAL
    assert lib.cas_rope_table(None, C.byref(cfg), 0, 4, None) == B.CAS_EINVAL
    assert lib.cas_rope(None, None, 4, 64, 0, 0, None, 0, 1, 128, 1, None) == B.CAS_EINVAL
    assert lib.cas_attention_shared(None, None, 0, 1, one, 0, 1, None, one, 8, None, None, one, None) == B.CAS_EINVAL
    assert lib.cas_attention_weights(None, None, 0, 0, 1, None, 1, 8, None, None, 1, None, None, None, 0) == B.CAS_EINVAL
    assert lib.cas_kv_select(None, None, 1, 1, 1, 1, 0, 0, None, None, 0) == B.CAS_EINVAL
    assert lib.cas_kv_evict(None, None, 0, 1, 0, 0, None, 1) == B.CAS_EINVAL
    assert lib.cas_attention_shared_bytes(None, 1, one, 0, one, 8, one) == 0
    assert lib.cas_attention_weights_bytes(None, 0, 1, 8, 1) == 0


def test_buffer_accesses_are_checked_over_their_whole_distance():
    """Raw buffer accesses are held to the descriptor's length by their lane offset alone: nothing may be in the scalar offset."""
    import glob
    import os
    import re
    import paper_2605_26558_amd as P
    seen = 0
    for path in sorted(glob.glob(os.path.join(os.path.dirname(P.__file__), "csrc", "*"))):
        text = open(path, encoding="utf-8").read() if os.path.isfile(path) else ""
        for m in re.finditer(r"__builtin_amdgcn_raw_buffer_(load|store)_\w+\(", text):
            args, depth, at = [""], 0, m.end()
            while depth >= 0:
                c = text[at]
                depth += (c in "([{") - (c in ")]}")
                if c == "," and depth == 0:
                    args.append("")
                elif depth >= 0:
                    args[-1] += c
                at += 1
            seen += 1
            assert args[-2].strip() == "0", (os.path.basename(path), m.group(0) + ",".join(args))
    assert seen > 10


def test_a_magnitude_that_fp32_does_not_hold_is_refused():
    from paper_2605_26558_amd import binding as B
    for magnitude in (2.0 ** -126, 3.4028234663852886e38):   # the smallest normal and the largest number of the table
        assert len(B.cas_rope_freqs(_cfg(B, magnitude=magnitude))) == 64
    for magnitude in (1e-39, 2.0 ** -150, 3.5e38, 1e300):
        with pytest.raises(B.CasError) as e:
            B.cas_rope_freqs(_cfg(B, magnitude=magnitude))
        assert e.value.code == B.CAS_EINVAL, magnitude


@pytest.fixture
def wrappers(monkeypatch):
    """The binding with tensors that say they are on the GPU and a context that is none: a call whose arguments the wrapper
    takes comes back from the library as CAS_EINVAL, one that it does not take raises AssertionError."""
    import types
    import torch
    from paper_2605_26558_amd import binding as B

    class OnGpu(torch.Tensor):
        is_cuda = True

    def check(rc, what):
        if rc != B.CAS_OK:
            raise B.CasError(rc, what)

    ctx = types.SimpleNamespace(_torch=torch, h=None, _check=check)
    kv = types.SimpleNamespace(h=None, desc=types.SimpleNamespace(n_kv_heads=2, head_dim=128))
    monkeypatch.setattr(B, "cas_kv_len", lambda kv, seq: 10)
    return torch, B, ctx, kv, lambda *shape, dtype=torch.bfloat16: torch.zeros(*shape, dtype=dtype).as_subclass(OnGpu)


def _taken(B, call):
    with pytest.raises((B.CasError, AssertionError)) as e:
        call()
    return isinstance(e.value, B.CasError) and e.value.code == B.CAS_EINVAL


def test_wrappers_take_bf16_bits_and_no_other_two_byte_numbers(wrappers):
    torch, B, ctx, kv, t = wrappers
    table, bits = t(4, 64, 2, dtype=torch.float32), (torch.bfloat16, torch.int16, torch.uint16)
    for dtype in (*bits, torch.float32, torch.float16, torch.float64, torch.int32):
        x = t(3, 2, 128, dtype=dtype)
        assert _taken(B, lambda: B.cas_rope(ctx, table, [x])) == (dtype in bits or dtype == torch.float32), dtype
        y = t(3, 2, 128, dtype=dtype)
        assert _taken(B, lambda: B.cas_rope(ctx, table, [t(3, 2, 128)], outs=[y])) == (dtype in bits), dtype
        for i in range(4):
            a = [t(1, 4, 128), t(1, 2, 128), t(1, 2, 128), t(1, 4, 128)]
            a[i] = a[i].to(dtype).as_subclass(type(table))
            q, k, v, o = a
            assert _taken(B, lambda: B.cas_attention_shared(ctx, kv, 0, [0], 0, True, [q], [k], [v], outs=[o])) == (dtype in bits), (i, dtype)
            assert _taken(B, lambda: B.cas_attention_weights(ctx, kv, 0, 0, True, q, k, v, score_out=t(2, 11, dtype=torch.float32), out=o)) == (dtype in bits), (i, dtype)


def test_scores_of_one_kv_head_lie_anywhere(wrappers):
    """A single row has no next one, so its step does not matter; rows of several heads lie the same distance apart."""
    torch, B, ctx, kv, t = wrappers
    f = lambda *shape: t(*shape, dtype=torch.float32)  # noqa: E731
    for heads in (1, 2):
        kv.desc.n_kv_heads = heads
        q, k, v = t(1, 4, 128), t(1, heads, 128), t(1, heads, 128)
        forms = [f(heads, 11), f(heads, 40)[:, :11], f(40, heads, 20)[3, :, 5:16]] + [f(11).expand(1, 11)] * (heads == 1)
        for a in forms + [None]:
            for b in forms:
                want = heads == 1 or a is None or a.stride() == b.stride()
                assert _taken(B, lambda: B.cas_attention_weights(ctx, kv, 0, 0, True, q, k, v, a, score_out=b)) == want, (heads, a, b)
        assert not _taken(B, lambda: B.cas_attention_weights(ctx, kv, 0, 0, True, q, k, v, f(heads, 22)[:, ::2], score_out=f(heads, 11)))
        assert not _taken(B, lambda: B.cas_attention_weights(ctx, kv, 0, 0, True, q, k, v, f(heads, 10), score_out=f(heads, 11)))


def test_pools_of_a_cache_are_given_both_or_not_at_all(wrappers):
    torch, B, ctx, _, t = wrappers
    for pools in (dict(spec_pool=t(1 << 20)), dict(verif_pool=t(1 << 20))):
        with pytest.raises(AssertionError, match="both"):
            B.KVCache(ctx, 1, 2, 4, 1, 4, **pools)
