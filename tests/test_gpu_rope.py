"""Rotary positions through the C ABI: the table against angles in 64 bits for every scaling, the rotation against complex
products in 64 bits over layouts, partial heads, types, strides and orders of positions, gradients against differences,
and the refusals."""
import math

import numpy as np
import pytest

import synth

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2605_26558_amd import binding as B
    return torch, B, B.Context()


def _freqs(rot, scaling, base, factor, trained, low, high):
    out = []
    for i in range(rot // 2):
        b = base * factor ** (rot / (rot - 2)) if scaling == 2 else base
        f = b ** (-2.0 * i / rot)
        if scaling == 1:
            f /= factor
        if scaling == 3:
            g = min(1.0, max(0.0, (trained * f / (2 * math.pi) - low) / (high - low)))
            f = g * f + (1 - g) * f / factor
        out.append(f)
    return np.array(out)


@pytest.mark.parametrize("rot,scaling,pos0,n,factor,mag", [
    (128, 0, 0, 1000, 1.0, 1.0), (128, 3, 0, 4097, 16.0, 1.2772588722239782), (2, 0, 5, 33, 1.0, 1.0), (6, 1, 100, 257, 4.0, 1.0),
    (256, 2, 0, 70, 8.0, 1.0), (64, 3, (1 << 24) - 300, 300, 40.0, 0.5), (80, 2, 1 << 20, 1, 3.5, 1.0), (4, 2, 0, 1, 1.0, 2.0),
    (126, 0, 99991, 513, 1.0, 1.0),
])
def test_table_matches_angles_in_64_bits(env, rot, scaling, pos0, n, factor, mag):
    torch, B, ctx = env
    base, trained, low, high = 10000.0, 4096, 1.0, 32.0
    print(f"case rot={rot} scaling={scaling} pos0={pos0} n={n}", flush=True)
    cfg = B.cas_rope_cfg(rot, scaling, base, factor, trained, low, high, mag)
    f = _freqs(rot, scaling, base, factor, trained, low, high)
    # powers and products of some operations in 64 bits on either side
    np.testing.assert_allclose(B.cas_rope_freqs(cfg), f, rtol=1e-13)
    out = torch.full((n + 1, rot // 2, 2), 7.0, dtype=torch.float32, device="cuda")
    B.cas_rope_table(ctx, cfg, pos0, n, out=out[:n])
    torch.cuda.synchronize()
    a = np.arange(pos0, pos0 + n, dtype=np.float64)[:, None] * f
    ref = mag * np.stack([np.cos(a), np.sin(a)], -1)
    got = out.cpu().numpy()
    # the documented 2e-7 * magnitude: the reduced angle as fp32 (2^-25), the series (two units of 2^-24), the magnitude's
    # and the product's roundings (2^-24 each); and the frequencies of the two sides, equal to some units of 2^-53
    assert np.abs(got[:n] - ref).max() <= 2e-7 * mag + (pos0 + n) * 1e-14
    assert (got[n] == 7.0).all()


def test_table_is_the_models(env):
    """rot = 128, plain: the table that the model passes take (computed on the host until now), to the last bits of fp32."""
    torch, B, ctx = env
    t = B.cas_rope_table(ctx, B.cas_rope_cfg(128, B.CAS_ROPE_PLAIN, 500000.0, 1.0, 0, 0.0, 0.0, 1.0), 0, 2000)
    ref = synth.rope_table(2000, 128, 500000.0)
    assert t.shape == ref.shape
    assert np.abs(t.cpu().numpy() - ref).max() <= 2e-7


def _ref(x, table, pos, rot, inter, transposed):
    """x: float64 [tok, heads, dim] as rounded to bf16; complex products with the fp32 table."""
    z = table[pos, :, 0] + 1j * table[pos, :, 1] * (-1 if transposed else 1)
    y = x.copy()
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if inter else (x[..., :rot // 2], x[..., rot // 2:rot])
    w = (a + 1j * b) * z[:, None, :]
    if inter:
        y[..., 0:rot:2], y[..., 1:rot:2] = w.real, w.imag
    else:
        y[..., :rot // 2], y[..., rot // 2:rot] = w.real, w.imag
    big = np.zeros_like(x)  # |x_a cos| + |x_b sin| of every value
    c, s = np.abs(z.real)[:, None, :], np.abs(z.imag)[:, None, :]
    pa, pb = np.abs(a) * c + np.abs(b) * s, np.abs(b) * c + np.abs(a) * s
    if inter:
        big[..., 0:rot:2], big[..., 1:rot:2] = pa, pb
    else:
        big[..., :rot // 2], big[..., rot // 2:rot] = pa, pb
    return y, big


CASES = [  # tokens, heads of the parts, dim, rot, interleaved, fp32, pad
    (1, (32, 8, 8), 128, 128, False, True, 0), (5, (4, 2, 2), 128, 128, False, False, 0), (7, (3, 1, 1), 256, 64, True, False, 40),
    (33, (2, 2, 2), 80, 20, False, True, 3), (9, (5,), 96, 96, True, True, 0), (2, (7, 7), 2, 2, True, False, 1),
    (300, (8, 2, 2, 1), 64, 32, False, False, 8), (1500, (2, 1), 128, 16, True, True, 4), (64, (1,), 6, 4, False, False, 0),
    (3, (1, 1), 256, 256, False, True, 0), (17, (40,), 128, 66, False, False, 16), (11, (0, 3), 128, 128, False, False, 0),
    (1, (3, 2), 255, 254, True, False, 1),
]


@pytest.mark.parametrize("tok,heads,dim,rot,inter,fp32,pad", CASES)
@pytest.mark.parametrize("transposed", [False, True])
def test_rotation_matches_complex_products(env, tok, heads, dim, rot, inter, fp32, pad, transposed):
    torch, B, ctx = env
    print(f"case {tok=} {heads=} {dim=} {rot=} {inter=} {fp32=} {pad=} {transposed=}", flush=True)
    n_pos = 700
    table = B.cas_rope_table(ctx, B.cas_rope_cfg(rot, 0, 10000.0, 1.0, 0, 0.0, 0.0, 1.0), 0, n_pos)
    rng = np.random.Generator(np.random.Philox(3))
    pos = rng.integers(0, n_pos, tok).astype(np.int32)   # any order, the same more than once
    width = sum(heads) * dim
    buf = torch.from_numpy(rng.standard_normal((tok, width + pad)).astype(np.float32)).cuda()
    x = buf if fp32 else buf.bfloat16()
    xs, at = [], 0
    for h in heads:
        xs.append(x[:, at:at + h * dim].unflatten(1, (h, dim)))
        at += h * dim
    turn = [i < 2 for i in range(len(heads))]
    ys = B.cas_rope(ctx, table, xs, pos=torch.from_numpy(pos).cuda(), layout=int(inter), transposed=transposed, turn=turn)
    torch.cuda.synchronize()
    tab = table.cpu().numpy().astype(np.float64)
    for i, (xi, yi) in enumerate(zip(xs, ys)):
        xr = xi.bfloat16().double().cpu().numpy()
        got = yi.view(torch.bfloat16).double().cpu().numpy()
        if not turn[i]:
            np.testing.assert_array_equal(got, xr)
            continue
        ref, big = _ref(xr, tab, pos, rot, inter, transposed)
        # two products and a sum in fp32 (2^-24 each, relative to what they add), the result rounded to bf16 once (2^-8)
        err, tol = np.abs(got - ref), 2.0 ** -8 * np.abs(ref) + 4 * 2.0 ** -24 * big
        assert (err <= tol).all(), float((err / np.maximum(tol, 1e-300)).max())


def test_rotation_is_that_of_the_model_passes(env):
    """The model's split: bf16 of the projection, then a0 c - a1 s and a1 c + a0 s in fp32, bf16 (the oracle's rope)."""
    torch, B, ctx = env
    from oracle import cassandra_oracle as O
    table = synth.rope_table(50, 128, 500000.0)
    x = synth.normal_bf16((6, 3, 128), 1.0, seed=4)
    y = B.cas_rope(ctx, torch.from_numpy(table).cuda(), [torch.from_numpy(x.view(np.int16)).cuda()], pos0=9)[0]
    ref = np.stack([O.rope(x[t], 9 + t, table) for t in range(6)])
    got = O.bf16_to_f64(y.cpu().numpy().view(np.uint16))
    want = O.bf16_to_f64(ref)
    # the oracle forms the value in 64 bits: both are the exact value rounded, up to 2^-23 of the pair's size before that
    pair = np.hypot(O.bf16_to_f64(x)[..., :64], O.bf16_to_f64(x)[..., 64:])
    tol = 2.0 ** -7 * np.maximum(np.abs(got), np.abs(want)) + 2.0 ** -22 * np.concatenate([pair, pair], -1)
    assert (np.abs(got - want) <= tol).all()
    assert (got == want).mean() > 0.99


def test_in_place_padding_and_positions_outside(env):
    torch, B, ctx = env
    table = B.cas_rope_table(ctx, B.cas_rope_cfg(64, 0, 10000.0, 1.0, 0, 0.0, 0.0, 1.0), 0, 100)
    x = torch.randn(6, 4, 128, device="cuda").bfloat16()
    pos = torch.tensor([3, -1, 99, 100, 2**31 - 1, 0], dtype=torch.int32, device="cuda")
    apart = B.cas_rope(ctx, table, [x], pos=pos, outs=[torch.full_like(x, 5.0)])[0]
    inplace = x.clone()
    B.cas_rope(ctx, table, [inplace], pos=pos, outs=[inplace])
    torch.cuda.synchronize()
    for t in (1, 3, 4):       # padding: nothing of it is written
        assert (apart[t] == 5.0).all() and torch.equal(inplace[t], x[t])
    for t in (0, 2, 5):
        assert torch.equal(apart[t], inplace[t])
    assert torch.equal(inplace[5], x[5])                    # position 0 turns nothing
    rows = B.cas_rope(ctx, table, [x], pos0=97, outs=[torch.full_like(x, 5.0)])[0]   # 97, 98, 99, then behind the table
    torch.cuda.synchronize()
    assert torch.equal(rows[2], B.cas_rope(ctx, table, [x[2:3]], pos0=99)[0][0]) and (rows[3:] == 5.0).all()
    assert B.cas_rope(ctx, table, [x[:0]])[0].shape == (0, 4, 128)


@pytest.mark.parametrize("pad", [0, 1])
def test_tokens_far_apart(env, pad):
    """Two tokens more than 2^32 bytes apart, on the aligned and on the other path."""
    torch, B, ctx = env
    table = B.cas_rope_table(ctx, B.cas_rope_cfg(128, 0, 10000.0, 1.0, 0, 0.0, 0.0, 1.0), 0, 20)
    ld = (1 << 31) + 8 + pad
    far = torch.empty(ld + 256, dtype=torch.bfloat16, device="cuda")
    x = far.as_strided((2, 2, 128), (ld, 128, 1))
    x.copy_(torch.randn(2, 2, 128, device="cuda"))
    near = x.contiguous()
    want = B.cas_rope(ctx, table, [near], pos0=5)[0]
    B.cas_rope(ctx, table, [x], pos0=5, outs=[x])
    torch.cuda.synchronize()
    assert torch.equal(x.contiguous(), want)
    del far, x
    torch.cuda.empty_cache()


def test_infinities_and_nan_stay_in_their_pair(env):
    torch, B, ctx = env
    table = B.cas_rope_table(ctx, B.cas_rope_cfg(128, 0, 10000.0, 1.0, 0, 0.0, 0.0, 1.0), 0, 20)
    x = torch.randn(4, 2, 128, device="cuda")
    y0 = B.cas_rope(ctx, table, [x], pos0=7)[0].view(torch.bfloat16)
    x[1, 0, 5], x[2, 1, 70] = math.inf, math.nan
    y1 = B.cas_rope(ctx, table, [x], pos0=7)[0].view(torch.bfloat16)
    torch.cuda.synchronize()
    changed = {(1, 0, 5), (1, 0, 69), (2, 1, 70), (2, 1, 6)}
    same = (y0 == y1).cpu().numpy()
    assert {tuple(map(int, i)) for i in np.argwhere(~same)} <= changed
    assert not torch.isfinite(y1[1, 0, 5]) and torch.isnan(y1[2, 1, 70])


@pytest.mark.parametrize("inter", [0, 1])
def test_gradient_is_the_transposed_rotation(env, inter):
    """<g, R x> = <R^T g, x>, and R^T g against differences of a loss, both in what bf16 leaves."""
    torch, B, ctx = env
    table = B.cas_rope_table(ctx, B.cas_rope_cfg(32, 3, 10000.0, 4.0, 64, 1.0, 32.0, 1.25), 0, 300)
    g = torch.Generator(device="cuda").manual_seed(1)
    x, dy = (torch.randn(8, 3, 64, device="cuda", generator=g).bfloat16() for _ in range(2))
    pos = torch.tensor([0, 1, 5, 299, 17, 17, 100, 250], dtype=torch.int32, device="cuda")
    f = lambda v, t=False: B.cas_rope(ctx, table, [v], pos=pos, layout=inter, transposed=t)[0].double()  # noqa: E731
    dx = f(dy, True)
    a, b = (dy.double() * f(x)).sum(), (dx * x.double()).sum()
    size = (dy.double().abs() * f(x).abs()).sum() + (dx.abs() * x.double().abs()).sum()
    assert abs(a - b) <= 2.0 ** -8 * size
    # differences along channels: the loss <dy, R x> is linear, so steps of 1 in x give the gradient itself
    for tok, h, ch in ((3, 1, 0), (6, 2, 31), (7, 0, 16), (1, 0, 50)):
        e = torch.zeros_like(x)
        e[tok, h, ch] = 1.0
        d = (dy.double() * f(e)).sum()
        tol = 2.0 ** -8 * ((dy.double() * f(e)).abs().sum() + dx[tok, h, ch].abs())
        assert abs(d - dx[tok, h, ch]) <= tol


def test_captured_and_on_another_stream(env):
    torch, B, _ = env
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        ctx = B.Context()
        cfg = B.cas_rope_cfg(128, 0, 10000.0, 1.0, 0, 0.0, 0.0, 1.0)
        table = torch.zeros(64, 64, 2, device="cuda")
        x = torch.randn(4, 2, 128, device="cuda")
        y = torch.zeros(4, 2, 128, dtype=torch.int16, device="cuda")
        pos = torch.tensor([1, 2, 3, 60], dtype=torch.int32, device="cuda")
        B.cas_rope_table(ctx, cfg, 0, 64, out=table)
        B.cas_rope(ctx, table, [x], pos=pos, outs=[y])
    s.synchronize()
    want = y.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        B.cas_rope_table(ctx, cfg, 0, 64, out=table)
        B.cas_rope(ctx, table, [x], pos=pos, outs=[y])
    for i in range(3):
        y.zero_(); table.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want), i
        pos.copy_(pos)            # the program's own work between replays
    x.mul_(2.0)
    torch.cuda.synchronize()
    graph.replay()
    torch.cuda.synchronize()
    ref = B.cas_rope(B.Context(), table, [x], pos=pos)[0]
    torch.cuda.synchronize()
    assert torch.equal(y, ref)


def test_refusals(env):
    torch, B, ctx = env
    ok = dict(rot=64, scaling=0, base=10000.0, factor=1.0, trained=0, low=0.0, high=0.0, magnitude=1.0)
    for change in (dict(rot=0), dict(rot=3), dict(rot=258), dict(scaling=4), dict(scaling=-1), dict(base=0.5), dict(base=math.inf),
                   dict(base=math.nan), dict(scaling=1, factor=0.5), dict(scaling=1, factor=math.nan), dict(scaling=2, rot=2),
                   dict(scaling=3, trained=0, high=1.0), dict(scaling=3, trained=8, low=2.0, high=2.0), dict(magnitude=0.0),
                   dict(scaling=3, trained=8, low=math.nan, high=2.0), dict(magnitude=math.inf)):
        cfg = B.cas_rope_cfg(*{**ok, **change}.values())
        with pytest.raises(B.CasError) as e:
            B.cas_rope_freqs(cfg)
        assert e.value.code == B.CAS_EINVAL, change
    cfg = B.cas_rope_cfg(*ok.values())
    for pos0, n in ((-1, 4), ((1 << 24) - 3, 4)):
        with pytest.raises(B.CasError):
            B.cas_rope_table(ctx, cfg, pos0, n)
    table = B.cas_rope_table(ctx, cfg, 0, 4)
    lib, x = B._lib(), torch.zeros(4, 2, 128, dtype=torch.bfloat16, device="cuda")

    def call(n_pos=4, rot=64, layout=0, n_tok=4, dim=128, parts=1, ldx=256, ldy=256, heads=2, fp32=0, xp=x.data_ptr(),
             yp=x.data_ptr(), tab=table.data_ptr(), pos0=0):
        p = (B.cas_rope_part * 5)(*[B.cas_rope_part(xp, yp, ldx, ldy, heads, fp32, 1, 0)] * 5)
        return lib.cas_rope(ctx.h, tab, n_pos, rot, layout, 0, None, pos0, n_tok, dim, parts, p)

    assert call() == B.CAS_OK
    for bad in (dict(n_pos=-1), dict(rot=0), dict(rot=63), dict(rot=130), dict(layout=2), dict(n_tok=-1), dict(parts=0), dict(parts=5),
                dict(ldx=255), dict(ldy=255), dict(heads=-1), dict(fp32=1), dict(xp=None), dict(yp=None), dict(tab=None),
                dict(tab=table.data_ptr() + 8), dict(xp=x.data_ptr() + 1), dict(ldx=264), dict(pos0=2**31 - 4)):
        assert call(**bad) == B.CAS_EINVAL, bad
    assert call(dim=264, ldx=528, ldy=528) == B.CAS_ENOTSUP
    assert call(n_tok=0, xp=None, yp=None, tab=None) == B.CAS_OK
    assert call(heads=0, xp=None, yp=None, tab=None) == B.CAS_OK


@pytest.mark.parametrize("rot,scaling,pos0,n,factor,mag", [
    (128, 0, 0, 20000, 1.0, 1.0), (128, 3, 0, 4097, 16.0, 1.2772588722239782), (64, 3, (1 << 24) - 300, 300, 40.0, 0.5),
    (128, 0, (1 << 24) - 5000, 5000, 1.0, 1.0), (256, 1, (1 << 24) - 2000, 2000, 3.0, 0.1), (80, 2, 1 << 20, 3000, 3.5, 1.7),
])
def test_table_within_its_bound_at_every_position(env, rot, scaling, pos0, n, factor, mag):
    """The documented 2e-7 * magnitude and nothing beside it, against the frequencies that cas_rope_freqs gives."""
    torch, B, ctx = env
    print(f"case {rot=} {scaling=} {pos0=} {n=}", flush=True)
    assert np.finfo(np.longdouble).nmant >= 63
    cfg = B.cas_rope_cfg(rot, scaling, 10000.0, factor, 4096, 1.0, 32.0, mag)
    f = np.array(B.cas_rope_freqs(cfg)).astype(np.longdouble)
    a = np.arange(pos0, pos0 + n).astype(np.longdouble)[:, None] * f   # 24 and 53 bits into 64: off by 2^24 * 2^-64
    ref = np.stack([np.cos(a), np.sin(a)], -1) * np.longdouble(mag)
    got = B.cas_rope_table(ctx, cfg, pos0, n).cpu().numpy()
    # relative to the magnitude: the reduced angle as fp32 2.6e-8, quarter turns per position in 64 bits 0.6e-8, the series 2.5e-8 and
    # its last rounding 3e-8 (at pi / 4, where the value is 0.71; 3e-8 alone at 1), magnitude and product 2^-24 of the value each
    assert float(np.abs(got - ref).max()) <= 2e-7 * mag


@pytest.mark.parametrize("mag", [2.0 ** -126, 3.4028234663852886e38])
def test_magnitudes_at_the_ends_of_fp32(env, mag):
    torch, B, ctx = env
    cfg = B.cas_rope_cfg(128, 0, 10000.0, 1.0, 0, 0.0, 0.0, mag)
    a = np.arange(500, 1500, dtype=np.float64)[:, None] * np.array(B.cas_rope_freqs(cfg))
    got = B.cas_rope_table(ctx, cfg, 500, 1000).cpu().numpy()
    # the documented bound; below the normal numbers a product is off by 2^-150, 2^-24 of the smallest normal one
    assert np.abs(got / mag - np.stack([np.cos(a), np.sin(a)], -1)).max() <= 2e-7


def test_as_many_tokens_as_a_launch_has(env):
    torch, B, ctx = env
    table = B.cas_rope_table(ctx, B.cas_rope_cfg(2, 0, 10000.0, 1.0, 0, 0.0, 0.0, 1.0), 0, 8)
    n = 1 << 24
    pos = torch.arange(n, dtype=torch.int32, device="cuda") & 7
    x = torch.randn(n, 1, 2, device="cuda").bfloat16()
    y = torch.full_like(x, 5.0)
    with pytest.raises(B.CasError) as e:
        B.cas_rope(ctx, table, [x], pos=pos, outs=[y])
    assert e.value.code == B.CAS_ENOTSUP
    torch.cuda.synchronize()
    assert bool((y == 5.0).all())
    B.cas_rope(ctx, table, [x[1:]], pos=pos[1:], outs=[y[1:]])
    torch.cuda.synchronize()
    for at in (1, n // 2 + 3, n - 9):   # the same eight positions in calls of their own
        want = B.cas_rope(ctx, table, [x[at:at + 9].contiguous()], pos=pos[at:at + 9].contiguous())[0]
        assert torch.equal(y[at:at + 9], want)
    assert bool((y[0] == 5.0).all()) and bool((y[1:, 0, 0].float() != 5.0).any())
