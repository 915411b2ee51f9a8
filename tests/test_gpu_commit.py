"""cas_commit of models of many layers: one launch for all of them, in the form that the number of vectors and the places ask for."""
import numpy as np
import pytest

import synth

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2605_26558_amd import binding as B
    return torch, B, B.Context(workspace=torch.empty(32 << 20, dtype=torch.uint8, device="cuda"))


def _model(torch, B, ctx, layers, n_kv, mode, keep, t):
    """A small model that has the same weights in all layers, its in-flight keys and values any finite numbers."""
    shape = synth.LlamaShape("many", 256, layers, n_kv, n_kv, 128, 512, 300)
    one = synth.LlamaShape("one", 256, 1, n_kv, n_kv, 128, 512, 300)
    w = synth.model_weights(one, seed=1)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a).view(np.int16)).cuda()  # noqa: E731
    L = {n: B.cas_encode_weight(ctx, dev(w["layers"][0][n]), 600, 4) for n in ("wqkv", "wo", "wgu", "wd")}
    L["g_attn"], L["g_ffn"] = dev(w["layers"][0]["g_attn"]), dev(w["layers"][0]["g_ffn"])
    head = B.cas_encode_weight(ctx, dev(w["lm_head"]), 600, 4)
    rope = torch.from_numpy(synth.rope_table(128, 128, shape.rope_theta)).cuda()
    m = B.Model(ctx, shape, [L] * layers, head, dev(w["embed"]), dev(w["g_final"]), rope, 32)
    g = torch.Generator(device="cuda").manual_seed(2)
    act = m.act.view(torch.int16)
    act.copy_(torch.randint(0x3C00, 0x4080, act.shape, generator=g, device="cuda", dtype=torch.int16))
    act[torch.rand(act.shape, generator=g, device="cuda") < 0.5] |= -32768
    kv = B.KVCache(ctx, layers, n_kv, n_pages=3, max_seqs=1, max_pages_per_seq=3, keep_permille=keep, trunc_bits=t, exp_mode=mode,
                   page_table=torch.tensor([[2, 0, 1]], dtype=torch.int32))
    return m, kv


def _rows(torch, kv, start, n):
    """Per pool, the bytes of positions start .. start + n - 1 of the only sequence, in all layers, heads, and both of K and V."""
    d, mx = kv.desc, kv.desc.fmt.exp_mode != 0
    out = []
    for pool, size, widths in ((kv.spec_pool, d.tile_spec_bytes, [4, 1, d.sw] if mx else [4, d.sw]), (kv.verif_pool, d.tile_verif_bytes, [d.lw, d.pw])):
        mask = torch.zeros(pool.shape, dtype=torch.bool, device="cuda")
        tiles = mask[:d.n_layers * d.n_pages * 2 * d.n_kv_heads * size].view(d.n_layers, d.n_pages, 2 * d.n_kv_heads, size)
        for i, page in enumerate(kv.page_table[0].tolist()):
            first, end, at = max(start - 64 * i, 0), min(start + n - 64 * i, 64), 0
            for w in widths:
                if first < end:
                    tiles[:, page, :, at + 4 * w * first:at + 4 * w * end] = True
                at += 64 * 4 * w
        out.append(mask)
    return out


@pytest.mark.parametrize("layers,n_kv,mode,keep,t", [(40, 8, 0, 600, 4), (126, 8, 0, 600, 4), (126, 8, 2, 600, 4), (48, 32, 0, 700, 3), (48, 32, 2, 333, 1), (48, 32, 2, 8, 3), (126, 8, 2, 1000, 4)])
def test_a_commit_is_the_first_tokens_of_a_longer_one(env, layers, n_kv, mode, keep, t):
    """The words of a position do not depend on how many are committed with it, nor do a commit's words lie anywhere else: every
    commit over what 32 tokens left changes nothing, and over other words only its own rows."""
    torch, B, ctx = env
    m, kv = _model(torch, B, ctx, layers, n_kv, mode, keep, t)
    for start in (0, 2, 13, 50):
        def commit(n):
            B.cas_kv_set_len(kv, 0, start)
            B.cas_commit(ctx, m, kv, 0, n - 1)
            assert B.cas_kv_len(kv, 0) == start + n
        kv.spec_pool.zero_()
        kv.verif_pool.zero_()
        commit(32)
        whole = kv.spec_pool.clone(), kv.verif_pool.clone()
        read = lambda n: [B.cas_kv_read(ctx, kv, layer, 0, 0, n, True) for layer in (0, layers // 2, layers - 1)]  # noqa: E731
        want = read(start + 32)
        # a value eight binary places and more below its block's largest is 0 under a shared exponent, so not all are other than 0
        assert not torch.equal(want[0][0][start:], want[1][0][start:]) and bool((want[2][1][start:] != 0).any(2).all())
        for n in (1, 2, 3, 4, 5, 7, 8, 9, 12, 15, 16, 17, 20, 31):
            commit(n)
            assert torch.equal(kv.spec_pool, whole[0]) and torch.equal(kv.verif_pool, whole[1]), (start, n)
        for n in (1, 4, 9, 12, 16, 17, 31):
            kv.spec_pool.zero_()
            kv.verif_pool.zero_()
            commit(n)
            for got, ref, rows in zip((kv.spec_pool, kv.verif_pool), whole, _rows(torch, kv, start, n)):
                assert torch.equal(got, torch.where(rows, ref, 0)), (start, n)
