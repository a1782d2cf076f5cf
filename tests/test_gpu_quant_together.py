"""The cache in 8 bits as a program uses it, with the operators that were there: prompts are written and their visual
rows remembered, layers are read back for the prompt's attention and its keys' weights, visual tokens are revisited,
tokens decoded.  Every attention is checked against a plain 64-bit form on the cache as it is then."""
import numpy as np
import pytest
import torch

import paper_2606_26631_amd as prcr
from attend_ref import HostCache, attention as chunk_form, key_weights
from gpu_util import DEV, to_dev
from quant_ref import CODES, Store, attention, check_attention, check_rows, turned
from test_gpu_chunk import check as check_chunk
from test_gpu_key_weights import check as check_weights

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", sorted(CODES))
@pytest.mark.parametrize("block", [0, 16])
def test_prompt_revisit_decode(block, kind):
    print(f"together block={block} {kind}", flush=True)
    D, H, G, NL, B, M, S = 128, 2, 4, 2, 2, 64, 120
    Hq, dt = H * G, torch.bfloat16
    rope = prcr.Rope(D, (24, 20, 20), True, 5e6)
    g = torch.Generator().manual_seed(1)
    rnd = lambda *s: torch.randn(s, generator=g).to(dt).to(DEV)
    rng = np.random.default_rng(2)
    store = Store(CODES[kind], B, NL, H, D, 256, block, seed=3)
    cache = store.to(DEV)
    host = lambda: store.take(cache)
    mem = prcr.Memory(torch.zeros((B, M, NL, H, D), dtype=dt, device=DEV), torch.zeros((B, M, NL, H, D), dtype=dt, device=DEV),
                      torch.zeros((B, M, 3), dtype=torch.int32, device=DEV), to_dev(np.array([M, M], np.int32)))
    n_tok = np.array([S, 93], np.int32)
    pos = np.repeat(np.arange(S, dtype=np.int32)[None, :, None], B, 0).repeat(3, 2)
    vis = np.arange(10, 10 + M)
    pos[:, vis] = 10 + np.stack([np.zeros(M), np.arange(M) // 8, np.arange(M) % 8], 1)
    mem.coords.copy_(to_dev(np.ascontiguousarray(pos[:, vis])))
    vis_rows = to_dev(np.repeat(vis[None].astype(np.int32), B, 0))
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    lens, start = to_dev(n_tok), to_dev(np.zeros(B, np.int32))
    off, q_len = to_dev(np.arange(B + 1, dtype=np.int32) * S), to_dev(n_tok)
    rows, flat = [(b * S, int(n_tok[b])) for b in range(B)], pos.reshape(B * S, 3)
    for layer in range(NL):
        k, v = rnd(B, S, H, D), rnd(B, S, H, D)
        prcr.quant_append(rope, cache, layer, k, v, to_dev(pos), lens, start, err=err)
        prcr.store_raw(mem, layer, k, v, vis_rows, err=err)
        # The prompt's attention and its last rows' weights, over the layer read back.
        back = prcr.Cache(*prcr.quant_read(cache, layer, lens, dt, err=err))
        q = rnd(B * S, Hq, D)
        out = torch.full((B * S, Hq, D), 7.0, dtype=dt, device=DEV)
        lse = torch.full((B * S, Hq), 7.0, device=DEV)
        prcr.chunk_attention(rope, back, 0, q, off, to_dev(flat), lens, q_len=q_len, out=out, lse=lse, err=err)
        w = prcr.key_weights(rope, back, 0, q, off, to_dev(flat), lens, lse, q_len=q_len, window=20, err=err)
        torch.cuda.synchronize()
        s = host()
        for b in range(B):
            slots = np.arange(int(n_tok[b]))
            c, sc = s.rows("k", b, slots)
            check_rows(c[:, layer], sc[:, layer], turned(rope, k[b, slots].double().cpu().numpy(), pos[b, slots]), dt, s.kind)
            for name, t in (("k", back.k), ("v", back.v)):
                c, sc = s.rows(name, b, slots)
                want = (torch.from_numpy(c[:, layer]).float() * torch.from_numpy(sc[:, layer])[..., None]).to(dt)
                assert torch.equal(t[b, 0, :, :len(slots)].cpu(), want.transpose(0, 1))
        plain = HostCache(back.k, back.v, None, 0)
        check_chunk(out, lse, chunk_form(rope, plain, q, flat, rows, n_tok, D ** -0.5, dt))
        want, bound = key_weights(rope, plain, q, flat, rows, n_tok, D ** -0.5, dt, lse.cpu().numpy(), 20)
        check_weights(w, want, bound)
    assert int(err.item()) == 0

    # A revisit of 16 and 9 visual tokens, then two decoded tokens.
    picks = [np.sort(rng.choice(M, n, replace=False)).astype(np.int32) for n in (16, 9)]
    s_off, s_idx = to_dev(np.array([0, 16, 25], np.int32)), to_dev(np.concatenate(picks))
    new_pos, next_pos = prcr.reassign_coords(mem, s_off, s_idx, to_dev(n_tok - 1), "pcr", 2, err=err)
    before = host()
    lens, slots = prcr.quant_rebind_inject(rope, mem, s_off, s_idx, new_pos, cache, lens, err=err)
    torch.cuda.synchronize()
    s = host()
    assert lens.tolist() == [136, 102] and int(err.item()) == 0
    for b in range(B):
        at = n_tok[b] + np.arange(len(picks[b]))
        y = turned(rope, mem.k[b, picks[b]].double().cpu().numpy(), new_pos[s_off[b]:s_off[b + 1]].cpu().numpy())
        c, sc = s.rows("k", b, at)
        check_rows(c, sc, y, dt, s.kind)
        c, sc = s.rows("v", b, at)
        # (a value is quantised as it was when it was appended)
        old, old_scale = before.rows("v", b, vis[picks[b]])
        assert np.array_equal(c, old) and np.array_equal(sc, old_scale)
    for step in range(2):
        p = (next_pos + step).cpu().numpy().astype(np.int32)
        for layer in range(NL):
            prcr.quant_append(rope, cache, layer, rnd(B, 1, H, D), rnd(B, 1, H, D), to_dev(np.repeat(p[:, None, None], 3, 2)),
                              to_dev(np.ones(B, np.int32)), lens + step, err=err)
            q = rnd(B, Hq, D)
            out = prcr.quant_decode_attention(rope, cache, layer, q, to_dev(p), lens + step + 1, err=err)
            torch.cuda.synchronize()
            check_attention(out, attention(rope, host(), layer, q.cpu(), p, (lens + step + 1).tolist(), D ** -0.5))
            # Near the decode step over the same layer read back in float32.
            back = prcr.Cache(*prcr.quant_read(cache, layer, lens + step + 1, torch.float32, err=err))
            other = prcr.decode_attention(rope, back, 0, q.float(), to_dev(p), lens + step + 1, err=err)
            torch.cuda.synchronize()
            check_attention(other, attention(rope, host(), layer, q.cpu(), p, (lens + step + 1).tolist(), D ** -0.5))
    assert int(err.item()) == 0
