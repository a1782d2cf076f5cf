"""The operators as a program uses them, together with the ones that were there: a prompt is
captured and attended, its keys are weighed, tokens are decoded and a visual selection is
revisited, the cache is cut back, and decoding goes on; every attention is checked against a plain
64-bit form on the cache as it is then."""
import numpy as np
import pytest
import torch

import paper_2606_26631_amd as prcr
from attend_ref import HostCache, attention, evict, key_weights
from gpu_util import DEV, to_dev
from test_gpu_chunk import check as check_chunk
from test_gpu_key_weights import check as check_weights

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("paged", [False, True])
def test_prompt_weights_revisit_eviction_decode(paged):
    print(f"together, paged={paged}", flush=True)
    D, H, G, NL, B, M = 128, 2, 4, 2, 2, 64
    Hq, S, cap, dt = H * G, 120, 256, torch.bfloat16
    rope = prcr.Rope(D, (24, 20, 20), True, 5e6)
    g = torch.Generator().manual_seed(1)
    rnd = lambda *s: torch.randn(s, generator=g).to(dt).to(DEV)
    rng = np.random.default_rng(2)
    n_tok = np.array([120, 93], np.int32)
    table = rng.permutation(B * 16).astype(np.int32).reshape(B, 16) if paged else None
    shape = (NL, B * 16, 16, H, D) if paged else (B, NL, H, cap, D)
    cache = prcr.Cache(torch.zeros(shape, dtype=dt, device=DEV), torch.zeros(shape, dtype=dt, device=DEV),
                       to_dev(table) if paged else None)
    mem = prcr.Memory(torch.zeros((B, M, NL, H, D), dtype=dt, device=DEV), torch.zeros((B, M, NL, H, D), dtype=dt, device=DEV),
                      torch.zeros((B, M, 3), dtype=torch.int32, device=DEV), to_dev(np.array([M, M], np.int32)))
    pos = np.zeros((B, S, 3), np.int32)
    vis = np.full((B, S), -1, np.int32)
    for b in range(B):
        pos[b] = np.arange(S)[:, None]
        pos[b, 10:10 + M] = 10 + np.stack([np.zeros(M), np.arange(M) // 8, np.arange(M) % 8], 1)
        vis[b, 10:10 + M] = np.arange(M)
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    host = lambda layer: HostCache(cache.k, cache.v, table, layer)
    off, q_len = to_dev(np.arange(B + 1, dtype=np.int32) * S), to_dev(n_tok)
    lens, start = to_dev(n_tok), to_dev(np.zeros(B, np.int32))
    rows = [(b * S, int(n_tok[b])) for b in range(B)]
    weights = torch.zeros((B, H, cap), device=DEV)
    total, bound = np.zeros((B, H, cap)), np.full((B, H, cap), 1e-6)
    flat = pos.reshape(B * S, 3)
    for layer in range(NL):
        prcr.prefill_capture(rope, mem, layer, rnd(B, S, H, D), rnd(B, S, H, D), to_dev(pos), lens, to_dev(vis), cache, start, err=err)
        q = rnd(B * S, Hq, D)
        out = torch.full((B * S, Hq, D), 7.0, dtype=dt, device=DEV)
        lse = torch.full((B * S, Hq), 7.0, device=DEV)
        prcr.chunk_attention(rope, cache, layer, q, off, to_dev(flat), lens, q_len=q_len, out=out, lse=lse, err=err)
        prcr.key_weights(rope, cache, layer, q, off, to_dev(flat), lens, lse, q_len=q_len, window=20, weights=weights,
                         accumulate=True, err=err)
        torch.cuda.synchronize()
        check_chunk(out, lse, attention(rope, host(layer), q, flat, rows, n_tok, D ** -0.5, dt))
        w, e = key_weights(rope, host(layer), q, flat, rows, n_tok, D ** -0.5, dt, lse.cpu().numpy(), 20)
        total, bound = total + w, bound + e
    check_weights(weights, total, bound + 2.0 ** -23 * total)
    assert int(err.item()) == 0

    # A revisit of 16 visual tokens appends to the cache; then two tokens at once attend to all.
    sel = np.sort(np.stack([rng.choice(M, 16, replace=False) for _ in range(B)]), 1).astype(np.int32)
    _, next_pos, lens, _ = prcr.revisit(rope, mem, to_dev(np.array([0, 16, 32], np.int32)), to_dev(sel.reshape(-1)),
                                        to_dev(n_tok - 1), cache, lens, err=err)
    t_off = to_dev(np.array([0, 2, 4], np.int32))
    t_pos = (next_pos.cpu().numpy()[:, None, None] + np.arange(2)[None, :, None] + np.zeros((1, 1, 3), np.int64)).astype(np.int32)
    lens = lens + 2
    grown = lens.cpu().numpy()
    none = to_dev(np.full((B, 2), -1, np.int32))
    for layer in range(NL):
        prcr.prefill_capture(rope, mem, layer, rnd(B, 2, H, D), rnd(B, 2, H, D), to_dev(t_pos), to_dev(np.array([2, 2], np.int32)),
                             none, cache, lens - 2, err=err)
        q = rnd(4, Hq, D)
        out, lse = prcr.chunk_attention(rope, cache, layer, q, t_off, to_dev(t_pos.reshape(4, 3)), lens, err=err)
        torch.cuda.synchronize()
        check_chunk(out, lse, attention(rope, host(layer), q, t_pos.reshape(4, 3), [(0, 2), (2, 2)], grown, D ** -0.5, dt))
        prcr.key_weights(rope, cache, layer, q, t_off, to_dev(t_pos.reshape(4, 3)), lens, lse, weights=weights,
                         accumulate=True, err=err)

    # Cut back to 80 slots, and one more token: by itself, and by the decode step.
    torch.cuda.synchronize()
    kept = evict(weights.cpu().numpy(), grown, 80, 4, 10)
    before = [host(layer) for layer in range(NL)]
    lens, got, weights = prcr.evict(cache, lens, weights, 80, 4, 10, mem=mem, err=err)
    torch.cuda.synchronize()
    assert int(err.item()) == 0 and got.tolist() == kept and lens.tolist() == [80, 80]
    q = rnd(B, Hq, D)
    p1 = t_pos[:, -1] + 1
    for layer in range(NL):
        for b in range(B):
            old = before[layer].rows(before[layer].v, b, int(grown[b]))[0]
            assert np.array_equal(host(layer).rows(cache.v.cpu(), b, 80)[0], old[kept[b]])
        one = to_dev(np.arange(B + 1, dtype=np.int32))
        out, lse = prcr.chunk_attention(rope, cache, layer, q, one, to_dev(p1), lens, err=err)
        step = prcr.decode_attention(rope, cache, layer, q, to_dev(p1[:, 0]), lens, err=err)
        torch.cuda.synchronize()
        want = attention(rope, host(layer), q, p1, [(0, 1), (1, 1)], [80, 80], D ** -0.5, dt)
        check_chunk(out, lse, want)
        # the decode step keeps its query in float32: it differs by the query's rounding, half a step
        # of bf16 (2^-8) in each of 128 products
        mag = 2.0 ** -8 * float(q.float().abs().max() * before[layer].k.float().abs().max()) * 128 * D ** -0.5
        assert float((out.float() - step).abs().max()) <= min(2 * mag, 1.0) * float(cache.v.float().abs().max())
    assert int(err.item()) == 0
