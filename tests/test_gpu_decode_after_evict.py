"""Decoding in a cache that was cut back: the decode step after an eviction, and after tokens that were
appended to the cut cache, against a plain 64-bit attention over the rows that are to be there, taken
from the cache as it was before.

decode_attention keeps its query in float32, as attend_ref's float32 form does; its tolerance is that
of its own tests, 5e-5 of the largest attended value (+ 1e-6).  A step that gave zeros, that went on
in the cache of before, or that missed what was appended is seen to be beyond it."""
import numpy as np
import pytest
import torch

import paper_2606_26631_amd as prcr
from attend_ref import HostCache, attention, evict
from gpu_util import DEV, to_dev
from test_gpu_chunk import Inputs

pytestmark = pytest.mark.gpu


def plain(x, k, v, lens, q, pos, layer):
    """One row per sequence over slots 0 .. lens[b] - 1 of the given tensors."""
    B = len(lens)
    return attention(x.rope, HostCache(k, v, x.table, layer), q.cpu(), pos, [(b, 1) for b in range(B)], lens,
                     x.D ** -0.5, torch.float32)[0]


def kept_rows(x, t, kept):
    """The tensor with every kept row at its new slot."""
    new = t.clone()
    for b, slots in enumerate(kept):
        host = HostCache(t, t, x.table, 0)
        to, frm = host.at(b, np.arange(len(slots)))[0], host.at(b, np.array(slots))[0]
        for layer in range(t.shape[1 if x.table is None else 0]):
            if x.table is None:
                new[b, layer][:, to] = t[b, layer][:, frm]
            else:
                new[layer][to[0], to[1]] = t[layer][frm[0], frm[1]]
    return new


@pytest.mark.parametrize("block", [0, 16, 5])
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 64)])
def test_decode_goes_on(dtype, D, block):
    print(f"decode after eviction {dtype} {D} {block}", flush=True)
    H, G, NL, B, budget = 2, 4, 2, 3, 90
    x = Inputs(dtype, D, H, G, [20, 20, 20], [240, 130, 60], block, seed=D + block, cap=256, layers=NL)
    x.k *= 1.5                               # (weights that differ, so that it matters which rows are read)
    cache = x.cache()
    args = x.args(cache)
    cap = 256 if x.table is None else x.table.shape[1] * block
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    weights = torch.zeros((B, H, cap), device=DEV)
    for layer in range(NL):
        call = (x.rope, cache, layer) + args[3:]
        lse = prcr.chunk_attention(*call, err=err)[1]
        prcr.key_weights(*call, lse, window=8, weights=weights, accumulate=True, err=err)
    kept = evict(weights.cpu().numpy(), x.lens, budget, 4, 16)
    lens, got, _ = prcr.evict(cache, args[6], weights, budget, 4, 16, err=err)
    torch.cuda.synchronize()
    cut = [len(s) for s in kept]
    assert lens.tolist() == cut == [90, 90, 60] and got[0].tolist() == kept[0]
    k, v = kept_rows(x, x.k, kept), kept_rows(x, x.v, kept)
    g = torch.Generator().manual_seed(7)
    rnd = lambda *s: torch.randn(s, generator=g).to(x.dtype)
    # The cut cache, then two more tokens in it, one after the other.
    for turn in range(3):
        p = np.full((B, 3), 5000 + turn, np.int32)
        if turn > 0:
            mem = prcr.Memory(torch.zeros((B, 1, NL, H, D), dtype=x.dtype, device=DEV),
                              torch.zeros((B, 1, NL, H, D), dtype=x.dtype, device=DEV),
                              torch.zeros((B, 1, 3), dtype=torch.int32, device=DEV), to_dev(np.zeros(B, np.int32)))
            new_k, new_v = rnd(NL, B, 1, H, D), rnd(NL, B, 1, H, D) * 3
            for layer in range(NL):
                prcr.prefill_capture(x.rope, mem, layer, new_k[layer].to(DEV), new_v[layer].to(DEV), to_dev(p[:, None]),
                                     to_dev(np.ones(B, np.int32)), to_dev(np.full((B, 1), -1, np.int32)), cache, lens, err=err)
            lens = lens + 1
            before = k.clone(), v.clone(), list(cut)
            # where the new rows are to be (their keys' rotation has tests of its own)
            host = HostCache(cache.k, cache.v, x.table, 0)
            for b in range(B):
                at = host.at(b, [cut[b]])[0]
                for layer in range(NL):
                    if x.table is None:
                        k[b, layer, :, cut[b]] = host.k[b, layer, :, cut[b]]
                        v[b, layer, :, cut[b]] = new_v[layer, b, 0]
                    else:
                        k[layer, at[0][0], at[1][0]] = host.k[layer, at[0][0], at[1][0]]
                        v[layer, at[0][0], at[1][0]] = new_v[layer, b, 0]
            cut = [n + 1 for n in cut]
        else:
            before = x.k, x.v, list(x.lens)
        for layer in range(NL):
            q = rnd(B, H * G, D)
            step = prcr.decode_attention(x.rope, cache, layer, q.to(DEV), to_dev(p[:, 0]), lens, err=err)
            torch.cuda.synchronize()
            out = step.cpu().numpy().astype(np.float64)
            want, old = plain(x, k, v, cut, q, p, layer), plain(x, *before, q, p, layer)
            vmax = float(v.float().abs().max())
            bound = 5e-5 * vmax + 1e-6
            assert np.abs(out - want).max() <= bound
            # what would be wrong is far beyond it, for every sequence that was cut (or appended to)
            for b in range(B):
                assert np.abs(want[b]).max() > 100 * bound
                if turn > 0 or len(kept[b]) < x.lens[b]:
                    assert np.abs(want[b] - old[b]).max() > 20 * bound
    assert int(err.item()) == 0
