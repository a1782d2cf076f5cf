"""Caches of more than 2^32 bytes: what lies in their last blocks, or with their last sequence, is
attended to, weighed and moved as in a small cache.  (The rest of the large tensors is
left as it comes: nothing but a sequence's own slots may matter.)"""
import numpy as np
import pytest
import torch

import paper_2606_26631_amd as prcr
from attend_ref import key_weights, spans
from gpu_util import DEV, to_dev
from test_gpu_attend_many_rows import expect
from test_gpu_chunk import Inputs, check, run
from test_gpu_key_weights import check as check_weights

pytestmark = pytest.mark.gpu


def all_of(x, cache, budget=100):
    """Everything that a run of the operators gives: attention, weights, eviction, and the slots then."""
    args = (x.rope, cache, x.layer) + x.args(None)[3:]
    T = int(x.off[-1])
    out, lse = prcr.chunk_attention(*args)
    w = prcr.key_weights(*args, lse)
    lens, kept, new = prcr.evict(cache, args[6], w, budget, 2, 5)
    torch.cuda.synchronize()
    n = int(x.lens.max())
    return out[:T], lse[:T], w[:, :, :n].contiguous(), lens, kept, new[:, :, :n].contiguous()


def same(a, b):
    for i, (s, t) in enumerate(zip(a, b)):
        assert torch.equal(s.contiguous().view(torch.uint8), t.contiguous().view(torch.uint8)), i


@pytest.mark.parametrize("ns", [[5, 40], [400, 700]])
def test_last_blocks_of_a_large_pool(ns):
    print(f"large pool, rows {ns}", flush=True)
    H, G, D, block = 2, 4, 128, 16
    x = Inputs("bf16", D, H, G, ns, [300, 750], block, seed=1, cap=768, layers=2)
    small = x.cache()
    n_far = 2 ** 32 // (block * H * D * 2) + 300             # blocks of more than 4 GiB, in each layer
    far = [torch.empty((2, n_far, block, H, D), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    n = x.k.shape[1]
    for f, t in zip(far, (x.k, x.v)):
        f[:, -n:] = t.to(DEV)
    cache = prcr.Cache(far[0], far[1], to_dev(x.table + (n_far - n)))
    same(all_of(x, cache), all_of(x, small))
    for f, t in zip(far, (small.k, small.v)):
        assert torch.equal(f[:, -n:].contiguous().view(torch.int16), t.view(torch.int16))


@pytest.mark.parametrize("ns", [[5, 40, 7], [400, 700, 300]])
def test_last_sequence_of_a_large_cache(ns):
    print(f"large cache, rows {ns}", flush=True)
    H, G, D = 2, 4, 128
    x = Inputs("bf16", D, H, G, ns, [300, 750, 720], seed=2, cap=768, layers=1)
    small = x.cache()
    s_max = 2 ** 31 // (H * D * 2) + 9                       # a sequence is more than 2 GiB
    far = [torch.empty((3, 1, H, s_max, D), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    for f, t in zip(far, (x.k, x.v)):
        f[:, :, :, :768] = t.to(DEV)
    cache = prcr.Cache(*far)
    # (Another capacity splits keys and rows otherwise: attention and weights are compared with the
    # 64-bit form, and eviction is given the same weights.)
    args = (x.rope, cache, 0) + x.args(None)[3:]
    out, lse, _ = run(x, cache)
    check(out, lse, expect(x))
    wa = prcr.key_weights(*args, lse)
    torch.cuda.synchronize()
    want = key_weights(x.rope, x.host(), x.q, x.pos, spans(x.off, None, 3), x.lens, D ** -0.5, x.dtype, lse.cpu().numpy())
    check_weights(wa[:, :, :768], *want)
    assert not wa[:, :, 768:].any()
    wb = wa[:, :, :768].contiguous()
    ea, eb = prcr.evict(cache, args[6], wa, 100, 2, 5), prcr.evict(small, args[6], wb, 100, 2, 5)
    torch.cuda.synchronize()
    same(ea[:2] + (ea[2][:, :, :768],), eb)
    for f, t in zip(far, (small.k, small.v)):
        assert torch.equal(f[:, :, :, :768].contiguous().view(torch.int16), t.view(torch.int16))
