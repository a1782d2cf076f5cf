"""Caches in 8 bits of more than 2^32 bytes: what lies in their last blocks, or with their last sequence, is written,
attended to and read as in a small cache.  (The rest of the large tensors is left as it comes.)"""
import numpy as np
import pytest
import torch

import paper_2606_26631_amd as prcr
from gpu_util import DEV, to_dev
from quant_ref import Store, attention, check_attention
from test_gpu_quant_write import Revisit, Tokens, picks_of

pytestmark = pytest.mark.gpu

ROPE = (128, (24, 20, 20), True, 5e6)
H, D = 4, 128


def steps(cache, x, y, q, q_pos, lens):
    """The operators one after the other; what they return."""
    rope, err = prcr.Rope(*ROPE), torch.zeros(1, dtype=torch.int32, device=DEV)
    x.append(rope, cache, 0, err=err)
    new_len, slots = y.run(rope, cache, err=err)
    out = prcr.quant_decode_attention(rope, cache, 0, q, to_dev(q_pos), to_dev(lens), err=err)
    k, v = (torch.zeros(3, 1, H, int(max(lens)), D, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    prcr.quant_read(cache, 0, to_dev(lens), torch.bfloat16, k=k, v=v, err=err)
    torch.cuda.synchronize()
    assert int(err.item()) == 0
    return out, k, v, new_len, slots


def inputs():
    x = Tokens("bf16", D, H, 20, [20, 13, 7], [300, 500, 0], seed=1)
    y = Revisit("bf16", D, 1, H, 30, picks_of([5, 9, 3], 30, 2), [320, 513, 7], seed=2)
    lens = np.array([325, 522, 10], np.int32)
    q = torch.randn(3, H * 2, D, generator=torch.Generator().manual_seed(3)).bfloat16()
    return x, y, q, np.array([400, 600, 30], np.int32), lens


@pytest.mark.parametrize("block", [16, 24])
def test_last_blocks_of_a_large_pool(block):
    print(f"large pool of 8-bit rows, block={block}", flush=True)
    x, y, q, q_pos, lens = inputs()
    store = Store(torch.float8_e4m3fn, 3, 1, H, D, 528, block, seed=4).fill(seed=5)
    small = store.to(DEV)
    n, n_far = store.k.shape[1], 2 ** 32 // (block * H * D) + 300       # blocks of more than 4 GiB
    far = [torch.empty((1, n_far, block, H, D), dtype=torch.uint8, device=DEV).view(store.kind) for _ in range(2)]
    scales = [torch.empty((1, n_far, H, block), device=DEV) for _ in range(2)]
    for f, t in zip(far + scales, (store.k, store.v, store.k_scale, store.v_scale)):
        f[:, -n:] = t.to(DEV)
    cache = prcr.QuantCache(*far, *scales, to_dev(store.table + (n_far - n)))
    a, b = steps(cache, x, y, q.to(DEV), q_pos, lens), steps(small, x, y, q.to(DEV), q_pos, lens)
    for i, (s, t) in enumerate(zip(a[:3], b[:3])):
        assert torch.equal(s, t), i
    assert np.array_equal(a[4], b[4] + (n_far - n) * block)
    for f, t in zip(far + scales, (small.k, small.v, small.k_scale, small.v_scale)):
        assert torch.equal(f[:, -n:].contiguous().view(torch.uint8), t.view(torch.uint8))


def test_last_sequence_of_a_large_cache():
    print("large cache of 8-bit rows", flush=True)
    x, y, q, q_pos, lens = inputs()
    store = Store(torch.int8, 3, 1, H, D, 528).fill(seed=5)
    small = store.to(DEV)
    s_max = 2 ** 31 // (H * D) + 9                           # a sequence is more than 2 GiB
    far = [torch.empty((3, 1, H, s_max, D), dtype=torch.uint8, device=DEV).view(store.kind) for _ in range(2)]
    scales = [torch.empty((3, 1, H, s_max), device=DEV) for _ in range(2)]
    for f, t in zip(far + scales, (store.k, store.v, store.k_scale, store.v_scale)):
        f[:, :, :, :528] = t.to(DEV)
    a = steps(prcr.QuantCache(*far, *scales), x, y, q.to(DEV), q_pos, lens)
    b = steps(small, x, y, q.to(DEV), q_pos, lens)
    assert torch.equal(a[1], b[1]) and torch.equal(a[2], b[2])
    assert np.array_equal(a[4] % s_max, b[4] % 528) and np.array_equal(a[4] // s_max, b[4] // 528)
    for f, t in zip(far + scales, (small.k, small.v, small.k_scale, small.v_scale)):
        assert torch.equal(f[:, :, :, :528].contiguous().view(torch.uint8), t.view(torch.uint8))
    # (Another capacity splits the keys otherwise: compared with the 64-bit form.)
    want = attention(prcr.Rope(*ROPE), store.take(small), 0, q, q_pos, lens, D ** -0.5)
    check_attention(a[0], want)
    check_attention(b[0], want)


def test_length_near_the_end_of_a_long_sequence():
    """The last slots of a sequence of 2^24 + 5."""
    print("long sequence of 8-bit rows", flush=True)
    n = 2 ** 24 + 5
    x = Tokens("bf16", D, 1, 40, [40], [n - 40], seed=6)
    c = prcr.QuantCache(*(torch.zeros((1, 1, 1, n, D), dtype=torch.uint8, device=DEV).view(torch.int8) for _ in range(2)),
                        *(torch.full((1, 1, 1, n), 2.0 ** -126, device=DEV) for _ in range(2)))
    rope, err = prcr.Rope(*ROPE), torch.zeros(1, dtype=torch.int32, device=DEV)
    x.append(rope, c, 0, err=err)
    lens = to_dev(np.array([n], np.int32))
    q = torch.randn(1, 3, D, generator=torch.Generator().manual_seed(7)) * 30      # (the last keys have the weight)
    out = prcr.quant_decode_attention(rope, c, 0, q.to(DEV), to_dev(np.array([777], np.int32)), lens, err=err)
    torch.cuda.synchronize()
    assert int(err.item()) == 0
    store = Store(torch.int8, 1, 1, 1, D, 41)
    for name in ("k", "v"):
        for t in (name, name + "_scale"):
            getattr(store, t).view(torch.uint8)[:] = getattr(c, t)[:, :, :, n - 41:].cpu().contiguous().view(torch.uint8)
    want, bound = attention(rope, store, 0, q, np.array([777]), [41], D ** -0.5)
    # The other n - 41 keys score 0: their weight beside the 41's, as a bound of what they take away.
    k, ks = store.rows("k", 0, np.arange(41))
    v, vs = store.rows("v", 0, np.arange(41))
    from quant_ref import turned
    s = (k[:, 0, 0] * ks[:, 0, 0, None]) @ turned(rope, q.double().numpy(), np.array([[777] * 3]))[0].T * D ** -0.5
    share = (n - 41) / np.exp(s).sum(0)                      # [3]
    want = want / (1 + share)[None, :, None]
    e = np.exp(s - s.max(0))
    p = e / e.sum(0) / (1 + share)
    err = ((D + 8) * (np.abs(k[:, 0, 0] * ks[:, 0, 0, None]) @ np.abs(turned(rope, q.double().numpy(), np.array([[777] * 3]))[0]).T) *
           D ** -0.5).max(0) * 2.0 ** -24
    # Sums of n weights: by tiles, waves and chunks, far fewer roundings in a row than n, of which 2^16 are allowed.
    bound = ((2 * err + 2 * (2 ** 16 + 64) * 2.0 ** -24)[:, None] * (p.T @ np.abs(v[:, 0, 0] * vs[:, 0, 0, None])) + 1e-30)[None]
    check_attention(out, (want, bound))
