"""Eviction against a plain form: which slots are kept, where their rows go in every layer, and
that nothing else changes.  Everything is compared bit for bit."""
import numpy as np
import pytest
import torch

import paper_2606_26631_amd as prcr
from attend_ref import HostCache, evict
from gpu_util import DEV, to_dev

pytestmark = pytest.mark.gpu


def make(dtype, D, B, NL, H, cap, block, seed):
    g = torch.Generator().manual_seed(seed)
    rng = np.random.default_rng(seed)
    table = None
    if block:
        per = -(-cap // block)
        table = rng.permutation(B * per + 3)[:B * per].astype(np.int32).reshape(B, per)
        shape, cap = (NL, B * per + 3, block, H, D), per * block
    else:
        shape = (B, NL, H, cap, D)
    k, v = (torch.randn(shape, generator=g).to(dtype) for _ in range(2))
    return k, v, table, cap, rng


def moved(x, table, kept):
    """The cache tensor with every kept row at its new slot."""
    new = x.clone()
    for b, slots in enumerate(kept):
        for layer in range(x.shape[1] if table is None else x.shape[0]):
            host = HostCache(x, x, table, layer)
            to, ok_to = host.at(b, np.arange(len(slots)))
            frm, ok_frm = host.at(b, np.array(slots, np.int64))
            both = ok_to & ok_frm
            if table is None:
                new[b, layer][:, to[both]] = x[b, layer][:, frm[both]]
            else:
                new[layer][to[0][both], to[1][both]] = x[layer][frm[0][both], frm[1][both]]
    return new


def run(k, v, table, lens, w, budget, first=0, last=0, err_want=0, **kw):
    cache = prcr.Cache(k.to(DEV), v.to(DEV), None if table is None else to_dev(table))
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    cap = w.shape[2]
    clamped = np.clip(lens, 0, cap)
    kept = evict(w, clamped, budget, first, last)
    wd = to_dev(w)
    new_len, got, new_w = prcr.evict(cache, to_dev(np.asarray(lens, np.int32)), wd, budget, first, last, err=err, **kw)
    torch.cuda.synchronize()
    assert int(err.item()) == err_want
    assert new_len.tolist() == [len(s) for s in kept]
    want = np.full((len(kept), budget), -1, np.int32)
    want_w = np.zeros_like(w)
    for b, s in enumerate(kept):
        want[b, :len(s)] = s
        want_w[b, :, :len(s)] = w[b][:, s]
    assert np.array_equal(got.cpu().numpy(), want)
    assert np.array_equal(new_w.cpu().numpy().view(np.int32), want_w.view(np.int32))
    assert np.array_equal(wd.cpu().numpy().view(np.int32), w.view(np.int32)), "the weights were changed"
    bits = lambda t: t.contiguous().view(torch.uint8)
    assert torch.equal(bits(cache.k.cpu()), bits(moved(k, table, kept)))
    assert torch.equal(bits(cache.v.cpu()), bits(moved(v, table, kept)))
    return kept


@pytest.mark.parametrize("block", [0, 16, 5, 1])
@pytest.mark.parametrize("dtype,D", [(torch.bfloat16, 128), (torch.bfloat16, 64), (torch.float32, 128), (torch.float32, 64)])
@pytest.mark.parametrize("budget,first,last", [(100, 0, 0), (100, 4, 30), (64, 64, 0), (37, 0, 37), (1, 0, 0), (900, 3, 9)])
def test_parity(budget, first, last, dtype, D, block):
    print(f"evict to {budget} ({first}, {last}) {dtype} D={D} block={block}", flush=True)
    k, v, table, cap, rng = make(dtype, D, 5, 2, 3, 300, block, budget + D + block)
    w = (rng.random((5, 3, cap)) ** 8).astype(np.float32)
    run(k, v, table, [300, 101, 100, 0, 1], w, budget, first, last)


@pytest.mark.parametrize("block", [0, 16])
def test_longer_than_a_round(block):
    print(f"long {block}", flush=True)
    k, v, table, cap, rng = make(torch.bfloat16, 64, 2, 1, 2, 5000, block, 9)
    w = rng.random((2, 2, cap)).astype(np.float32)
    run(k, v, table, [5000, 4097], w, 4000, 1, 1)
    run(k, v, table, [5000, 4097], w, 1100, 0, 1024)


def test_order_of_scores():
    """Equal scores go to the lowest slots; NaN ranks last; zeros of both signs are equal."""
    print("ties", flush=True)
    k, v, table, cap, rng = make(torch.bfloat16, 64, 6, 1, 1, 2600, 0, 3)
    w = np.zeros((6, 1, cap), np.float32)
    w[1] = rng.integers(0, 3, cap)
    w[2] = np.where(rng.random(cap) < 0.5, np.float32(0.0), np.float32(-0.0))
    w[3] = np.where(rng.random(cap) < 0.9, np.nan, -rng.random(cap)).astype(np.float32)
    w[4] = rng.standard_normal(cap).astype(np.float32)
    w[4, 0, 7], w[4, 0, 8], w[4, 0, 9] = np.inf, -np.inf, np.nan
    w[5] = rng.random(cap).astype(np.float32) * 1e-42        # (below the normal numbers)
    for budget in (500, 1300, 2599):
        run(k, v, table, [2600] * 6, w, budget)
        run(k, v, table, [2600] * 6, w, budget, 2, 400)


def test_heads_are_summed_in_double():
    """Heads whose float32 sum would be the same, or overflow."""
    print("sums", flush=True)
    k, v, table, cap, rng = make(torch.bfloat16, 64, 2, 1, 3, 40, 0, 4)
    w = np.ones((2, 3, cap), np.float32)
    w[0, 0], w[0, 1] = 2.0 ** 24, rng.integers(0, 2, cap)
    w[0, 2] = 2.0 ** -30 * rng.integers(0, 2, cap)
    w[1, 0], w[1, 1] = 3e38, 3e38
    w[1, 2] = -3e38 * rng.random(cap).astype(np.float32)
    run(k, v, table, [40, 40], w, 17)


def test_bad_blocks_and_lengths():
    print("bad blocks", flush=True)
    k, v, table, cap, rng = make(torch.bfloat16, 64, 2, 2, 2, 160, 16, 5)
    w = rng.random((2, 2, cap)).astype(np.float32)
    table[0, 2], table[1, 5] = -1, k.shape[1]
    run(k, v, table, [160, 150], w, 70, 0, 20, err_want=prcr.DERR_BLOCK)
    print("bad lengths", flush=True)
    k, v, table, cap, rng = make(torch.bfloat16, 64, 2, 1, 1, 50, 0, 6)
    w = rng.random((2, 1, cap)).astype(np.float32)
    run(k, v, table, [900, -3], w, 20, err_want=prcr.DERR_CAPACITY)


def test_lengths_in_place_and_given_outputs():
    print("in place", flush=True)
    k, v, table, cap, rng = make(torch.bfloat16, 128, 3, 1, 2, 90, 16, 7)
    w = rng.random((3, 2, cap)).astype(np.float32)
    lens = np.array([90, 20, 55], np.int32)
    kept = evict(w, lens, 30, 0, 0)
    cache = prcr.Cache(k.to(DEV), v.to(DEV), to_dev(table))
    n = to_dev(lens)
    ws = torch.full((prcr.evict_workspace_bytes(cache, 30),), 255, dtype=torch.uint8, device=DEV)
    out = torch.full((3, 30), 9, dtype=torch.int32, device=DEV)
    got = prcr.evict(cache, n, to_dev(w), 30, new_cache_len=n, kept=out, workspace=ws)
    torch.cuda.synchronize()
    assert got[0] is n and got[1] is out and n.tolist() == [30, 20, 30]
    assert out[2].tolist() == kept[2]


def test_key_only_memory_is_renamed():
    """A revisit after the eviction finds its values at their new slots, and skips a token whose
    value is gone."""
    print("key-only memory", flush=True)
    D, H, NL, M, cap = 64, 2, 2, 12, 120
    k, v, _, _, rng = make(torch.bfloat16, D, 2, NL, H, cap, 0, 8)
    w = rng.random((2, H, cap)).astype(np.float32)
    v_slot = np.stack([rng.permutation(100)[:M], rng.permutation(30)[:M]]).astype(np.int32)
    v_slot[0, 3], v_slot[0, 4] = -1, 110     # not slots of the sequence
    lens, budget = np.array([100, 30], np.int32), 40
    kept = evict(w, lens, budget, 2, 5)
    mem_k = torch.randn((2, M, NL, H, D), generator=torch.Generator().manual_seed(1)).bfloat16()
    coords = torch.zeros((2, M, 3), dtype=torch.int32, device=DEV)
    mem = prcr.Memory(mem_k.to(DEV), None, coords, to_dev(np.array([M, M], np.int32)), to_dev(v_slot))
    cache = prcr.Cache(k.to(DEV), v.to(DEV))
    new_len, _, _ = prcr.evict(cache, to_dev(lens), to_dev(w), budget, 2, 5, mem=mem)
    torch.cuda.synchronize()
    want = np.array([[kept[b].index(s) if s in kept[b] else -1 for s in v_slot[b]] for b in range(2)])
    assert np.array_equal(mem.v_slot.cpu().numpy(), want) and (want[0] < 0).sum() > 2 and (want[1] >= 0).all()
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    off = to_dev(np.array([0, M, 2 * M], np.int32))
    idx = to_dev(np.tile(np.arange(M, dtype=np.int32), 2))
    _, _, _, slots = prcr.revisit(prcr.Rope(D, (32, 0, 0), False, 1e4), mem, off, idx, to_dev(lens), cache, new_len, err=err)
    torch.cuda.synchronize()
    assert int(err.item()) == prcr.DERR_INDEX
    slots = slots.cpu().numpy().reshape(2, M)
    for b in range(2):
        for m in range(M):
            assert (slots[b, m] < 0) == (want[b, m] < 0)
            if want[b, m] >= 0:
                at = slots[b, m] - b * cap
                assert torch.equal(cache.v[b, :, :, at].cpu(), v[b, :, :, int(v_slot[b, m])])
    full = prcr.Memory(mem_k.to(DEV), mem_k.to(DEV), coords, mem.n_visual)
    prcr.evict(cache, new_len, to_dev(w), budget, mem=full)   # (has its own values: nothing to rename)
    torch.cuda.synchronize()


def test_captured_and_replayed():
    print("captured", flush=True)
    k, v, table, cap, rng = make(torch.bfloat16, 128, 2, 2, 2, 200, 16, 10)
    cache = prcr.Cache(k.to(DEV), v.to(DEV), to_dev(table))
    n, w = to_dev(np.array([200, 150], np.int32)), torch.zeros((2, 2, cap), device=DEV)
    ws = torch.empty(prcr.evict_workspace_bytes(cache, 60), dtype=torch.uint8, device=DEV)
    outs = (torch.zeros(2, dtype=torch.int32, device=DEV), torch.zeros((2, 60), dtype=torch.int32, device=DEV),
            torch.zeros_like(w))
    call = lambda: prcr.evict(cache, n, w, 60, 1, 5, new_cache_len=outs[0], kept=outs[1], new_weights=outs[2], workspace=ws)
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for i in range(4):
        wh = np.random.default_rng(i).random(w.shape).astype(np.float32)
        w.copy_(torch.from_numpy(wh))
        cache.k.copy_(k)
        cache.v.copy_(v)
        ws.fill_(255)
        g.replay()
        torch.cuda.synchronize()
        kept = evict(wh, [200, 150], 60, 1, 5)
        assert outs[1].tolist() == kept
        assert torch.equal(cache.k.cpu(), moved(k, table, kept)) and torch.equal(cache.v.cpu(), moved(v, table, kept))
