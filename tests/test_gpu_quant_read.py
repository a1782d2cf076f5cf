"""Reading the decoder cache in 8 bits back: every code, layouts, lengths from none to the capacity, rows behind
the length, bad data."""
import numpy as np
import pytest
import torch

import paper_2606_26631_amd as prcr
from gpu_util import DEV, to_dev
from quant_ref import CODES, TYPES, Store

pytestmark = pytest.mark.gpu


def expect(store, layer, b, n, dtype, name, skip=()):
    """code scale in float32, rounded once to dtype (a product and a rounding: exactly these bits)."""
    c, s = store.rows(name, b, np.arange(n))
    x = torch.from_numpy(c[:, layer].astype(np.float32)) * torch.from_numpy(s[:, layer])[..., None]
    return x.to(dtype).transpose(0, 1)


@pytest.mark.parametrize("block", [0, 16, 5, 1])
@pytest.mark.parametrize("kind", sorted(CODES))
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("H,lens", [(2, [70, 0, 1, 33]), (5, [17]), (1, [5, 64, 71])])
def test_read(H, lens, dtype, D, kind, block):
    print(f"read H={H} {lens} {dtype} D={D} {kind} block={block}", flush=True)
    B, NL, layer, dt = len(lens), 2, 1, TYPES[dtype]
    store = Store(CODES[kind], B, NL, H, D, 71, block, seed=2).fill(seed=D)
    cache, err = store.to(DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    k = torch.full((B, 1, H, 80, D), 7.0, dtype=dt, device=DEV)
    v = torch.full_like(k, 9.0)
    got = prcr.quant_read(cache, layer, to_dev(np.array(lens, np.int32)), dt, k=k, v=v, err=err)
    torch.cuda.synchronize()
    assert got[0] is k and got[1] is v and int(err.item()) == 0
    for name, t, fill in (("k", k, 7.0), ("v", v, 9.0)):
        for b, n in enumerate(lens):
            assert torch.equal(t[b, 0, :, :n].cpu(), expect(store, layer, b, n, dt, name)), (name, b)
            assert bool((t[b, 0, :, n:] == fill).all())
    a, _ = prcr.quant_read(cache, 0, to_dev(np.array(lens, np.int32)), dt)
    assert a.shape == (B, 1, H, store.cap, D)
    assert torch.equal(a[0, 0, :, :lens[0]].cpu(), expect(store, 0, 0, lens[0], dt, "k"))


@pytest.mark.parametrize("kind", sorted(CODES))
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_every_code(dtype, kind):
    """All 256 codes, at the smallest, an odd, a NaN and the largest scale."""
    print(f"every code {dtype} {kind}", flush=True)
    D = 128
    store = Store(CODES[kind], 1, 1, 2, D, 4)
    store.k = torch.arange(256, dtype=torch.uint8).view(1, 1, 2, 1, D).expand(1, 1, 2, 4, D).contiguous().view(CODES[kind])
    store.v = store.k.clone()
    store.k_scale[..., :] = torch.tensor([2.0 ** -126, 0.0123456, float("nan"), 3.4e38 / 448])
    store.v_scale.copy_(store.k_scale)
    k, v = prcr.quant_read(store.to(DEV), 0, to_dev(np.array([4], np.int32)), TYPES[dtype])
    for name, t in (("k", k), ("v", v)):
        want = expect(store, 0, 0, 4, TYPES[dtype], name)
        assert torch.equal(t[0, 0].cpu().isnan(), want.isnan())
        assert torch.equal(t[0, 0].cpu().nan_to_num(1), want.nan_to_num(1))


@pytest.mark.parametrize("block", [0, 16])
def test_bad_data(block):
    print(f"read bad data, block={block}", flush=True)
    B, H, D = 3, 2, 64
    store = Store(torch.int8, B, 1, H, D, 32, block).fill(seed=1)

    def run(lens, S):
        err = torch.zeros(1, dtype=torch.int32, device=DEV)
        k = torch.full((B, 1, H, S, D), 7.0, dtype=torch.bfloat16, device=DEV)
        v = torch.full_like(k, 7.0)
        prcr.quant_read(store.to(DEV), 0, to_dev(np.array(lens, np.int32)), torch.bfloat16, k=k, v=v, err=err)
        return k, int(err.item())

    for lens, S, n in (([33, 2 ** 31 - 1, -1], 40, [32, 32, 0]), ([20, 9, 3], 9, [9, 9, 3])):
        k, err = run(lens, S)
        assert err == prcr.DERR_CAPACITY
        for b in range(B):
            assert torch.equal(k[b, 0, :, :n[b]].cpu(), expect(store, 0, b, n[b], torch.bfloat16, "k"))
            assert bool((k[b, 0, :, n[b]:] == 7).all())
    if block:
        good = store.table.copy()
        store.table[1, 1], store.table[2, 0] = -5, store.k.shape[1]
        k, err = run([32, 32, 10], 32)
        assert err == prcr.DERR_BLOCK
        store.table = good
        assert torch.equal(k[0, 0].cpu(), expect(store, 0, 0, 32, torch.bfloat16, "k"))
        assert torch.equal(k[1, 0, :, :16].cpu(), expect(store, 0, 1, 16, torch.bfloat16, "k"))
        assert bool((k[1, 0, :, 16:] == 7).all()) and bool((k[2] == 7).all())
