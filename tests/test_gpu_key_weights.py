"""The keys' weights against a plain 64-bit form, whose lse (rounded to float32) the calls are
given; tolerances are element by element (attend_ref.key_weights)."""
import numpy as np
import pytest
import torch

import paper_2606_26631_amd as prcr
from attend_ref import attention, key_weights, spans
from gpu_util import DEV, to_dev
from test_gpu_chunk import SHAPES, Inputs

pytestmark = pytest.mark.gpu


def run(x, window=None, start=None, q_len=None, scale=None, lse=None, accumulate=None, **kw):
    """(weights, expected, bound, err); start: weights that are there before (accumulated to)."""
    B = len(x.ns)
    sc = x.D ** -0.5 if scale is None else scale
    rows = spans(x.off, q_len, B)
    if lse is None:
        lse = attention(x.rope, x.host(), x.q, x.pos, rows, x.lens, sc, x.dtype)[1].astype(np.float32)
    want, bound = key_weights(x.rope, x.host(), x.q, x.pos, rows, x.lens, sc, x.dtype, lse, window)
    cache = x.cache()
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    weights = None
    if start is not None:
        weights = to_dev(start)
        want = want + start.astype(np.float64)
        bound = bound + 2.0 ** -24 * (np.abs(want) + np.abs(start))
    got = prcr.key_weights(*x.args(cache), to_dev(lse), window=window, weights=weights, err=err, scale=scale,
                           q_len=None if q_len is None else to_dev(q_len),
                           accumulate=start is not None if accumulate is None else accumulate, **kw)
    torch.cuda.synchronize()
    assert weights is None or got is weights
    return got, want, bound, int(err.item())


def check(got, want, bound):
    got = got.cpu().numpy().astype(np.float64)
    assert np.array_equal(np.isfinite(got), np.isfinite(want))
    fine = np.isfinite(want)
    d = np.abs(np.where(fine, got - np.where(fine, want, 0), 0)) - np.where(fine, bound, 0)
    assert d.max() <= 0, (np.unravel_index(d.argmax(), d.shape), d.max())


@pytest.mark.parametrize("block", [0, 16, 5, 128])
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("shape", sorted(SHAPES))
def test_parity(shape, dtype, D, block):
    H, G, ns, lens = SHAPES[shape]
    x = Inputs(dtype, D, H, G, ns, lens, block, seed=len(shape) + D + block)
    print(f"weights {shape} {dtype} D={D} block={block}", flush=True)
    for window in (None, 1, 33):
        got, want, bound, err = run(x, window)
        assert err == 0
        check(got, want, bound)
    start = np.random.default_rng(1).random(want.shape).astype(np.float32)
    got, want, bound, err = run(x, start=start)
    check(got, want, bound)
    for b, n in enumerate(x.lens):           # slots from the length on are left as they were
        assert np.array_equal(got[b, :, n:].cpu().numpy(), start[b, :, n:])


@pytest.mark.parametrize("dtype,block", [("bf16", 0), ("bf16", 16), ("f32", 0), ("f32", 24)])
def test_many_rows(dtype, block):
    """Rows enough for several workgroups to share a stretch of keys."""
    x = Inputs(dtype, 64, 1, 8, [300, 500], [300, 700], block, seed=5)
    print(f"many rows {dtype} {block}", flush=True)
    T, Hq = x.q.shape[0], 8
    plain = T * Hq * 64 * (2 if dtype == "bf16" else 4)
    assert prcr.key_weights_workspace_bytes(x.cache(), T, Hq) > plain + 255
    got, want, bound, err = run(x)
    assert err == 0
    check(got, want, bound)
    start = np.random.default_rng(2).random(want.shape).astype(np.float32)
    got, want, bound, err = run(x, start=start)
    check(got, want, bound)


def test_padded_rows_and_scale():
    n = np.array([9, 4, 0, 1], np.int32)
    x = Inputs("bf16", 128, 2, 2, [9] * 4, [40, 4, 9, 1], 16, seed=3)
    print("padded", flush=True)
    got, want, bound, err = run(x, q_len=n, scale=-0.15, window=3)
    assert err == 0
    check(got, want, bound)


def test_weights_of_a_row_sum_to_its_heads():
    x = Inputs("bf16", 128, 2, 4, [50, 1], [300, 64], 16, seed=21)
    cache = x.cache()
    print("with the attention's own lse", flush=True)
    out, lse = prcr.chunk_attention(*x.args(cache))
    w = prcr.key_weights(*x.args(cache), lse)
    torch.cuda.synchronize()
    # each row's weights sum to one; an lse is off by at most 1e-4 here
    assert torch.allclose(w.sum(-1), torch.tensor([[200.0] * 2, [4.0] * 2], device=DEV), rtol=1e-4)


def test_one_row_with_nan():
    """A NaN query: NaN for the keys it sees, and no others."""
    x = Inputs("bf16", 64, 1, 2, [40], [100], seed=22)
    x.q[10, 1, 3] = float("nan")             # sees slots 0 .. 70
    print("NaN row", flush=True)
    got, want, bound, err = run(x)
    g = got.cpu().numpy()[0, 0]
    assert np.isnan(g[:71]).all() and np.isfinite(g[71:]).all()
    check(got, want, bound)


def test_bad_data():
    x = Inputs("bf16", 64, 2, 2, [30, 30], [80, 100], 16, seed=13)
    x.table[0, 1], x.table[1, 0], x.table[1, -1] = -1, x.k.shape[1], -7
    print("bad blocks", flush=True)
    got, want, bound, err = run(x)
    assert err == prcr.DERR_BLOCK
    check(got, want, bound)
    x = Inputs("bf16", 64, 1, 8, [400], [400], 16, seed=13, cap=400)
    x.table[0, 3] = 999
    assert prcr.key_weights_workspace_bytes(x.cache(), x.q.shape[0], 8) > x.q.numel() * 2 + 255
    got, want, bound, err = run(x)
    assert err == prcr.DERR_BLOCK
    check(got, want, bound)
    x = Inputs("bf16", 64, 1, 2, [4, 6, 5], [20, 30, 40], seed=14, cap=50)
    good = x.off
    lse = attention(x.rope, x.host(), x.q, x.pos, spans(good, None, 3), x.lens, 0.125, x.dtype)[1].astype(np.float32)
    print("bad offsets", flush=True)
    for off in ([-5, 4, 10, 15], [0, 4, 10, 9000], [9, 8, 7, 6]):
        x.off = np.array(off, np.int32)
        cache = x.cache()
        for window in (None, 2):
            err = torch.zeros(1, dtype=torch.int32, device=DEV)
            w = prcr.key_weights(*x.args(cache), to_dev(lse), window=window, err=err)
            torch.cuda.synchronize()
            assert int(err.item()) == prcr.DERR_OFFSETS and not w.isnan().any()


def test_no_rows():
    x = Inputs("bf16", 64, 1, 2, [0, 0], [3, 4], extra=0, seed=1)
    print("no rows", flush=True)
    got, want, bound, err = run(x)
    assert not got.any()
    start = np.ones(want.shape, np.float32)
    got, _, _, _ = run(x, start=start)
    assert bool((got == 1).all())


def test_captured_and_replayed():
    x = Inputs("bf16", 128, 2, 4, [300, 200], [700, 300], 16, seed=15)
    cache = x.cache()
    args = list(x.args(cache))
    lse = prcr.chunk_attention(*args)[1]
    ws = torch.empty(prcr.key_weights_workspace_bytes(cache, x.q.shape[0], 8), dtype=torch.uint8, device=DEV)
    w = torch.zeros((2, 2, x.table.shape[1] * 16), device=DEV)
    call = lambda: prcr.key_weights(*args, lse, weights=w, workspace=ws)
    call()
    torch.cuda.synchronize()
    print("captured", flush=True)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for i in range(4):
        args[3].copy_(torch.randn(x.q.shape, generator=torch.Generator().manual_seed(i)).bfloat16())
        lse.copy_(prcr.chunk_attention(*args)[1])
        ws.fill_(255)
        w.fill_(5.0)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(w, prcr.key_weights(*args, lse))
