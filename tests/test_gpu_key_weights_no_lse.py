"""Rows whose log-sum-exp is -infinity give no weight to any key, whether they see live slots or
not and whatever their queries hold: the program masked them, their blocks were missing when they
attended, or all that they see scores -infinity.

The expected weights are those of the same call without such rows (attend_ref.key_weights, with a
log-sum-exp that leaves nothing and a clean query in their place)."""
import numpy as np
import pytest
import torch

import paper_2606_26631_amd as prcr
from attend_ref import attention, key_weights, spans
from gpu_util import DEV, to_dev
from test_gpu_chunk import Inputs
from test_gpu_key_weights import check

pytestmark = pytest.mark.gpu

# name: (dtype, D, H, G, rows, lengths, block, capacity).  The stretches of 128 or 256 keys that a
# row sees whole and those that it does not are summed by different code.
CASES = {
    "tokens": ("bf16", 128, 2, 4, [1, 1, 1], [700, 64, 300], 16, None),
    "turn": ("bf16", 128, 2, 4, [60, 3], [700, 400], 0, None),
    "turn_f32": ("f32", 64, 2, 2, [60, 3], [500, 400], 16, None),
    "f32": ("f32", 128, 1, 3, [50], [290], 0, None),
    "shared": ("bf16", 64, 1, 8, [300, 500], [900, 700], 0, None),
    "shared_f32": ("f32", 64, 1, 8, [300, 500], [300, 700], 24, None),
    "two_blocks": ("bf16", 128, 4, 4, [300, 310], [1100, 400], 0, 20000),
}


def silent_rows(x, rng):
    """Of each sequence the last row, a run of rows and some single ones; some of one head alone."""
    T, Hq = x.q.shape[:2]
    none = np.zeros((T, Hq), bool)
    for b, n in enumerate(x.ns):
        r0 = int(x.off[b])
        none[r0 + n - 1] = n > 1 or b == 0
        none[r0 + n // 3:r0 + n // 3 + n // 4] = True
        none[r0:r0 + n] |= rng.random((n, Hq)) < 0.1
    return none


@pytest.mark.parametrize("window", [None, 40])
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("name", sorted(CASES))
def test_masked_by_the_program(name, accumulate, window):
    dtype, D, H, G, ns, lens, block, cap = CASES[name]
    print(f"silent rows: {name}, accumulate={accumulate}, window={window}", flush=True)
    x = Inputs(dtype, D, H, G, ns, lens, block, seed=31, cap=cap)
    rng = np.random.default_rng(5)
    rows, B = spans(x.off, None, len(ns)), len(ns)
    lse = attention(x.rope, x.host(), x.q, x.pos, rows, x.lens, D ** -0.5, x.dtype)[1].astype(np.float32)
    none = silent_rows(x, rng)
    want, bound = key_weights(x.rope, x.host(), x.q, x.pos, rows, x.lens, D ** -0.5, x.dtype,
                              np.where(none, np.float32(1e30), lse), window)
    start = rng.random(want.shape).astype(np.float32)
    if accumulate:
        want = want + start.astype(np.float64)
        bound = bound + 2.0 ** -24 * (np.abs(want) + start)
    # Some of the silent rows' queries are not numbers either.
    bad = none & (rng.random(none.shape) < 0.3)
    x.q[torch.from_numpy(bad)] = float("nan")
    x.q[torch.from_numpy(none & ~bad & (rng.random(none.shape) < 0.3))] = 1e30
    lse[none] = -np.inf
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    got = prcr.key_weights(*x.args(x.cache()), to_dev(lse), window=window, err=err,
                           weights=to_dev(start) if accumulate else None, accumulate=accumulate)
    torch.cuda.synchronize()
    assert int(err.item()) == 0 and none.any() and np.isfinite(want).all()
    check(got, want, bound)


@pytest.mark.parametrize("dtype,D,n,past", [("bf16", 128, 40, 200), ("f32", 64, 3, 300), ("bf16", 64, 300, 40)])
def test_scores_of_minus_infinity(dtype, D, n, past):
    """Keys that score -infinity have no weight; a row that sees no others is like one that sees
    nothing: out 0, lse -infinity, no weight for any key."""
    print(f"scores of -infinity {dtype} {D} {n} {past}", flush=True)
    H, G = 2, 2
    x = Inputs(dtype, D, H, G, [n, n], [past + n, past + n], seed=4)
    x.pos[:] = 0                             # (unrotated)
    x.q = x.q.abs() + 0.5
    x.k[1, x.layer, :, :past + n // 2, 3] = -float("inf")     # sequence 1: the last rows see some others
    x.k[0, x.layer, 0, :10, 5] = -float("inf")
    cache = x.cache()
    out, lse = prcr.chunk_attention(*x.args(cache))
    w = prcr.key_weights(*x.args(cache), lse)
    torch.cuda.synchronize()
    out, lse, w = (t.float().cpu().numpy() for t in (out, lse, w))
    blind = n + n // 2                       # rows n .. blind - 1 see only such keys
    assert np.isneginf(lse[n:blind]).all() and not out[n:blind].any()
    assert np.isfinite(lse[:n]).all() and np.isfinite(lse[blind:2 * n]).all()
    assert np.isfinite(out[:2 * n]).all() and np.isfinite(w).all()
    assert not w[0, 0, :10].any() and not w[1, :, :past + n // 2].any()
    # each of the other rows gives its heads' sum of one; an lse is off by at most 1e-4
    assert np.allclose(w[0].sum(-1), n * G, rtol=1e-4) and np.allclose(w[1].sum(-1), (n - n // 2) * G, rtol=1e-4)


def test_block_mapped_after_the_attention():
    """A sequence whose blocks were outside the pool when it attended (lse -infinity), and are
    there when its keys are weighed."""
    print("block mapped later", flush=True)
    x = Inputs("bf16", 64, 2, 2, [20, 20], [90, 60], 16, seed=7)
    good = x.table.copy()
    x.table[1] = -1
    bad = x.cache()
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    out, lse = prcr.chunk_attention(*x.args(bad), err=err)
    x.table = good
    w = prcr.key_weights(*x.args(x.cache()), lse)
    torch.cuda.synchronize()
    assert int(err.item()) == prcr.DERR_BLOCK and bool(torch.isneginf(lse[20:40]).all())
    w = w.cpu().numpy()
    assert not w[1].any() and np.allclose(w[0].sum(-1), 40, rtol=1e-4)
