"""Calls without any row: the keys' weights that are written (not added to) still look at the lengths
and the offsets, and report what is wrong with them; calls that write nothing launch nothing."""
import numpy as np
import pytest
import torch

import paper_2606_26631_amd as prcr
from gpu_util import DEV, to_dev
from test_gpu_chunk import Inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("block", [0, 16])
@pytest.mark.parametrize("lens,off,q_len,want", [
    ([3, 4], [0, 0, 0], None, 0),
    ([3, 4000], [0, 0, 0], None, prcr.DERR_CAPACITY),
    ([-1, 4], [0, 0, 0], None, prcr.DERR_CAPACITY),
    ([3, 4], [0, 1, 0], None, prcr.DERR_OFFSETS),
    ([3, 4], [0, 0, 0], [0, 1], prcr.DERR_OFFSETS),
    ([3, 4000], [0, -1, 0], None, prcr.DERR_CAPACITY | prcr.DERR_OFFSETS),
])
def test_no_rows_are_reported_on(lens, off, q_len, want, block):
    print(f"no rows: lengths {lens}, offsets {off}, counts {q_len}", flush=True)
    x = Inputs("bf16", 64, 1, 2, [0, 0], [3, 4], block, extra=0, seed=1)
    x.lens, x.off = np.array(lens, np.int32), np.array(off, np.int32)
    args = x.args(x.cache())
    n = None if q_len is None else to_dev(np.array(q_len, np.int32))
    lse = torch.empty((0, 2), device=DEV)
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    w = prcr.key_weights(*args, lse, q_len=n, err=err)
    torch.cuda.synchronize()
    assert int(err.item()) == want and not w.any()
    err.zero_()
    old = torch.rand_like(w)
    w = prcr.key_weights(*args, lse, q_len=n, weights=old.clone(), accumulate=True, err=err)
    out, got = prcr.chunk_attention(*args, q_len=n, err=err)
    torch.cuda.synchronize()
    assert int(err.item()) == 0 and torch.equal(w, old) and out.shape == (0, 2, 64) and got.shape == (0, 2)
