"""Workspace sizes of the operators on several tokens per sequence: that of one shape says nothing about
another's, fewer rows may need more; the bounds that the header gives hold for all of them."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2606_26631_amd as prcr
from test_abi import host_only
from test_attend_refusals import attend, contiguous, paged
from test_gpu_chunk import Inputs
from gpu_util import DEV

SHAPE = 2


def chunk_bytes(cache, *shape):
    n = ctypes.c_size_t()
    assert prcr.lib().prcr_chunk_workspace_size(ctypes.byref(cache), *shape, ctypes.byref(n)) == 0
    return n.value


def weights_bytes(cache, *shape):
    n = ctypes.c_size_t()
    assert prcr.lib().prcr_key_weights_workspace_size(ctypes.byref(cache), *shape, ctypes.byref(n)) == 0
    return n.value


def most_chunk(D):
    return 2 ** 18 * (D + 2)


def most_weights(total_q, Hq, D, dtype):
    return -(-total_q * Hq * D * (2 if dtype else 4) // 256) * 256 + 2 ** 22


@pytest.mark.parametrize("seed", range(4))
def test_bounds(seed):
    rng = np.random.default_rng(seed)
    log = lambda hi: int(np.exp(rng.uniform(0, np.log(hi))))
    split = np.zeros(2, int)
    for _ in range(5000):
        H, D, dtype = log(64), int(rng.choice([64, 128])), int(rng.integers(0, 2))
        Hq, batch, T = H * log(64), log(65535), log(2 ** 21)
        if T * Hq > 2 ** 30:
            continue
        c = contiguous(log(2 ** 28)) if rng.random() < 0.5 else paged(log(512), log(2 ** 20), log(2 ** 20))
        n = chunk_bytes(c, batch, T, Hq, H, D)
        assert n <= most_chunk(D)
        window = int(rng.choice([0, 1, 32, 5000]))
        m = weights_bytes(c, dtype, batch, T, Hq, H, D, window)
        assert T * Hq * D * (2 if dtype else 4) <= m <= most_weights(T, Hq, D, dtype)
        split += [n > 0, m > most_weights(T, Hq, D, dtype) - 2 ** 22]
    assert (split > 20).all()                # (calls with partial results are among them)


@host_only
def test_the_size_of_more_rows_does_not_do():
    c = contiguous(4400)
    many, few = chunk_bytes(c, 1, 256, 32, 8, 128), chunk_bytes(c, 1, 128, 32, 8, 128)
    assert many < few
    assert attend("chunk", cache=c, batch=1, n_q_heads=32, n_kv_heads=8, total_q=128, bytes=many) == SHAPE
    c, shape = contiguous(20000), (8, 2, 128, 0)
    assert attend("weights", cache=c, batch=1, n_q_heads=8, n_kv_heads=2, total_q=600,
                  bytes=weights_bytes(c, 1, 1, 600, *shape) - 1) == SHAPE


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,block", [("bf16", 0), ("f32", 16)])
def test_one_workspace_for_calls_of_every_size(dtype, block):
    D, H, G = 64, 4, 4
    ws = torch.empty(most_weights(700, H * G, D, dtype == "bf16") + most_chunk(D), dtype=torch.uint8, device=DEV)
    sizes = set()
    for n in (1, 7, 128, 256, 400, 700):
        print(f"workspace of the bound's size, {n} rows, {dtype} {block}", flush=True)
        x = Inputs(dtype, D, H, G, [n], [n + 1900], block, seed=n, extra=0, layers=1, cap=2600)
        cache = x.cache()
        args = x.args(cache)
        sizes.add(prcr.chunk_workspace_bytes(cache, n, H * G))
        a, b = prcr.chunk_attention(*args, workspace=ws), prcr.chunk_attention(*args)
        wa, wb = prcr.key_weights(*args, a[1], workspace=ws), prcr.key_weights(*args, b[1])
        torch.cuda.synchronize()
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and torch.equal(wa, wb)
    assert len(sizes) > 3
