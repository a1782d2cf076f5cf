"""Revisits into the cache in 8 bits by batches of 6 to 65 sequences that revisit few tokens each or none, as a server's
do at most steps: the tokens of one wave then belong to several sequences.  Every call is compared with the plain 64-bit
form, rows, slots and lengths, and must report nothing."""
import numpy as np
import pytest
import torch

import paper_2606_26631_amd as prcr
from gpu_util import DEV
from quant_ref import CODES, Store
from test_gpu_quant_write import ROPES, Revisit, picks_of

pytestmark = pytest.mark.gpu

NL, H, M = 2, 1, 9


def revisit(counts, dtype, D, kind="e4m3", block=0, key_only=False, change=None):
    B = len(counts)
    x = Revisit(dtype, D, NL, H, M, picks_of(counts, M, B), np.arange(B) % 5 + 1, seed=B + D, key_only=key_only)
    if change is not None:
        change(x)
        x.idx = np.concatenate(x.picks).astype(np.int32)
    store = Store(CODES[kind], B, NL, H, D, 16, block, seed=4)
    if key_only:
        store.fill(seed=9)
    cache, err = store.to(DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    rope = prcr.Rope(*ROPES[D][B % len(ROPES[D])])
    new_len, slots = x.run(rope, cache, err=err)
    assert int(err.item()) == 0, (B, counts)
    x.check(rope, store, store.take(cache), new_len, slots, store if key_only else None)


def selections(B):
    """Tokens per sequence, sparse and dense."""
    rng = np.random.default_rng(B)
    ends = np.zeros(B, int)
    ends[0], ends[B // 2], ends[-1] = 1, 3, 4
    some = rng.integers(0, 5, B)
    few = (rng.random(B) < 0.3).astype(int)
    one = few.copy()
    one[rng.integers(B)] = 8
    return [np.ones(B, int), np.full(B, 2), some, few, one, ends]


@pytest.mark.parametrize("key_only", [False, True], ids=["values", "key_only"])
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
def test_batches(dtype, D, key_only):
    print(f"revisit, batches of few tokens, {dtype} D={D} key_only={key_only}", flush=True)
    for B in range(6, 66):
        for i, counts in enumerate(selections(B)):
            revisit(counts, dtype, D, ("e4m3", "i8")[(B + i) % 2], (0, 16, 5)[(B // 2 + i) % 3], key_only)


def only(B, **tokens):
    """Counts of a batch in which the named sequences (s0, s16) alone revisit."""
    c = [0] * B
    for name, n in tokens.items():
        c[int(name[1:])] = n
    return c


# Selections of which a token lies in a wave with those of a sequence on the far side of the search.
FAR = ([("bf16", 128, only(B, s0=1, s16=3)) for B in range(17, 24)] + [("bf16", 64, only(9, s0=1, s8=3)),
       ("bf16", 128, [8] * 29 + [1] * 4), ("f32", 128, only(33, s0=1, s32=3)), ("f32", 64, only(17, s0=1, s16=3))] +
       [(dtype, D, [n] * B) for dtype, D in (("bf16", 128), ("bf16", 64), ("f32", 64), ("f32", 128)) for n in (1, 2)
        for B in (21, 37, 41, 42, 43, 45, 53, 57, 58, 59, 61, 63, 64, 65)])


@pytest.mark.parametrize("key_only", [False, True], ids=["values", "key_only"])
def test_far_apart(key_only):
    for dtype, D, counts in FAR:
        print(f"revisit, far apart, {dtype} D={D} {len(counts)} sequences of {sum(counts)} tokens", flush=True)
        revisit(counts, dtype, D, key_only=key_only)


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
def test_the_same_token_twice(dtype, D):
    """A sequence may revisit a token several times: each copy has its slot, with the position given for it."""
    print(f"revisit, the same token twice, {dtype} D={D}", flush=True)

    def twice(x):
        picked = [b for b in range(len(x.picks)) if len(x.picks[b]) >= 2]
        assert len(picked) >= 3
        for b in picked:
            x.picks[b][-1] = x.picks[b][0]
        x.picks[picked[0]][:] = x.picks[picked[0]][0]

    revisit([4, 0, 2, 1, 7, 3] * 4, dtype, D, change=twice)
    revisit([4, 0, 2, 1, 7, 3] * 4, dtype, D, "i8", 5, key_only=True, change=twice)
