"""Decode attention over the cache in 8 bits against a plain 64-bit form: types, codes, head layouts, lengths from
none to some thousands, odd blocks, rows that are not finite in hidden places and in seen ones, bad data.

Tolerances are element by element and come from the arithmetic (quant_ref.attention)."""
import numpy as np
import pytest
import torch

import paper_2606_26631_amd as prcr
from gpu_util import DEV, to_dev
from quant_ref import CODES, TYPES, Store, attention, check_attention

pytestmark = pytest.mark.gpu

ROPES = {64: (64, (8, 12, 12), False, 1e6), 128: (128, (24, 20, 20), True, 5e6)}


def inputs(dtype, D, H, G, lens, seed):
    g = torch.Generator().manual_seed(seed)
    q = torch.randn((len(lens), H * G, D), generator=g).to(TYPES[dtype])
    q_pos = np.random.default_rng(seed).integers(0, 100000, len(lens)).astype(np.int32)
    return q, q_pos, np.asarray(lens, np.int32)


def run(rope, cache, layer, q, q_pos, lens, **kw):
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    out = prcr.quant_decode_attention(rope, cache, layer, q.to(DEV), to_dev(q_pos), to_dev(lens), err=err, **kw)
    torch.cuda.synchronize()
    return out, int(err.item())


SHAPES = {
    # name: (H, G, lengths, capacity)
    "lengths": (2, 4, [1, 0, 31, 32, 33, 129, 300], 300),
    "seven": (4, 7, [500, 333, 64], 512),
    "one": (1, 1, [1], 8),
    "two": (3, 2, [700, 20], 1000),
    "eight": (1, 8, [257, 4, 96], 260),
    "three": (5, 3, [90], 2100),
    "long": (1, 6, [5000], 5001),
    "roomy": (2, 4, [40, 1100], 9000),
    "pairs of heads": (8, 4, [1100, 40, 0, 900], 1200),
    "ten heads": (10, 3, [2100], 2150),
    "many rows": (4, 2, [33, 0, 64, 200, 1, 130, 299, 300], 300),
    "odd rows": (6, 1, [90, 7, 250], 2500),
}


@pytest.mark.parametrize("block", [0, 16, 5, 64])
@pytest.mark.parametrize("kind", sorted(CODES))
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("f32", 128), ("bf16", 64), ("f32", 64)])
@pytest.mark.parametrize("shape", sorted(SHAPES))
def test_parity(shape, dtype, D, kind, block):
    H, G, lens, cap = SHAPES[shape]
    print(f"quant decode {shape} {dtype} D={D} {kind} block={block}", flush=True)
    store = Store(CODES[kind], len(lens), 2, H, D, cap, block, seed=1).fill(seed=len(shape))
    x = inputs(dtype, D, H, G, lens, seed=D + block)
    rope = prcr.Rope(*ROPES[D])
    out, err = run(rope, store.to(DEV), 1, *x)
    assert err == 0
    check_attention(out, attention(rope, store, 1, *x, D ** -0.5))


def test_many_sequences():
    """More sequences than are dealt out by length, and more than there are compute units."""
    print("quant decode, many sequences", flush=True)
    for B in (65, 300):
        lens = (np.arange(B) * 37) % 90
        store = Store(torch.float8_e4m3fn, B, 1, 2, 64, 96, 16, seed=1).fill(seed=1)
        x = inputs("bf16", 64, 2, 4, lens, seed=2)
        rope = prcr.Rope(*ROPES[64])
        out, err = run(rope, store.to(DEV), 0, *x)
        assert err == 0
        check_attention(out, attention(rope, store, 0, *x, 0.125))


@pytest.mark.parametrize("block", [0, 16])
@pytest.mark.parametrize("D", [64, 128])
def test_several_chunks_of_sequences_that_differ(D, block):
    """Enough pairs of sequence and head for two rounds of workgroups over the chip, lengths from none to the
    capacity."""
    print(f"quant decode, chunks of many sequences, D={D} block={block}", flush=True)
    rng = np.random.default_rng(D + block)
    lens = np.concatenate([[0, 1, 2100, 1023, 1024, 1025], rng.integers(2, 2100, 26)])
    store = Store(torch.int8, 32, 1, 8, D, 2100, block, seed=1).fill(seed=1)
    x = inputs("bf16", D, 8, 1, lens, seed=2)
    rope = prcr.Rope(*ROPES[D])
    out, err = run(rope, store.to(DEV), 0, *x)
    assert err == 0
    check_attention(out, attention(rope, store, 0, *x, D ** -0.5))


@pytest.mark.parametrize("scale", [0.0, -0.3, 4.0])
def test_scales(scale):
    print(f"quant decode scale={scale}", flush=True)
    store = Store(torch.int8, 2, 1, 2, 128, 200).fill(seed=3, spread=0.2)
    x = inputs("f32", 128, 2, 5, [200, 77], seed=4)
    rope = prcr.Rope(*ROPES[128])
    out, err = run(rope, store.to(DEV), 0, *x, scale=scale)
    assert err == 0
    check_attention(out, attention(rope, store, 0, *x, scale))


def poison(store, b, slots, kind):
    """Scales and codes that spoil whatever they take part in."""
    i, j = store.at(b, slots)
    i, j = (torch.from_numpy(np.atleast_1d(a)) for a in np.broadcast_arrays(i, j))
    for name in ("k", "v"):
        codes, scales = getattr(store, name).view(torch.uint8), getattr(store, name + "_scale")
        if store.block:
            codes[:, i, j] = 0x7F
            scales.transpose(2, 3)[:, i, j] = float("nan") if kind == "nan" else float("inf")
        else:
            codes[b][:, :, j] = 0x7F
            scales[b][:, :, j] = float("nan") if kind == "nan" else float("inf")


@pytest.mark.parametrize("kind", sorted(CODES))
@pytest.mark.parametrize("block", [0, 16, 5])
@pytest.mark.parametrize("what", ["nan", "inf"])
def test_hidden_rows_do_not_matter(what, block, kind):
    """Rows behind the length, of other sequences' and of unused blocks, whatever they are."""
    print(f"quant decode hidden {what} block={block} {kind}", flush=True)
    lens = [7, 0, 100, 31, 64]
    for D, dtype in ((128, "bf16"), (64, "f32")):
        store = Store(CODES[kind], 5, 1, 2, D, 130, block, seed=1).fill(seed=5)
        x = inputs(dtype, D, 2, 4, lens, seed=6)
        rope = prcr.Rope(*ROPES[D])
        want = attention(rope, store, 0, *x, D ** -0.5)
        for b, n in enumerate(lens):
            poison(store, b, np.arange(n, store.cap), what)
        out, err = run(rope, store.to(DEV), 0, *x)
        assert err == 0
        check_attention(out, want)
        assert not out[1].any()


@pytest.mark.parametrize("array", ["k", "v"])
@pytest.mark.parametrize("at", [0, 40, 99])
def test_a_row_without_values_that_is_seen(array, at):
    """A seen row's scale of NaN makes its heads NaN, and no others."""
    print(f"quant decode NaN in {array} at {at}", flush=True)
    store = Store(torch.float8_e4m3fn, 3, 1, 2, 128, 100).fill(seed=7)
    x = inputs("bf16", 128, 2, 3, [100, 100, 50], seed=8)
    rope = prcr.Rope(*ROPES[128])
    want, bound = attention(rope, store, 0, *x, 0.1)
    getattr(store, array + "_scale")[1, 0, 1, at] = float("nan")
    out, err = run(rope, store.to(DEV), 0, *x, scale=0.1)
    assert err == 0
    want[1, 3:] = np.nan
    check_attention(out, (want, bound))


@pytest.mark.parametrize("block", [0, 16, 7])
def test_bad_data(block):
    print(f"quant decode bad data block={block}", flush=True)
    D = 128
    rope = prcr.Rope(*ROPES[D])
    store = Store(torch.int8, 3, 1, 2, D, 112, block, seed=1).fill(seed=9)
    x = inputs("bf16", D, 2, 4, [113, -4, 2 ** 31 - 1], seed=10)
    out, err = run(rope, store.to(DEV), 0, *x)
    assert err == prcr.DERR_CAPACITY
    check_attention(out, attention(rope, store, 0, *x, D ** -0.5))
    if block:
        x = inputs("bf16", D, 2, 4, [112, 60, block], seed=10)
        bad = {(0, 2), (1, 0), (2, 0)}
        want = attention(rope, store, 0, *x, D ** -0.5, skip=bad)
        for i, (b, n) in enumerate(sorted(bad)):
            store.table[b, n] = [-1, store.k.shape[1], 2 ** 31 - 1][i]
        out, err = run(rope, store.to(DEV), 0, *x)
        assert err == prcr.DERR_BLOCK
        check_attention(out, want)
        assert not out[2].any()


def test_tiny_and_large_scales():
    """Rows of zeros, of the smallest and of very large numbers, side by side."""
    print("quant decode tiny and large rows", flush=True)
    for kind in CODES.values():
        store = Store(kind, 1, 1, 1, 128, 90).fill(seed=11)
        store.k_scale[..., ::3] = 2.0 ** -126
        store.v_scale[..., 1::3] = 2.0 ** -126
        store.v_scale[..., 2::5] = 2.0 ** 90
        x = inputs("f32", 128, 1, 8, [90], seed=12)
        rope = prcr.Rope(*ROPES[128])
        out, err = run(rope, store.to(DEV), 0, *x)
        assert err == 0
        check_attention(out, attention(rope, store, 0, *x, 128 ** -0.5))


def test_result_of_a_sequence_does_not_depend_on_the_others():
    print("quant decode, batch invariance of a run", flush=True)
    store = Store(torch.float8_e4m3fn, 3, 1, 2, 128, 700).fill(seed=13)
    q, q_pos, lens = inputs("bf16", 128, 2, 4, [700, 300, 9], seed=14)
    rope = prcr.Rope(*ROPES[128])
    cache = store.to(DEV)
    a, _ = run(rope, cache, 0, q, q_pos, lens)
    b, _ = run(rope, cache, 0, q, q_pos, np.array([700, 1, 650], np.int32))
    c, _ = run(rope, cache, 0, q, q_pos, lens)
    assert torch.equal(a[0], b[0]) and torch.equal(a, c)
