"""Chunk attention against a plain 64-bit form: types, head layouts, lengths from none to some
thousands, odd blocks, masks that leave rows or sequences empty, values that are not finite in
hidden places, bad data, captured calls and calls on another stream.

Tolerances are element by element and come from the arithmetic (attend_ref.attention)."""
import numpy as np
import pytest
import torch

import paper_2606_26631_amd as prcr
from attend_ref import HostCache, attention, spans
from gpu_util import DEV, to_dev

pytestmark = pytest.mark.gpu

ROPES = {64: (64, (8, 12, 12), False, 1e6), 128: (128, (24, 20, 20), True, 5e6)}
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


class Inputs:
    def __init__(self, dtype, D, H, G, ns, lens, block=0, seed=0, extra=3, cap=None, layers=2):
        g = torch.Generator().manual_seed(seed)
        rng = np.random.default_rng(seed)
        self.dtype, self.H, self.G, self.D, self.layer = TYPES[dtype], H, G, D, layers - 1
        self.ns, self.lens = np.asarray(ns), np.asarray(lens, np.int32)
        B = len(ns)
        cap = cap or int(max(max(lens), 1)) + 5
        rnd = lambda *s: torch.randn(s, generator=g).to(self.dtype)
        self.table = None
        if block:
            per = -(-cap // block)
            self.table = rng.permutation(B * per).astype(np.int32).reshape(B, per)
            shape = (layers, B * per, block, H, D)
        else:
            shape = (B, layers, H, cap, D)
        self.k, self.v = rnd(*shape) * 1.5, rnd(*shape)
        T = int(self.ns.sum()) + extra       # rows behind the last sequence
        self.q = rnd(T, H * G, D)
        self.off = np.concatenate([[0], np.cumsum(self.ns)]).astype(np.int32)
        self.pos = rng.integers(0, 5000, (T, 3)).astype(np.int32)
        self.rope = prcr.Rope(*ROPES[D])

    def cache(self):
        return prcr.Cache(self.k.to(DEV), self.v.to(DEV), None if self.table is None else to_dev(self.table))

    def args(self, cache):
        return (self.rope, cache, self.layer, self.q.to(DEV), to_dev(self.off), to_dev(self.pos), to_dev(self.lens))

    def host(self):
        return HostCache(self.k, self.v, self.table, self.layer)

    def expect(self, scale=None, q_len=None):
        return attention(self.rope, self.host(), self.q, self.pos, spans(self.off, q_len, len(self.ns)), self.lens,
                         self.D ** -0.5 if scale is None else scale, self.dtype)


def check(out, lse, want, fill=7.0):
    o, l, b_o, b_l, rows = want
    out, lse = out.float().cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64)
    mine = np.broadcast_to(rows[:, None], l.shape)
    none = ~mine
    assert np.array_equal(out[none], np.full_like(out[none], fill)), "a row of no sequence was written"
    assert np.array_equal(lse[none], np.full_like(lse[none], fill)), "an lse of no sequence was written"
    assert np.array_equal(np.isfinite(o[mine]), np.isfinite(out[mine])), "other elements are finite"
    empty = mine & np.isneginf(l)
    assert not out[empty].any() and np.isneginf(lse[empty]).all()
    fine = np.isfinite(o) & mine[..., None]
    d = np.abs(np.where(fine, out - np.where(fine, o, 0), 0)) - np.where(fine, b_o, 0)
    assert d.max(initial=-1) <= 0, (np.unravel_index(d.argmax(), d.shape), d.max())
    fl = np.isfinite(l) & mine
    d = np.abs(np.where(fl, lse - np.where(fl, l, 0), 0)) - np.where(fl, b_l, 0)
    assert d.max(initial=-1) <= 0, (np.unravel_index(d.argmax(), d.shape), d.max())


def run(x, cache=None, **kw):
    cache = cache or x.cache()
    T = x.q.shape[0]
    out = torch.full((T, x.H * x.G, x.D), 7.0, dtype=x.dtype, device=DEV)
    lse = torch.full((T, x.H * x.G), 7.0, dtype=torch.float32, device=DEV)
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    got = prcr.chunk_attention(*x.args(cache), out=out, lse=lse, err=err, **kw)
    torch.cuda.synchronize()
    assert got[0] is out and got[1] is lse
    return out, lse, int(err.item())


SHAPES = {
    # name: (H, G, rows per sequence, lengths)
    "tokens": (2, 4, [1, 1, 1, 1], [1, 300, 64, 65]),
    "mixed": (2, 3, [1, 40, 0, 7, 130], [17, 200, 90, 7, 131]),
    "prompts": (1, 8, [97, 33, 256], [97, 33, 256]),
    "empty": (2, 2, [0, 3, 5, 0], [10, 0, 3, 0]),      # more rows than slots: rows that see nothing
    "one": (1, 1, [1], [1]),
    "wide": (3, 16, [9, 2], [70, 300]),
    "seven": (4, 7, [60, 19], [500, 333]),
}


@pytest.mark.parametrize("block", [0, 16, 5, 1, 128])
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("shape", sorted(SHAPES))
def test_parity(shape, dtype, D, block):
    H, G, ns, lens = SHAPES[shape]
    x = Inputs(dtype, D, H, G, ns, lens, block, seed=len(shape) + D + block)
    print(f"chunk {shape} {dtype} D={D} block={block}", flush=True)
    out, lse, err = run(x)
    assert err == 0
    check(out, lse, x.expect())


@pytest.mark.parametrize("dtype,block", [("bf16", 0), ("bf16", 16), ("f32", 0), ("bf16", 24)])
def test_longer(dtype, block):
    """A prompt of many tiles beside a chunk on a long past, and a call whose keys are split."""
    print(f"longer {dtype} {block}", flush=True)
    x = Inputs(dtype, 128, 2, 4, [700, 100], [700, 1500], block, seed=5)
    out, lse, err = run(x)
    assert err == 0
    check(out, lse, x.expect())
    x = Inputs(dtype, 64, 1, 2, [2], [2900], block, seed=6, cap=3000)
    assert prcr.chunk_workspace_bytes(x.cache(), x.q.shape[0], 2) > 0
    out, lse, err = run(x)
    assert err == 0
    check(out, lse, x.expect())


@pytest.mark.parametrize("B", [64, 65, 130, 4097])
def test_many_sequences(B):
    print(f"{B} sequences", flush=True)
    rng = np.random.default_rng(B)
    ns = rng.integers(0, 4, B)
    x = Inputs("bf16", 64, 1, 2, ns, np.maximum(ns, rng.integers(1, 9, B)), 8 if B == 130 else 0, seed=B)
    out, lse, err = run(x)
    assert err == 0
    check(out, lse, x.expect())


@pytest.mark.parametrize("block", [0, 16])
def test_rows_that_fill_their_tiles(block):
    """64 sequences of which some have exactly one tile of 32 or 128 rows, or a row more, or none."""
    print(f"whole tiles, block {block}", flush=True)
    ns = np.array([32, 0, 33, 1, 31, 128, 0, 129, 64, 16] * 6 + [0, 0, 32, 5])
    x = Inputs("bf16", 64, 2, 1, ns, ns + np.arange(64) % 7 * 40, block, seed=21)
    out, lse, err = run(x)
    assert err == 0
    check(out, lse, x.expect())


@pytest.mark.parametrize("H,G,n,past", [(4, 7, 400, 1500), (8, 4, 400, 100), (2, 4, 40, 4000)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_and_keys_shared_out(dtype, H, G, n, past):
    """One sequence: tiles of 128 rows, or of 32, with the keys split."""
    print(f"shared out {dtype} {H} {G} {n} {past}", flush=True)
    x = Inputs(dtype, 64, H, G, [n], [n + past], seed=n + past, layers=1)
    assert prcr.chunk_workspace_bytes(x.cache(), x.q.shape[0], H * G) > 0
    out, lse, err = run(x)
    assert err == 0
    check(out, lse, x.expect())


@pytest.mark.parametrize("seed", range(6))
def test_float32_scores_of_one_token(seed):
    """One token over 300 slots, scores of some tens: the whole error stays below 1e-6.  (The
    scores in four sums of 16 products, the sums' errors kept: 0.3 units of 2^-24 x 30 each, and
    a weight's exponential and the sums' roundings about three of 2^-24.)"""
    print(f"float32 scores, seed {seed}", flush=True)
    x = Inputs("f32", 64, 2, 2, [1], [300], seed=seed)
    x.q, x.k = x.q * 2, x.k * 2
    out, lse, err = run(x)
    assert err == 0
    o, l, _, _, rows = x.expect()
    got = out.cpu().numpy().astype(np.float64)[rows]
    assert np.linalg.norm(got - o[rows]) <= 1e-6 * np.linalg.norm(o[rows])


def test_padded_rows():
    """A padded [B, S] batch: offsets b S and the rows' counts; padding is left as it is."""
    S, n = 9, np.array([9, 4, 0, 1], np.int32)
    x = Inputs("bf16", 128, 2, 2, [S] * 4, [40, 4, 9, 1], 16, seed=3)
    print("padded rows", flush=True)
    out, lse, err = run(x, q_len=to_dev(n))
    assert err == 0
    check(out, lse, x.expect(q_len=n))


@pytest.mark.parametrize("scale", [-0.2, 0.0, 3.0])
def test_scale(scale):
    x = Inputs("bf16", 64, 2, 2, [40, 1], [90, 30], seed=8)
    print(f"scale {scale}", flush=True)
    out, lse, err = run(x, scale=scale)
    check(out, lse, x.expect(scale=scale))


def test_far_positions():
    x = Inputs("f32", 128, 1, 2, [20], [60], seed=9)
    x.pos = np.random.default_rng(1).integers(-2 ** 31, 2 ** 31, x.pos.shape).astype(np.int32)
    print("far positions", flush=True)
    out, lse, err = run(x)
    check(out, lse, x.expect())


@pytest.mark.parametrize("dtype,block", [("bf16", 0), ("f32", 0), ("bf16", 16)])
def test_hidden_places(dtype, block):
    """NaN and infinities behind the length, and at newer tokens than a row's own."""
    x = Inputs(dtype, 128, 1, 2, [50, 3], [90, 20], block, seed=11)
    print(f"hidden places {dtype} {block}", flush=True)
    host = x.host()

    def put(tensor, b, slot, value):
        at, _ = host.at(b, [slot])
        if x.table is None:
            tensor[b, x.layer, :, slot] = value
        else:
            tensor[x.layer, at[0][0], at[1][0]] = value

    for j in range(90, 95):
        put(x.k, 0, j, float("nan"))
        put(x.v, 0, j, float("inf"))
    put(x.v, 0, 60, float("inf"))            # row 20 of sequence 0: seen from there on
    put(x.v, 0, 70, float("-inf"))           # row 30: with the one above, NaN
    put(x.v, 0, 75, float("nan"))
    put(x.k, 1, 19, float("nan"))            # the last row of sequence 1 only
    out, lse, err = run(x)
    want = x.expect()
    check(out, lse, want)
    o = out.float().cpu().numpy()
    assert np.isfinite(o[:20]).all() and np.isposinf(o[20:30]).all() and np.isnan(o[30:50]).all()
    assert np.isfinite(o[50:52]).all() and np.isnan(o[52]).all()
    lse = lse.cpu().numpy()
    assert np.isfinite(lse[:52]).all() and np.isnan(lse[52]).all()


def test_nan_query_stays_in_its_row():
    x = Inputs("bf16", 128, 2, 2, [40], [70], seed=12)
    clean, _, _ = run(x)
    x.q[7, 3, 5] = float("nan")
    print("NaN query", flush=True)
    out, lse, _ = run(x)
    o = out.float().cpu()
    assert torch.isnan(o[7, 3]).all() and torch.isnan(lse[7, 3])
    o[7, 3] = clean.float().cpu()[7, 3]
    assert torch.equal(o, clean.float().cpu())


@pytest.mark.parametrize("block", [16, 5])
def test_bad_blocks(block):
    x = Inputs("bf16", 64, 2, 2, [30, 30], [80, 100], block, seed=13)
    x.table[0, 1], x.table[1, 0], x.table[1, -1] = -1, x.k.shape[1], -7
    print(f"bad blocks {block}", flush=True)
    out, lse, err = run(x)
    assert err == prcr.DERR_BLOCK
    check(out, lse, x.expect())


def test_bad_offsets_and_lengths():
    x = Inputs("bf16", 64, 1, 2, [4, 6, 5], [20, 30, 40], seed=14, cap=50)
    print("bad lengths", flush=True)
    x.lens = np.array([20, 30, 4000], np.int32)
    out, lse, err = run(x)
    assert err == prcr.DERR_CAPACITY
    x.lens = np.array([20, 30, 50], np.int32)
    check(out, lse, x.expect())
    print("bad counts", flush=True)
    n = np.array([4, 7, 5], np.int32)        # one more row than the second sequence has
    out, lse, err = run(x, q_len=to_dev(n))
    assert err == prcr.DERR_OFFSETS
    check(out, lse, x.expect(q_len=np.array([4, 0, 5])))
    print("bad offsets", flush=True)
    x.off = np.array([0, 4, 2, 15], np.int32)
    out, lse, err = run(x)
    assert err == prcr.DERR_OFFSETS
    for off in ([-5, 4, 10, 15], [0, 4, 10, 9000], [9, 8, 7, 6]):
        x.off = np.array(off, np.int32)
        assert run(x)[2] == prcr.DERR_OFFSETS


def test_no_rows():
    x = Inputs("bf16", 64, 1, 2, [0, 0], [3, 4], extra=0, seed=1)
    print("no rows", flush=True)
    out, lse, err = run(x)
    assert out.shape == (0, 2, 64) and err == 0


def test_offsets_beyond_32_bits():
    """A sequence whose rows lie more than 2^32 bytes from the cache's start."""
    D, n = 64, 35_000_000
    k = torch.zeros((1, 1, 1, n + 8, D), dtype=torch.bfloat16, device=DEV)
    v = torch.zeros_like(k)
    assert n * D * 2 > 2 ** 32
    at = n - 3
    rope = prcr.Rope(D, (32, 0, 0), False, 1e4)
    q = torch.ones((2, 1, D), dtype=torch.bfloat16, device=DEV)
    pos = torch.zeros((2, 3), dtype=torch.int32, device=DEV)
    k[0, 0, 0, at] = 8.0                     # score 64 against 0: weight all but 35e6 e^-64
    v[0, 0, 0, at] = torch.arange(D, device=DEV).bfloat16()
    print("beyond 32 bits", flush=True)
    cache = prcr.Cache(k, v)
    off, lens = to_dev(np.array([0, 2], np.int32)), to_dev(np.array([n], np.int32))
    out, lse = prcr.chunk_attention(rope, cache, 0, q, off, pos, lens)
    torch.cuda.synchronize()
    assert torch.equal(out[:, 0].float(), torch.arange(D, device=DEV).float().expand(2, D))
    assert torch.allclose(lse, torch.full_like(lse, 64.0), rtol=1e-6)
    w = prcr.key_weights(rope, cache, 0, q, off, pos, lens, lse)
    torch.cuda.synchronize()
    assert abs(float(w[0, 0, at]) - 2.0) < 1e-4 and float(w[0, 0, n - 1]) < 1e-20 and float(w[0, 0, n]) == 0


def test_captured_and_replayed():
    x = Inputs("bf16", 128, 2, 4, [3, 60], [700, 90], 16, seed=15)
    cache = x.cache()
    args = list(x.args(cache))
    ws = torch.empty(max(prcr.chunk_workspace_bytes(cache, x.q.shape[0], 8), 4), dtype=torch.uint8, device=DEV)
    out = torch.full((x.q.shape[0], 8, 128), 7.0, dtype=x.dtype, device=DEV)
    lse = torch.full((x.q.shape[0], 8), 7.0, device=DEV)
    call = lambda: prcr.chunk_attention(*args, out=out, lse=lse, workspace=ws)
    call()
    torch.cuda.synchronize()
    print("captured", flush=True)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for i in range(4):
        x.q = torch.randn(x.q.shape, generator=torch.Generator().manual_seed(i)).bfloat16()
        x.lens = np.array([700 - 100 * i, 60 + 10 * i], np.int32)
        args[3].copy_(x.q)
        args[6].copy_(torch.from_numpy(x.lens))
        out.fill_(7.0)
        lse.fill_(7.0)
        ws.fill_(255)                        # (nothing is kept there from call to call)
        g.replay()
        torch.cuda.synchronize()
        check(out, lse, x.expect())
        eager = prcr.chunk_attention(*args)
        torch.cuda.synchronize()
        assert torch.equal(eager[0][:63], out[:63]) and torch.equal(eager[1][:63], lse[:63])


def test_other_stream_and_two_at_once():
    a, b = (Inputs("bf16", 128, 2, 4, [3, 60], [700, 90], 16, seed=s) for s in (16, 17))
    ca, cb = a.cache(), b.cache()
    xa, xb = a.args(ca), b.args(cb)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    print("two streams", flush=True)
    for _ in range(3):
        ra = prcr.chunk_attention(*xa, stream=side)
        rb = prcr.chunk_attention(*xb)
    torch.cuda.synchronize()
    for x, (out, lse) in ((a, ra), (b, rb)):
        out[63:], lse[63:] = 7.0, 7.0
        check(out, lse, x.expect())


def test_same_results_each_time():
    x = Inputs("bf16", 128, 2, 4, [500, 1], [900, 900], 16, seed=18)
    cache = x.cache()
    first = [t.clone() for t in run(x, cache)[:2]]
    for _ in range(5):
        again = run(x, cache)[:2]
        assert torch.equal(first[0].view(torch.int16), again[0].view(torch.int16)) and torch.equal(first[1], again[1])
