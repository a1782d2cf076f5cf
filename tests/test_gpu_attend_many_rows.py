"""The forms that the operators on several tokens per sequence take for rows in quantity: chunk attention
in tiles of 128 rows, a wave 32 of them, contiguous and paged, with the keys split and not; the
keys' weights with two key blocks a wave and with the rotation of four heads a thread.  Types, head
sizes, ragged and padded batches, more than 64 sequences, values that are not finite in hidden
places, blocks outside the pool, signs of the scale, captured calls and calls on another stream.

Expected values are those of attend_ref, with its bounds; here rows are taken together where no
hidden value can matter."""
import numpy as np
import pytest
import torch

import paper_2606_26631_amd as prcr
import attend_ref
from attend_ref import BF16_HALF, F32_HALF, key_weights, scores, spans
from gpu_util import DEV, to_dev
from test_gpu_chunk import Inputs, check, run
from test_gpu_key_weights import check as check_weights

pytestmark = pytest.mark.gpu


def attention(rope, cache, q, pos, rows, lens, scale, dtype):
    """attend_ref.attention of finite values, all rows of a head at a time."""
    T, Hq = q.shape[0], q.shape[1]
    D = rope.head_dim
    out, lse = np.full((T, Hq, D), np.nan), np.full((T, Hq), np.nan)
    b_out, b_lse, mine = np.zeros((T, Hq, D)), np.zeros((T, Hq)), np.zeros(T, bool)
    half = BF16_HALF if dtype == torch.bfloat16 else 0.0
    last = BF16_HALF if dtype == torch.bfloat16 else F32_HALF
    H, values = cache.k.shape[2 if cache.table is None else 3], {}
    for b, h, g, r0, s, err, sees in scores(rope, cache, q, pos, rows, lens, scale, dtype):
        n, L = s.shape
        if n == 0:
            continue
        mine[r0:r0 + n] = True
        qh = h * (Hq // H) + g
        if b not in values:
            values[b] = cache.rows(cache.v, b, L)[0]
        some = sees.any(1)
        m = np.where(some, np.max(s, axis=1, initial=-np.inf), 0.0)
        e = np.where(sees, np.exp(s - m[:, None]), 0.0)
        l = e.sum(1)
        p = e / np.where(l == 0, 1, l)[:, None]
        v = values[b][:, h]
        o = p @ v
        out[r0:r0 + n, qh] = o
        d = err.max(1, initial=0.0)
        sums = (sees.sum(1) + 8) * F32_HALF
        b_out[r0:r0 + n, qh] = ((2 * d + 2 * sums + half) * 1.01)[:, None] * (p @ np.abs(v)) + last * np.abs(o) + 1e-30
        with np.errstate(divide="ignore"):
            lse[r0:r0 + n, qh] = np.where(some, np.log(l) + m, -np.inf)
        b_lse[r0:r0 + n, qh] = d + sums + 8 * F32_HALF * (1 + np.where(some, np.abs(np.log(np.where(some, l, 1)) + m), 0) + np.abs(m))
    return out, lse, b_out, b_lse, mine


def expect(x, scale=None, q_len=None, of=attention):
    return of(x.rope, x.host(), x.q, x.pos, spans(x.off, q_len, len(x.ns)), x.lens, x.D ** -0.5 if scale is None else scale,
              x.dtype)


def in_quantity(x):
    """More workgroups than compute units in tiles of 32 rows (see plan_chunk)."""
    B, rows = len(x.ns), x.q.shape[0] * x.G
    return B * -(-rows // (32 * B)) * x.H > 256


TYPES = [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)]
SHAPES = {
    # name: (H, G, rows per sequence, lengths, whether the keys are split)
    "ragged": (8, 4, [400, 0, 250, 1, 97], [700, 9, 250, 300, 64], False),
    "sevens": (4, 7, [170, 131], [170, 500], None),          # (of head_dim 64 only)
    "blind": (8, 2, [1025, 1040], [900, 17], False),         # more rows than slots: rows that see nothing
    "blind_split": (8, 1, [1025, 40], [900, 17], True),
    "split": (8, 4, [300], [2300], True),
}


def test_reference():
    """Rows together and rows one by one are the same."""
    x = Inputs("bf16", 64, 2, 2, [9, 3], [20, 2], 16, seed=1)
    for a, b in zip(expect(x), x.expect()):
        assert np.allclose(a, b, rtol=1e-12, atol=0, equal_nan=True)


@pytest.mark.parametrize("block", [0, 16, 5, 128])
@pytest.mark.parametrize("dtype,D", TYPES)
@pytest.mark.parametrize("shape", sorted(SHAPES))
def test_parity(shape, dtype, D, block):
    H, G, ns, lens, split = SHAPES[shape]
    print(f"chunk, many rows: {shape} {dtype} D={D} block={block}", flush=True)
    x = Inputs(dtype, D, H, G, ns, lens, block, seed=len(shape) + D + block)
    cache = x.cache()
    assert in_quantity(x)
    assert (prcr.chunk_workspace_bytes(cache, x.q.shape[0], H * G) > 0) == (D == 64 if split is None else split)
    out, lse, err = run(x, cache)
    assert err == 0
    check(out, lse, expect(x))


@pytest.mark.parametrize("scale", [-0.2, 0.0])
@pytest.mark.parametrize("block", [0, 16])
def test_scale(scale, block):
    print(f"many rows, scale {scale} block {block}", flush=True)
    x = Inputs("bf16", 128, 4, 4, [333, 200, 97], [400, 333, 97], block, seed=8)
    assert in_quantity(x)
    out, lse, err = run(x, scale=scale)
    check(out, lse, expect(x, scale=scale))


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("f32", 64)])
def test_padded(dtype, D):
    print(f"many rows, padded {dtype} {D}", flush=True)
    n = np.array([150, 1, 0, 60, 128], np.int32)
    x = Inputs(dtype, D, 4, 4, [150] * 5, [400, 4, 9, 60, 500], 16, seed=3)
    assert in_quantity(x)
    out, lse, err = run(x, q_len=to_dev(n))
    assert err == 0
    check(out, lse, expect(x, q_len=n))


@pytest.mark.parametrize("block", [0, 24])
@pytest.mark.parametrize("B", [64, 65, 131])
def test_many_sequences(B, block):
    """Up to 64 sequences have their tiles counted; of more, slots are left free."""
    print(f"many rows of {B} sequences, block {block}", flush=True)
    rng = np.random.default_rng(B)
    ns = rng.integers(0, 80, B)
    ns[5], ns[B - 1] = 32, 33
    x = Inputs("bf16", 128, 4, 4, ns, ns + rng.integers(0, 60, B), block, seed=B, layers=1)
    assert in_quantity(x)
    out, lse, err = run(x)
    assert err == 0
    check(out, lse, expect(x))


@pytest.mark.parametrize("dtype,D,block", [("bf16", 128, 0), ("bf16", 128, 16), ("bf16", 64, 5), ("f32", 128, 0),
                                           ("f32", 128, 16), ("f32", 64, 0)])
def test_hidden_places(dtype, D, block):
    """NaN and infinities behind the lengths and at newer tokens than a row's own, in tiles at the
    first rows' last slots and in ones that the other rows of a workgroup see whole."""
    print(f"many rows, hidden places {dtype} {D} {block}", flush=True)
    x = Inputs(dtype, D, 8, 2, [520, 40], [600, 90], block, seed=11, layers=1)
    assert in_quantity(x)
    host = x.host()

    def put(tensor, b, slot, value):
        at, _ = host.at(b, [slot])
        if x.table is None:
            tensor[b, x.layer, :, slot] = value
        else:
            tensor[x.layer, at[0][0], at[1][0]] = value

    for j in range(90, 93):
        put(x.k, 1, j, float("nan"))
        put(x.v, 1, j, float("inf"))
    for j in (600, 603):
        put(x.k, 0, j, float("inf"))
        put(x.v, 0, j, float("nan"))
    put(x.v, 0, 130, float("inf"))           # row 50 of sequence 0: seen from there on
    put(x.v, 0, 200, float("-inf"))          # row 120: with the one above, NaN
    put(x.k, 0, 580, float("nan"))           # row 500
    put(x.v, 1, 60, float("nan"))            # row 10 of sequence 1
    out, lse, err = run(x)
    check(out, lse, expect(x, of=attend_ref.attention))
    o, l = out.float().cpu().numpy(), lse.cpu().numpy()
    assert np.isfinite(o[:50]).all() and np.isposinf(o[50:120]).all() and np.isnan(o[120:520]).all()
    assert np.isfinite(o[520:530]).all() and np.isnan(o[530:560]).all()
    assert np.isfinite(l[:500]).all() and np.isnan(l[500:520]).all() and np.isfinite(l[520:560]).all()


def test_nan_query_stays_in_its_row():
    print("many rows, NaN query", flush=True)
    x = Inputs("bf16", 128, 4, 4, [600], [700], 16, seed=12)
    assert in_quantity(x)
    want = expect(x)
    x.q[300, 7, 5] = float("nan")
    out, lse, _ = run(x)
    assert torch.isnan(out[300, 7]).all() and torch.isnan(lse[300, 7])
    # (The other rows need not keep their bits.  A wave's 32 rows take a new maximum together, as soon
    # as one of them needs it, so that row 300 has a say in when the others do; any maximum within
    # 2^8 of a row's own leaves its sums as exact, to float32's roundings, which the bounds count.)
    out[300, 7], lse[300, 7] = torch.from_numpy(want[0][300, 7]).to(out), float(want[1][300, 7])
    check(out, lse, want)


@pytest.mark.parametrize("dtype,D,block", [("bf16", 128, 16), ("bf16", 128, 5), ("bf16", 64, 128), ("f32", 128, 16),
                                           ("f32", 64, 24)])
def test_bad_blocks(dtype, D, block):
    """Blocks outside the pool among the tiles that all rows see whole, and among the others."""
    print(f"many rows, bad blocks {dtype} {D} {block}", flush=True)
    x = Inputs(dtype, D, 4, 4, [333, 0, 333], [900, 40, 400], block, seed=13)
    assert in_quantity(x)
    last = x.table.shape[1] - 1
    for b, at, value in ((0, 2, -1), (0, 300 // block, 1 << 30), (0, 800 // block, x.k.shape[1]), (2, 0, -7), (2, last, -1)):
        x.table[b, min(at, last)] = value
    out, lse, err = run(x)
    assert err == prcr.DERR_BLOCK
    check(out, lse, expect(x))


@pytest.mark.parametrize("name,ns,lens,cap", [("unsplit", [333, 200, 97], [400, 333, 97], 600), ("split", [300], [1900], 2300)])
def test_captured_and_replayed(name, ns, lens, cap):
    x = Inputs("bf16", 128, 8 if name == "split" else 4, 4, ns, lens, 16, seed=15, cap=cap, layers=1)
    assert in_quantity(x)
    cache = x.cache()
    args = list(x.args(cache))
    T, Hq = x.q.shape[:2]
    n = prcr.chunk_workspace_bytes(cache, T, Hq)
    assert (n > 0) == (name == "split")
    ws = torch.empty(max(n, 16), dtype=torch.uint8, device=DEV)
    out, lse = torch.full((T, Hq, 128), 7.0, dtype=x.dtype, device=DEV), torch.full((T, Hq), 7.0, device=DEV)
    call = lambda: prcr.chunk_attention(*args, out=out, lse=lse, workspace=ws)
    call()
    torch.cuda.synchronize()
    print(f"many rows, captured, {name}", flush=True)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for i in range(4):
        x.q = torch.randn(x.q.shape, generator=torch.Generator().manual_seed(i)).bfloat16()
        x.lens = np.minimum(np.array(lens) + 60 * (2 - i), cap).astype(np.int32)
        args[3].copy_(x.q)
        args[6].copy_(torch.from_numpy(x.lens))
        out.fill_(7.0)
        lse.fill_(7.0)
        ws.fill_(255)
        g.replay()
        torch.cuda.synchronize()
        check(out, lse, expect(x))
        eager = prcr.chunk_attention(*args)
        torch.cuda.synchronize()
        rows = sum(ns)
        assert torch.equal(eager[0][:rows], out[:rows]) and torch.equal(eager[1][:rows], lse[:rows])


def test_two_streams_and_the_same_each_time():
    a, b = (Inputs("bf16", 128, 4, 4, [333, 200, 97], [700, 333, 97], 16, seed=s) for s in (16, 17))
    ca, cb = a.cache(), b.cache()
    xa, xb = a.args(ca), b.args(cb)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    print("many rows, two streams", flush=True)
    got = [(prcr.chunk_attention(*xa, stream=side), prcr.chunk_attention(*xb)) for _ in range(4)]
    torch.cuda.synchronize()
    n = 630
    for x, i in ((a, 0), (b, 1)):
        for other in got[1:]:
            assert torch.equal(got[0][i][0][:n].view(torch.int16), other[i][0][:n].view(torch.int16))
            assert torch.equal(got[0][i][1][:n], other[i][1][:n])
        out, lse = got[0][i]
        out[n:], lse[n:] = 7.0, 7.0
        check(out, lse, expect(x))


# --- the keys' weights -----------------------------------------------------------------------

WEIGHTS = {
    # name: (H, G, rows, lengths, capacity); plan_key_weights takes two key blocks for rows x stretches of 128
    # slots of 1,500,000 and more: the capacity, which stands for the lengths there, makes them many.
    "shares": (4, 4, [300, 310], [420, 700], 20000),
    "one_share": (4, 4, [129, 128, 127, 100, 140], [129, 300, 127, 513, 900], 20000),
    "long": (4, 8, [480, 500, 470], [2600, 500, 1900], 4300),
    "blind": (4, 4, [300, 310], [250, 12], 20000),
}


def two_blocks(x, cap):
    T, B = x.q.shape[0], len(x.ns)
    return -(-T // B) * x.G * -(-cap // 128) * B * x.H >= 1500000


def four_heads(x):
    """The rotation takes four heads a thread (see rotate_dim)."""
    return x.q.shape[0] * x.H * x.G * (x.D // 16) >= 1 << 16


def weigh(x, window=None, start=None, q_len=None, scale=None):
    sc = x.D ** -0.5 if scale is None else scale
    rows = spans(x.off, q_len, len(x.ns))
    lse = expect(x, scale=sc, q_len=q_len)[1].astype(np.float32)
    want, bound = key_weights(x.rope, x.host(), x.q, x.pos, rows, x.lens, sc, x.dtype, lse, window)
    if start is not None:
        want, bound = want + start, bound + 2.0 ** -24 * (2 * np.abs(start) + want)
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    got = prcr.key_weights(*x.args(x.cache()), to_dev(lse), window=window, scale=scale, err=err,
                           q_len=None if q_len is None else to_dev(q_len),
                           weights=None if start is None else to_dev(start), accumulate=start is not None)
    torch.cuda.synchronize()
    return got, want, bound, int(err.item())


@pytest.mark.parametrize("block", [0, 16, 5])
@pytest.mark.parametrize("D", [128, 64])
@pytest.mark.parametrize("name", sorted(WEIGHTS))
def test_two_key_blocks(name, D, block):
    H, G, ns, lens, cap = WEIGHTS[name]
    print(f"two key blocks: {name} D={D} block={block}", flush=True)
    x = Inputs("bf16", D, H, G, ns, lens, block, seed=len(name) + D + block, cap=cap, layers=1)
    assert two_blocks(x, cap)
    got, want, bound, err = weigh(x)
    assert err == 0
    check_weights(got, want, bound)
    start = np.random.default_rng(1).random(want.shape).astype(np.float32)
    got, want, bound, err = weigh(x, start=start)
    check_weights(got, want, bound)
    for b, n in enumerate(x.lens):
        assert np.array_equal(got[b, :, n:].cpu().numpy(), start[b, :, n:])


def test_two_key_blocks_scale_nan_and_bad_blocks():
    H, G, ns, lens, cap = WEIGHTS["shares"]
    print("two key blocks, negative scale, NaN, bad blocks", flush=True)
    x = Inputs("bf16", 128, H, G, ns, lens, 16, seed=9, cap=cap, layers=1)
    assert two_blocks(x, cap)
    x.table[0, 3], x.table[1, 0], x.table[1, 43] = -1, x.k.shape[1], -7
    got, want, bound, err = weigh(x, scale=-0.11)
    assert err == prcr.DERR_BLOCK
    check_weights(got, want, bound)
    x = Inputs("bf16", 128, H, G, ns, lens, 0, seed=9, cap=cap, layers=1)
    args = x.args(x.cache())
    lse = prcr.chunk_attention(*args)[1]
    clean = prcr.key_weights(*args, lse)
    q = args[3].clone()
    q[10, 1, 3] = float("nan")               # sequence 0, head 0, slots 0 .. 130
    got = prcr.key_weights(*args[:3], q, *args[4:], lse)
    torch.cuda.synchronize()
    assert bool(got[0, 0, :131].isnan().all())
    got[0, 0, :131] = clean[0, 0, :131]
    assert torch.equal(got, clean)


@pytest.mark.parametrize("H,G", [(4, 4), (3, 3), (1, 5), (2, 7)])
@pytest.mark.parametrize("D", [128, 64])
def test_rotation_of_four_heads(D, H, G):
    """Heads that fill their groups of four, and that do not; all rows, windows, padded rows."""
    n = -(-(1 << 16) // (H * G * (D // 16) * 4)) + 3
    print(f"rotation of four heads, D={D} {H}x{G}, {n} rows each", flush=True)
    x = Inputs("bf16", D, H, G, [n, n, n, n], [n, n + 60, n // 2, n], 16, seed=D + H, layers=1)
    assert four_heads(x) and not two_blocks(x, x.table.shape[1] * 16)
    some = np.array([n, n - 9, 3, 0], np.int32)
    for kw in (dict(), dict(window=32), dict(window=5, q_len=some), dict(q_len=some, scale=-0.1)):
        got, want, bound, err = weigh(x, **kw)
        assert err == 0
        check_weights(got, want, bound)


def test_weights_captured_and_replayed():
    H, G, ns, lens, cap = WEIGHTS["shares"]
    x = Inputs("bf16", 128, H, G, ns, lens, 16, seed=15, cap=cap, layers=1)
    assert two_blocks(x, cap) and four_heads(x)
    args = list(x.args(x.cache()))
    lse = prcr.chunk_attention(*args)[1]
    ws = torch.empty(prcr.key_weights_workspace_bytes(args[1], *x.q.shape[:2]), dtype=torch.uint8, device=DEV)
    w = torch.zeros((2, H, x.table.shape[1] * 16), device=DEV)
    call = lambda: prcr.key_weights(*args, lse, weights=w, workspace=ws)
    call()
    torch.cuda.synchronize()
    print("two key blocks, captured", flush=True)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for i in range(4):
        args[3].copy_(torch.randn(x.q.shape, generator=torch.Generator().manual_seed(i)).bfloat16())
        args[6].copy_(torch.tensor([420 + 300 * i, 700 - 100 * i], dtype=torch.int32))
        lse.copy_(prcr.chunk_attention(*args)[1])
        ws.fill_(255)
        w.fill_(5.0)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(w, prcr.key_weights(*args, lse))
        # every row of the two sequences gives its heads' sum of one
        sees = np.minimum(np.array(ns), args[6].cpu().numpy())
        assert torch.allclose(w.sum(-1), torch.tensor(sees * G, dtype=torch.float32, device=DEV)[:, None].expand(2, H), rtol=1e-4)
