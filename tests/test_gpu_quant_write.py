"""Writing the decoder cache in 8 bits, tokens as a layer makes them and revisited ones, against a plain
64-bit form: types, codes, head layouts, odd sizes, blocks, rows that are not finite, bad data.
What a call does not write is compared byte for byte with what was there."""
import numpy as np
import pytest
import torch

import paper_2606_26631_amd as prcr
from gpu_util import DEV, to_dev
from quant_ref import CODES, TYPES, Store, check_rows, quantised32, turned

pytestmark = pytest.mark.gpu

ROPES = {64: [(64, (8, 12, 12), False, 1e6), (64, (11, 11, 10), True, 1e6), (64, (32, 0, 0), False, 1e4)],
         128: [(128, (16, 24, 24), False, 1e6), (128, (22, 21, 21), True, 5e6), (128, (24, 20, 20), True, 5e6),
               (128, (64, 0, 0), False, 1e6)]}


def error():
    return torch.zeros(1, dtype=torch.int32, device=DEV)


class Tokens:
    def __init__(self, dtype, D, H, S, n, start, seed=0, far=5000):
        g = torch.Generator().manual_seed(seed)
        rng = np.random.default_rng(seed)
        B = len(n)
        rnd = lambda: (torch.randn((B, S, H, D), generator=g) *
                       torch.exp(2 * torch.randn((B, S, H, 1), generator=g))).to(TYPES[dtype])
        self.k, self.v, self.dtype = rnd(), rnd(), TYPES[dtype]
        self.pos = rng.integers(0, far, (B, S, 3)).astype(np.int32)
        self.n, self.start = np.asarray(n, np.int32), np.asarray(start, np.int32)

    def append(self, rope, cache, layer, **kw):
        prcr.quant_append(rope, cache, layer, self.k.to(DEV), self.v.to(DEV), to_dev(self.pos), to_dev(self.n),
                          to_dev(self.start), **kw)
        torch.cuda.synchronize()

    def check(self, rope, store, got, layer, skip=()):
        """The written rows, and that nothing else is written; skip: (b, s) that must not be."""
        B, S = self.pos.shape[:2]
        for b in range(B):
            s = np.array([i for i in range(min(max(int(self.n[b]), 0), S)) if (b, i) not in skip], np.int64)
            slots = self.start[b] + s
            y = turned(rope, self.k[b, s].double().numpy(), self.pos[b, s])
            for name, want in (("k", y), ("v", self.v[b, s].double().numpy())):
                codes, scales = got.rows(name, b, slots)
                check_rows(codes[:, layer], scales[:, layer], want, self.dtype, got.kind, (name, b))
            got.clear(b, slots, [layer])
        assert got.untouched(), "other rows were written"


SIZES = {
    # name: (H, S, tokens per sequence, first slots, capacity)
    "token": (2, 1, [1], [299], 300),
    "step": (4, 1, [1, 1, 0, 1, 1], [0, 17, 3, 31, 8], 40),
    "prompts": (8, 37, [37, 0, 21], [0, 5, 64], 96),
    "odd": (3, 50, [49, 50, 1, 13], [3, 11, 0, 50], 66),
    "one head": (1, 9, [9, 4], [0, 1], 12),
    "wide": (13, 6, [5, 6], [7, 2], 20),
}


@pytest.mark.parametrize("block", [0, 16, 5, 1])
@pytest.mark.parametrize("kind", sorted(CODES))
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("size", sorted(SIZES))
def test_append(size, dtype, D, kind, block):
    H, S, n, start, cap = SIZES[size]
    print(f"append {size} {dtype} D={D} {kind} block={block}", flush=True)
    x = Tokens(dtype, D, H, S, n, start, seed=len(size) + D + block)
    rope = prcr.Rope(*ROPES[D][(block + len(size)) % len(ROPES[D])])
    store = Store(CODES[kind], len(n), 2, H, D, cap, block, seed=3)
    cache, err = store.to(DEV), error()
    x.append(rope, cache, 1, err=err)
    assert int(err.item()) == 0
    x.check(rope, store, store.take(cache), 1)


@pytest.mark.parametrize("kind", sorted(CODES))
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_tokens(dtype, kind):
    """More tokens than one round of workgroups over the chip takes, at far positions."""
    print(f"append many {dtype} {kind}", flush=True)
    x = Tokens(dtype, 128, 2, 1500, [1500, 1377, 1500, 900], [0, 100, 13, 7], seed=2, far=2 ** 31 - 1)
    rope = prcr.Rope(*ROPES[128][2])
    store = Store(CODES[kind], 4, 1, 2, 128, 1600)
    cache, err = store.to(DEV), error()
    x.append(rope, cache, 0, err=err)
    assert int(err.item()) == 0
    x.check(rope, store, store.take(cache), 0)


def edge_rows(dtype, D):
    """Rows where the format is at its edges: zeros, the smallest numbers, infinities, NaN, rows of one large
    element, halves of a code's step, every bf16 magnitude; and ordinary ones in number."""
    rng = np.random.default_rng(5)
    rows = [np.zeros(D), np.full(D, -0.0), np.full(D, 2.0 ** -149), np.full(D, 1e-38), np.full(D, 3.3e38)]
    for value in (np.inf, -np.inf, np.nan):
        for at in (0, 1, D // 2 - 1, D // 2, D - 1):
            r = rng.standard_normal(D)
            r[at] = value
            rows.append(r)
    for most in (448.0, 127.0, 1.0, 2.0 ** -120, 2.0 ** 100):
        r = rng.standard_normal(D) * most / 50
        r[rng.integers(D)] = most
        rows.append(r)
    for q in (448.0, 127.0):                  # multiples of half a step: ties
        for first in (0.0, 16.0, 60.0):
            r = first + np.arange(D) * 0.5
            r[1::2] *= -1
            r[3] = q
            rows.append(r)
        r = np.ldexp(rng.integers(8, 32, D) * 0.5, rng.integers(-14, 4, D))
        r[-1] = q
        rows.append(r)
    bits = np.arange(0x7F80, dtype=np.uint32)  # every finite bf16 magnitude, D to a row, largest of each row its last
    rows += list((bits[:len(bits) // D * D] << 16).view(np.float32).reshape(-1, D).astype(np.float64))
    rows += list(rng.standard_normal((4000, D)) * np.exp(rng.standard_normal((4000, 1))))
    with np.errstate(over="ignore"):
        x = torch.from_numpy(np.array(rows, np.float32)).to(TYPES[dtype])
    return x


@pytest.mark.parametrize("kind", sorted(CODES))
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("f32", 128), ("bf16", 64), ("f32", 64)])
def test_codes_are_those_of_the_format(dtype, D, kind):
    """Values, and keys at position 0 (not turned), bit for bit as the format's float32 arithmetic gives them."""
    print(f"codes {dtype} D={D} {kind}", flush=True)
    x = edge_rows(dtype, D)
    n = len(x)
    rope = prcr.Rope(*ROPES[D][0])
    store = Store(CODES[kind], 1, 1, 1, D, n)
    cache, err = store.to(DEV), error()
    raw = x.view(1, n, 1, D).to(DEV)
    prcr.quant_append(rope, cache, 0, raw, raw, torch.zeros(1, n, 3, dtype=torch.int32, device=DEV),
                      to_dev(np.array([n], np.int32)), to_dev(np.array([0], np.int32)), err=err)
    torch.cuda.synchronize()
    code, scale = quantised32(x.float().numpy(), CODES[kind])
    got = store.take(cache)
    # (A pair with an infinity or a NaN spoils its partner in a turned row as well: the row is one without values.)
    for name in ("k", "v"):
        c, s = got.rows(name, 0, np.arange(n))
        s = s[:, 0, 0]
        assert np.array_equal(np.isnan(s), np.isnan(scale)), name
        fine = ~np.isnan(scale)
        assert np.array_equal(s[fine].view(np.int32), scale[fine].view(np.int32)), name
        assert np.array_equal(c[:, 0, 0], code), (name, np.argwhere(c[:, 0, 0] != code)[:5])
    assert int(err.item()) == 0
    # What is read back is NaN in those rows alone.
    k, v = prcr.quant_read(cache, 0, to_dev(np.array([n], np.int32)), torch.float32)
    assert np.array_equal(v[0, 0, 0].isnan().all(-1).cpu().numpy(), np.isnan(scale))
    assert np.array_equal(v[0, 0, 0].isnan().any(-1).cpu().numpy(), np.isnan(scale))


@pytest.mark.parametrize("block", [0, 16])
def test_append_bad_data(block):
    print(f"append bad data, block={block}", flush=True)
    H, D = 2, 64
    rope = prcr.Rope(*ROPES[D][0])
    # Counts outside the rows: none, and all of them.
    x = Tokens("bf16", D, H, 6, [-3, 9, 2], [0, 1, 2], seed=1)
    store = Store(torch.int8, 3, 2, H, D, 16, block)
    cache, err = store.to(DEV), error()
    x.append(rope, cache, 0, err=err)
    assert int(err.item()) == prcr.DERR_INDEX
    x.check(rope, store, store.take(cache), 0)
    # Slots before the first and behind the last.
    x = Tokens("bf16", D, H, 6, [6, 6, 6], [-2, 13, 2 ** 31 - 4], seed=2)
    cache, err = store.to(DEV), error()
    x.append(rope, cache, 1, err=err)
    assert int(err.item()) == prcr.DERR_CAPACITY
    x.check(rope, store, store.take(cache), 1,
            skip={(0, 0), (0, 1)} | {(1, s) for s in range(3, 6)} | {(2, s) for s in range(6)})
    if block:
        store.table[1, 0], store.table[2, 0] = -1, store.k.shape[1]
        x = Tokens("bf16", D, H, 6, [6, 6, 6], [0, 0, 0], seed=3)
        cache, err = store.to(DEV), error()
        x.append(rope, cache, 1, err=err)
        assert int(err.item()) == prcr.DERR_BLOCK
        x.check(rope, store, store.take(cache), 1, skip={(b, s) for b in (1, 2) for s in range(6)})
    # Without a flag to report to, nothing else changes.
    x = Tokens("f32", D, H, 6, [9, 6, 6], [-2, 13, 0], seed=4)
    store = Store(torch.int8, 3, 2, H, D, 16, block)
    cache = store.to(DEV)
    x.append(rope, cache, 0)
    x.check(rope, store, store.take(cache), 0, skip={(0, 0), (0, 1)} | {(1, s) for s in range(3, 6)})


class Revisit:
    def __init__(self, dtype, D, NL, H, M, picks, lens, seed=0, key_only=False):
        g = torch.Generator().manual_seed(seed)
        rng = np.random.default_rng(seed)
        B = len(picks)
        rnd = lambda: torch.randn((B, M, NL, H, D), generator=g).to(TYPES[dtype])
        self.k, self.v, self.dtype, self.NL = rnd(), None if key_only else rnd(), TYPES[dtype], NL
        # (slots of the sequence's own, below its length)
        self.v_slot = np.stack([rng.integers(0, max(int(n), 1), M) for n in lens]).astype(np.int32)
        self.picks, self.lens = [np.asarray(p, np.int32) for p in picks], np.asarray(lens, np.int32)
        self.off = np.concatenate([[0], np.cumsum([len(p) for p in picks])]).astype(np.int32)
        self.idx = np.concatenate(self.picks).astype(np.int32)
        self.pos = rng.uniform(0, 3000, (len(self.idx), 3))
        self.n_visual = np.full(B, M, np.int32)
        self.coords = np.zeros((B, M, 3), np.int32)

    def memory(self):
        return prcr.Memory(self.k.to(DEV), None if self.v is None else self.v.to(DEV), to_dev(self.coords),
                           to_dev(self.n_visual), None if self.v is not None else to_dev(self.v_slot))

    def run(self, rope, cache, **kw):
        out = prcr.quant_rebind_inject(rope, self.memory(), to_dev(self.off), to_dev(self.idx), to_dev(self.pos), cache,
                                       to_dev(self.lens), **kw)
        torch.cuda.synchronize()
        return [t.cpu().numpy() for t in out]

    def check(self, rope, store, got, new_len, slots, before=None, skip=()):
        assert np.array_equal(new_len, self.lens + np.diff(self.off))
        for b, pick in enumerate(self.picks):
            j = np.array([i for i in range(len(pick)) if (b, i) not in skip], np.int64)
            t = self.off[b] + j
            at = self.lens[b] + j
            i0, i1 = got.at(b, at)
            assert np.array_equal(slots[t], i0 * got.block + i1 if got.block else b * got.cap + at)
            y = turned(rope, self.k[b, pick[j]].double().numpy(), self.pos[t])
            codes, scales = got.rows("k", b, at)
            check_rows(codes, scales, y, self.dtype, got.kind, ("k", b))
            codes, scales = got.rows("v", b, at)
            if self.v is not None:
                check_rows(codes, scales, self.v[b, pick[j]].double().numpy(), self.dtype, got.kind, ("v", b))
            else:
                c, s = before.rows("v", b, self.v_slot[b, pick[j]])
                assert np.array_equal(codes, c) and np.array_equal(scales, s)
        for b, i in skip:
            assert slots[self.off[b] + i] == -1
        # Nothing else: put back what was there.
        for b, pick in enumerate(self.picks):
            j = np.array([i for i in range(len(pick)) if (b, i) not in skip], np.int64)
            got.clear(b, self.lens[b] + j, range(self.NL))
            if before is not None:
                before.clear(b, self.lens[b] + j, range(self.NL))
        if before is None:
            assert got.untouched()
        else:
            for name in ("k", "v"):
                assert torch.equal(getattr(got, name).view(torch.uint8), getattr(before, name).view(torch.uint8))
                assert torch.equal(getattr(got, name + "_scale"), getattr(before, name + "_scale"))


def picks_of(counts, M, seed):
    rng = np.random.default_rng(seed)
    return [rng.permutation(M)[:n] for n in counts]


@pytest.mark.parametrize("key_only", [False, True], ids=["values", "key_only"])
@pytest.mark.parametrize("block", [0, 16, 5])
@pytest.mark.parametrize("kind", sorted(CODES))
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("NL,H,counts", [(3, 4, [9, 0, 17]), (11, 1, [1]), (2, 7, [5, 33, 8, 0, 2])])
def test_rebind(NL, H, counts, dtype, D, kind, block, key_only):
    print(f"rebind {NL}x{H} {counts} {dtype} D={D} {kind} block={block} key_only={key_only}", flush=True)
    B, M = len(counts), 40
    x = Revisit(dtype, D, NL, H, M, picks_of(counts, M, 7), np.arange(B) * 3 + 41, seed=D + block, key_only=key_only)
    rope = prcr.Rope(*ROPES[D][(block + NL) % len(ROPES[D])])
    store = Store(CODES[kind], B, NL, H, D, 96, block, seed=4)
    if key_only:
        store.fill(seed=9)
    cache, err = store.to(DEV), error()
    new_len, slots = x.run(rope, cache, err=err)
    assert int(err.item()) == 0
    x.check(rope, store, store.take(cache), new_len, slots, store if key_only else None)


def test_rebind_of_many_sequences_and_the_same_token_twice():
    print("rebind many sequences", flush=True)
    counts = [(7 * i) % 5 for i in range(150)]
    x = Revisit("bf16", 64, 2, 2, 12, picks_of(counts, 12, 1), np.arange(150) % 9, seed=3)
    x.picks[3][:] = x.picks[3][0] if len(x.picks[3]) else 0
    x.idx = np.concatenate(x.picks).astype(np.int32)
    rope = prcr.Rope(*ROPES[64][1])
    store = Store(torch.int8, 150, 2, 2, 64, 16)
    cache, err = store.to(DEV), error()
    new_len, slots = x.run(rope, cache, err=err)
    assert int(err.item()) == 0
    x.check(rope, store, store.take(cache), new_len, slots)


def test_rebind_of_nothing_writes_the_lengths():
    x = Revisit("bf16", 128, 2, 2, 5, [[], []], [4, 6])
    store = Store(torch.float8_e4m3fn, 2, 2, 2, 128, 16)
    cache = store.to(DEV)
    new_len, slots = x.run(prcr.Rope(*ROPES[128][0]), cache)
    assert new_len.tolist() == [4, 6] and len(slots) == 0 and store.take(cache).untouched()


@pytest.mark.parametrize("block", [0, 16])
def test_rebind_bad_data(block):
    print(f"rebind bad data, block={block}", flush=True)
    rope = prcr.Rope(*ROPES[64][0])

    def case(change, want, skip, key_only=False, cap=32):
        x = Revisit("bf16", 64, 2, 3, 10, picks_of([4, 3, 5], 10, 2), [12, 20, 14], seed=5, key_only=key_only)
        x.v_slot %= 12
        store = Store(torch.float8_e4m3fn, 3, 2, 3, 64, cap, block)
        if key_only:
            store.fill(seed=2)
        change(x, store)
        cache, err = store.to(DEV), error()
        new_len, slots = x.run(rope, cache, err=err)
        assert int(err.item()) == want, int(err.item())
        before = store if key_only else None
        x.check(rope, store, store.take(cache), new_len, slots, before, skip)

    def index(x, store):
        x.picks[0][1], x.picks[1][0], x.picks[2][4] = -1, 10, 7
        x.idx = np.concatenate(x.picks).astype(np.int32)
        x.n_visual[2] = 7

    hidden = {(0, 1), (1, 0)}
    y = picks_of([4, 3, 5], 10, 2)
    y[2][4] = 7
    case(index, prcr.DERR_INDEX, hidden | {(2, i) for i in range(5) if y[2][i] >= 7})

    def capacity(x, store):
        x.lens[:] = [30, -2, 31]
    case(capacity, prcr.DERR_CAPACITY, {(0, 2), (0, 3), (1, 0), (1, 1), (2, 1), (2, 2), (2, 3), (2, 4)})

    def v_slot(x, store):
        x.v_slot[0, x.picks[0][2]], x.v_slot[2, x.picks[2][0]] = -1, 14
    case(v_slot, prcr.DERR_INDEX, {(0, 2), (2, 0)}, key_only=True)
    if block:
        def table(x, store):
            store.table[0, 0], store.table[1, 1] = -1, store.k.shape[1]
        case(table, prcr.DERR_BLOCK, {(0, i) for i in range(4)} | {(1, i) for i in range(3)})

    # Offsets that do not belong to the selection.
    x = Revisit("bf16", 64, 2, 3, 10, picks_of([4, 3, 5], 10, 2), [12, 20, 14], seed=5)
    store = Store(torch.float8_e4m3fn, 3, 2, 3, 64, 32, block)
    for off in ([0, 4, 7, 13], [2, 4, 7, 12], [0, 4, 2, 12], [-1, 4, 7, 12]):
        x.off = np.array(off, np.int32)
        cache, err = store.to(DEV), error()
        x.run(rope, cache, err=err)
        assert int(err.item()) == prcr.DERR_OFFSETS


def test_a_row_revisited_where_it_was_appended_has_the_same_codes():
    print("append and revisit agree", flush=True)
    for dtype in ("bf16", "f32"):
        x = Tokens(dtype, 128, 3, 20, [20], [0], seed=6)
        rope = prcr.Rope(*ROPES[128][2])
        store = Store(torch.float8_e4m3fn, 1, 1, 3, 128, 64)
        cache = store.to(DEV)
        x.append(rope, cache, 0)
        mem = prcr.Memory(x.k.view(1, 20, 1, 3, 128).to(DEV), x.v.view(1, 20, 1, 3, 128).to(DEV),
                          torch.zeros(1, 20, 3, dtype=torch.int32, device=DEV), to_dev(np.array([20], np.int32)))
        prcr.quant_rebind_inject(rope, mem, to_dev(np.array([0, 20], np.int32)), to_dev(np.arange(20, dtype=np.int32)),
                                 to_dev(x.pos[0].astype(np.float64)), cache, to_dev(np.array([20], np.int32)))
        torch.cuda.synchronize()
        for t in (cache.k.view(torch.uint8), cache.v.view(torch.uint8), cache.k_scale, cache.v_scale):
            assert torch.equal(t[:, :, :, :20], t[:, :, :, 20:40])


@pytest.mark.parametrize("kind", sorted(CODES))
def test_the_largest_numbers(kind):
    """Rows whose largest magnitude is among the type's last 64: codes and scales bit for bit, and read back finite but
    for int8's largest float32, whose 127 scale rounds to an infinity."""
    print(f"the largest numbers {kind}", flush=True)
    D = 128
    x = np.tile(np.linspace(-1, 1, D, dtype=np.float32), (64, 1))
    x[:, 5] = np.arange(0x7F7FFFFF - 63, 0x7F800000, dtype=np.uint32).view(np.float32)
    store = Store(CODES[kind], 1, 1, 1, D, 64)
    cache, err = store.to(DEV), error()
    raw = torch.from_numpy(x).view(1, 64, 1, D).to(DEV)
    length = to_dev(np.array([64], np.int32))
    prcr.quant_append(prcr.Rope(*ROPES[D][0]), cache, 0, raw, raw, torch.zeros(1, 64, 3, dtype=torch.int32, device=DEV), length,
                      to_dev(np.array([0], np.int32)), err=err)
    k, v = prcr.quant_read(cache, 0, length, torch.float32)
    code, scale = quantised32(x, CODES[kind])
    got = store.take(cache)
    for name, t in (("k", k), ("v", v)):
        c, s = got.rows(name, 0, np.arange(64))
        assert np.array_equal(s[:, 0, 0].view(np.int32), scale.view(np.int32)) and np.array_equal(c[:, 0, 0], code)
        finite = t[0, 0, 0].isfinite().cpu().numpy()
        assert finite[:63].all() and np.array_equal(~finite[63], (np.arange(D) == 5) & (kind == "i8"))
    assert int(err.item()) == 0
