"""Plain 64-bit forms of the decoder cache in 8 bits, for the tests, on the host: a row's codes and
scale with the bounds that float32 arithmetic leaves them, the cache's layouts, and attention over
what it stands for."""
import numpy as np
import torch

from attend_ref import F32_HALF, bf16_nearest

LARGEST = {torch.float8_e4m3fn: 448.0, torch.int8: 127.0}
CODES = {"e4m3": torch.float8_e4m3fn, "i8": torch.int8}
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
FILL = 0x55                                  # what a cache holds before a test writes to it
FILL_SCALE = -7.0


def turned(rope, x, pos):
    """Rows x [n, ..., D] (float64) at pos [n, 3], in float64."""
    P = rope.head_dim // 2
    ang = np.asarray(pos, np.float64)[:, rope.pair_axis()] * np.asarray(rope.inv_freq())
    ang = ang.reshape(len(ang), *[1] * (x.ndim - 2), P)
    c, s = np.cos(ang), np.sin(ang)
    lo, hi = x[..., :P], x[..., P:]
    return np.concatenate([lo * c - hi * s, hi * c + lo * s], axis=-1)


def nearest_code(y, kind):
    """float64 to the nearest code's value, ties to even."""
    if kind == torch.int8:
        return np.rint(y)
    _, e = np.frexp(y)
    step = np.ldexp(1.0, np.maximum(e - 1, -6) - 3)
    return np.rint(y / step) * step


def quantised32(x, kind):
    """Codes and scales of float32 rows exactly as the format says, in float32."""
    x = x.astype(np.float32)
    with np.errstate(invalid="ignore", over="ignore"):
        most = np.abs(x).max(-1)
        scale = np.maximum(most / np.float32(LARGEST[kind]), np.float32(2.0 ** -126))
        y = x * (np.float32(1) / scale)[..., None]
        code = nearest_code(y.astype(np.float64), kind)
    bad = ~np.isfinite(x).all(-1)
    return np.where(bad[..., None], 0.0, code), np.where(bad, np.float32(np.nan), scale)


def check_rows(codes, scales, y, dtype, kind, what=""):
    """Codes and scales [..., D], [...] of rows whose values before any rounding are y (float64).

    In float32: a float32 row's own rounding (half a unit, 2^-24), the scale's, its inverse's and
    the product's each 2^-24 relative, so that a code is the nearest of a number within 2^-21 of
    x / scale, and the scale within 2^-23 of it.  bf16 rows are rounded to bf16 first, exactly."""
    x = bf16_nearest(y) if dtype == torch.bfloat16 else y
    s = np.maximum(np.abs(x).max(-1) / LARGEST[kind], 2.0 ** -126)
    off = np.abs(scales.astype(np.float64) - s) / s
    assert off.max(initial=0) <= 2.0 ** -23 * (1 + 2.0 ** -20), (what, "scale", off.max())
    v = x / s[..., None]
    if kind == torch.int8:
        half = np.full(v.shape, 0.5)
    else:
        _, e = np.frexp(v)
        half = np.ldexp(0.5, np.maximum(e - 1, -6) - 3)
    d = np.abs(codes - v) - half - np.abs(v) * 2.0 ** -21
    assert d.max(initial=-1) <= 0, (what, "code", np.unravel_index(d.argmax(), d.shape), d.max())


class Store:
    """A cache in 8 bits on the host, and where its rows are."""

    def __init__(self, kind, B, NL, H, D, cap, block=0, seed=0, spare=2):
        self.kind, self.shape, self.cap, self.block, self.table = kind, (B, NL, H, D), cap, block, None
        if block:
            per = -(-cap // block)
            self.cap = per * block
            n = B * per + spare
            self.table = np.random.default_rng(seed).permutation(n)[:B * per].astype(np.int32).reshape(B, per)
            rows = (NL, n, block, H, D)
            scales = (NL, n, H, block)
        else:
            rows, scales = (B, NL, H, cap, D), (B, NL, H, cap)
        self.k, self.v = (torch.full(rows, FILL, dtype=torch.uint8).view(kind) for _ in range(2))
        self.k_scale, self.v_scale = (torch.full(scales, FILL_SCALE) for _ in range(2))

    def fill(self, dtype=torch.float32, seed=0, spread=1.0):
        """Random quantised rows everywhere; codes and scales as a cache has them in use."""
        g = torch.Generator().manual_seed(seed)
        for name in ("k", "v"):
            shape = getattr(self, name).shape
            x = (torch.randn(shape, generator=g) * torch.exp(spread * torch.randn(shape[:-1], generator=g))[..., None])
            code, scale = quantised32(x.to(dtype).float().numpy(), self.kind)
            scale = torch.from_numpy(scale)
            setattr(self, name, torch.from_numpy(code).to(self.kind))
            setattr(self, name + "_scale", (scale.transpose(2, 3) if self.block else scale).contiguous())
        return self

    def to(self, device):
        import paper_2606_26631_amd as prcr
        return prcr.QuantCache(*(t.clone().to(device) for t in (self.k, self.v, self.k_scale, self.v_scale)),
                               None if self.table is None else torch.from_numpy(self.table).to(device))

    def take(self, cache):
        """A copy of this store that holds a device cache's tensors."""
        import copy
        s = copy.copy(self)
        s.k, s.v, s.k_scale, s.v_scale = (t.cpu().clone() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale))
        return s

    def at(self, b, slots):
        """Index of the slots' rows in views of [slot, layer, head]: see rows()."""
        slots = np.asarray(slots, np.int64)
        if not self.block:
            return b, slots
        return self.table[b, slots // self.block].astype(np.int64), slots % self.block

    def rows(self, name, b, slots):
        """(codes [n, NL, H, D], scales [n, NL, H]) of a sequence's slots, as float64."""
        i, j = self.at(b, slots)
        codes, scales = getattr(self, name), getattr(self, name + "_scale")
        if self.block:
            c = codes.view(torch.uint8)[:, torch.from_numpy(i), torch.from_numpy(j)].view(self.kind).transpose(0, 1)
            s = scales.transpose(2, 3)[:, torch.from_numpy(i), torch.from_numpy(j)].transpose(0, 1)
        else:
            c = codes.view(torch.uint8)[i][:, :, torch.from_numpy(j)].view(self.kind).permute(2, 0, 1, 3)
            s = scales[i][:, :, torch.from_numpy(j)].permute(2, 0, 1)
        return c.double().numpy(), s.numpy()

    def clear(self, b, slots, layers):
        """Sets the slots' rows back to what an unwritten cache holds."""
        i, j = self.at(b, slots)
        for name in ("k", "v"):
            codes, scales = getattr(self, name).view(torch.uint8), getattr(self, name + "_scale")
            for l in layers:
                if self.block:
                    codes[l][torch.from_numpy(i), torch.from_numpy(j)] = FILL
                    scales[l].transpose(1, 2)[torch.from_numpy(i), torch.from_numpy(j)] = FILL_SCALE
                else:
                    codes[i, l][:, torch.from_numpy(j)] = FILL
                    scales[i, l][:, torch.from_numpy(j)] = FILL_SCALE

    def untouched(self):
        """Whether nothing but FILL is in it."""
        return all(bool((t.view(torch.uint8) == FILL).all()) for t in (self.k, self.v)) and \
            all(bool((t == FILL_SCALE).all()) for t in (self.k_scale, self.v_scale))


def attention(rope, store, layer, q, q_pos, lens, scale, skip=()):
    """(out [B, Hq, D], bound) of one query row a sequence over the rows that the cache stands for;
    skip: table entries (b, block) outside the pool.

    Scores in float32: D + 8 roundings of sums of the products' magnitudes, the scales' of the score;
    a weight's relative error is its score's, twice (the denominator's too), and a few roundings
    for each of the n terms of the sums."""
    B, Hq, D = q.shape
    H = store.shape[2]
    G = Hq // H
    out, bound = np.zeros((B, Hq, D)), np.zeros((B, Hq, D))
    rq = turned(rope, q.double().numpy(), np.repeat(np.asarray(q_pos)[:, None], 3, 1))
    for b in range(B):
        slots = np.arange(min(max(int(lens[b]), 0), store.cap))
        if store.block:
            slots = np.array([s for s in slots if (b, s // store.block) not in skip], np.int64)
        if not len(slots):
            continue
        kc, ks = store.rows("k", b, slots)
        vc, vs = store.rows("v", b, slots)
        for h in range(H):
            k = kc[:, layer, h] * ks[:, layer, h].astype(np.float64)[:, None]
            v = vc[:, layer, h] * vs[:, layer, h].astype(np.float64)[:, None]
            for g in range(G):
                x = rq[b, h * G + g]
                s = k @ x * scale
                mag = np.abs(k) @ np.abs(x) * abs(scale)
                err = ((D + 8) * mag + 8 * np.abs(s)) * F32_HALF
                e = np.exp(s - s.max())
                p = e / e.sum()
                o = p @ v
                d = err.max()
                out[b, h * G + g] = o
                bound[b, h * G + g] = ((2 * d + (2 * len(slots) + 32) * F32_HALF) * 1.01 * (p @ np.abs(v)) +
                                       2 * F32_HALF * np.abs(o) + 1e-30)
    return out, bound


def check_attention(out, want):
    o, bound = want
    out = out.cpu().numpy().astype(np.float64)
    assert np.array_equal(np.isnan(out), np.isnan(o)), "other elements are NaN"
    d = np.abs(np.nan_to_num(out - o)) - np.nan_to_num(bound)
    assert d.max(initial=-1) <= 0, (np.unravel_index(d.argmax(), d.shape), d.max())
