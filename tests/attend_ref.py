"""Plain 64-bit forms of the operators on several tokens per sequence, for the tests: chunk
attention, the keys' weights and eviction, one sequence and head at a time, with the bounds
their tolerances are made of."""
import numpy as np
import torch

BF16_HALF = 2.0 ** -8          # a rounding to bf16 is off by at most this, relative to the value
F32_HALF = 2.0 ** -24


def bf16_nearest(y):
    """float64 to the nearest bf16 value, ties to even."""
    m, e = np.frexp(y)
    return np.ldexp(np.rint(np.ldexp(m, 8)), e - 8)


def rotate(rope, q, pos, dtype):
    """Rows q [T, Hq, D] at pos [T, 3], rotated in double and rounded once to the stored type."""
    q = q.double().cpu().numpy()
    P = rope.head_dim // 2
    ang = np.asarray(pos, np.float64)[:, rope.pair_axis()] * np.asarray(rope.inv_freq())
    c, s = np.cos(ang)[:, None, :], np.sin(ang)[:, None, :]
    lo, hi = q[..., :P], q[..., P:]
    y = np.concatenate([lo * c - hi * s, hi * c + lo * s], axis=-1)
    return bf16_nearest(y) if dtype == torch.bfloat16 else y.astype(np.float32).astype(np.float64)


class HostCache:
    """A cache's tensors on the host and where a sequence's slots are in them."""

    def __init__(self, k, v, table=None, layer=0):
        self.k, self.v, self.table, self.layer = k.cpu(), v.cpu(), table, layer

    def at(self, b, slots):
        """(tensor index of the slots' rows [n, H, D], which of them are in the pool)."""
        slots = np.asarray(slots)
        if self.table is None:
            return slots, np.ones(len(slots), bool)
        bs = self.k.shape[2]
        blk = self.table[b, slots // bs]
        ok = (blk >= 0) & (blk < self.k.shape[1])
        return (np.where(ok, blk, 0), slots % bs), ok

    def rows(self, x, b, n):
        """Slots 0..n-1 of sequence b as [n, H, D] float64, and which of them exist."""
        at, ok = self.at(b, np.arange(n))
        if self.table is None:
            r = x[b, self.layer, :, :n].transpose(0, 1)
        else:
            r = x[self.layer][torch.from_numpy(at[0].astype(np.int64)), torch.from_numpy(at[1].astype(np.int64))]
        return r.double().numpy(), ok

    def capacity(self):
        return self.k.shape[3] if self.table is None else self.table.shape[1] * self.k.shape[2]


def spans(q_off, q_len, B):
    return [(int(q_off[b]), int(q_off[b + 1] - q_off[b] if q_len is None else q_len[b])) for b in range(B)]


def scores(rope, cache, q, pos, rows, lens, scale, dtype):
    """For each (b, h, g): scaled scores [n, len] with -inf at what a row does not see, and a
    bound of a float32 computation's error in them: D + 2 roundings of sums of the products'
    magnitudes (the rotation's own among them), and the scale's of the score."""
    rq = rotate(rope, q, pos, dtype)
    H = cache.k.shape[2 if cache.table is None else 3]
    G = rq.shape[1] // H
    for b, (r0, n) in enumerate(rows):
        L = int(lens[b])
        k, ok = cache.rows(cache.k, b, L)
        sees = (np.arange(L)[None, :] <= (L - n + np.arange(n))[:, None]) & ok[None, :]
        for h in range(H):
            for g in range(G):
                x = rq[r0:r0 + n, h * G + g]
                kk = np.where(ok[:, None], k[:, h], 0.0)
                with np.errstate(invalid="ignore", over="ignore"):
                    s = x @ kk.T * scale
                    mag = np.abs(np.nan_to_num(x)) @ np.abs(np.nan_to_num(kk)).T * abs(scale)
                bound = (rope.head_dim + 2) * F32_HALF * mag + 4 * F32_HALF * np.abs(np.nan_to_num(s))
                yield b, h, g, r0, np.where(sees, s, -np.inf), np.where(sees, bound, 0.0), sees


def attention(rope, cache, q, pos, rows, lens, scale, dtype):
    """(out, lse, bounds of both, which rows are a sequence's): [T, Hq, D] and [T, Hq] each, [T].

    Bound of out: a weight's relative error is at most that of its exponent's, twice (the sum in
    the denominator has it too), plus a few float32 roundings and n in the sums; bf16 weights
    are rounded once more, as is the result.  All of them times sum p |v|."""
    T, Hq = q.shape[0], q.shape[1]
    D = rope.head_dim
    out, lse = np.full((T, Hq, D), np.nan), np.full((T, Hq), np.nan)
    b_out, b_lse = np.zeros((T, Hq, D)), np.zeros((T, Hq))
    half = BF16_HALF if dtype == torch.bfloat16 else 0.0
    last = BF16_HALF if dtype == torch.bfloat16 else F32_HALF
    values, mine = {}, np.zeros(T, bool)
    for b, h, g, r0, s, err, sees in scores(rope, cache, q, pos, rows, lens, scale, dtype):
        n, L = s.shape
        if n == 0:
            continue
        mine[r0:r0 + n] = True
        H = cache.k.shape[2 if cache.table is None else 3]
        qh = h * (Hq // H) + g
        if b not in values:
            values[b] = cache.rows(cache.v, b, L)[0]
        any_seen = sees.any(1)
        m = np.where(any_seen, np.max(s, axis=1, initial=-np.inf), 0.0)
        with np.errstate(invalid="ignore", over="ignore"):
            e = np.where(sees, np.exp(s - m[:, None]), 0.0)
        l = e.sum(1)
        p = e / np.where(l == 0, 1, l)[:, None]
        v = values[b][:, h]
        for i in range(n):                   # (a hidden value must not matter, whatever it is)
            vis = sees[i]
            with np.errstate(invalid="ignore"):
                out[r0 + i, qh] = p[i, vis] @ v[vis] if vis.any() else 0.0
                pv = p[i, vis] @ np.abs(np.nan_to_num(v[vis], nan=0, posinf=0, neginf=0))
            d = err[i].max(initial=0.0)
            sums = (vis.sum() + 8) * F32_HALF
            b_out[r0 + i, qh] = (2 * d + 2 * sums + half) * pv * 1.01 + last * np.abs(np.nan_to_num(out[r0 + i, qh])) + 1e-30
            lse[r0 + i, qh] = np.log(l[i]) + m[i] if vis.any() else -np.inf
            b_lse[r0 + i, qh] = d + sums + 8 * F32_HALF * (1 + abs(np.nan_to_num(lse[r0 + i, qh], neginf=0)) + abs(m[i]))
    return out, lse, b_out, b_lse, mine


def key_weights(rope, cache, q, pos, rows, lens, scale, dtype, lse, window=None):
    """weights [B, H, capacity] and their bounds, given lse [T, Hq] (float32)."""
    B = len(rows)
    H = cache.k.shape[2 if cache.table is None else 3]
    w, bound = np.zeros((B, H, cache.capacity())), np.zeros((B, H, cache.capacity()))
    if window is not None:
        rows = [(r0 + max(0, n - window), min(n, window)) for r0, n in rows]
    for b, h, g, r0, s, err, sees in scores(rope, cache, q, pos, rows, lens, scale, dtype):
        n, L = s.shape
        at = lse[r0:r0 + n, h * (q.shape[1] // H) + g].astype(np.float64)[:, None]
        with np.errstate(invalid="ignore", over="ignore"):
            e = np.where(sees, np.exp(s - at), 0.0)
        off = err + 8 * F32_HALF * (1 + np.abs(np.nan_to_num(at, neginf=0)) + np.abs(np.where(np.isfinite(s), s, 0)))
        w[b, h, :L] += e.sum(0)
        bound[b, h, :L] += (np.nan_to_num(e) * (off + 32 * F32_HALF)).sum(0)
    return w, bound + 2 * F32_HALF * np.abs(np.nan_to_num(w)) + 1e-37


def evict(w, lens, budget, first, last):
    """Kept slots of each sequence, as lists."""
    kept = []
    for b, n in enumerate(lens):
        n = int(n)
        if n <= budget:
            kept.append(list(range(n)))
            continue
        score = w[b, :, :n].astype(np.float64).sum(0)
        with np.errstate(over="ignore"):
            score = score.astype(np.float32)
        rank = sorted(range(first, n - last),
                      key=lambda j: (1, 0.0, j) if np.isnan(score[j]) else (0, -float(score[j]), j))
        kept.append(sorted(list(range(first)) + rank[:budget - first - last] + list(range(n - last, n))))
    return kept
