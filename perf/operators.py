"""Attention of several new tokens over the active cache, the weight each cached key gets from
it, and eviction by that weight, as cases that can be timed and compared.

A decoder attends over its cache with a whole prompt (prefill), with a user's next turn after a
revisit, or with a serving batch in which some sequences prefill a piece and others decode one
token (chunk_attention).  A program that bounds its cache adds up the weight that every cached
key received (key_weights), after each token or for the last tokens of a prompt, and now and
then keeps the slots of most weight (evict).  Shapes are those of workloads.py and bench.py:
28 layers x 4 KV heads x 7 and 36 layers x 8 KV heads x 4 query heads, head_dim 128, bf16, and a
small float32 decoder of head_dim 64.
"""
import math
import random

import numpy as np
import torch

own = False

# Rotary forms: name -> (head_dim, sections, interleaved, theta).
ROPES = {
    "d128_sections": (128, (16, 24, 24), False, 1e6),
    "d128_interleaved": (128, (22, 21, 21), True, 5e6),
    "d128_interleaved_24": (128, (24, 20, 20), True, 5e6),
    "d128_1d": (128, (64, 0, 0), False, 1e6),
    "d64_sections": (64, (8, 12, 12), False, 1e6),
    "d64_interleaved": (64, (11, 11, 10), True, 1e6),
    "d64_1d": (64, (32, 0, 0), False, 1e6),
}
# Bounds of a drawn case: the largest listed ones' scores, traffic and resident bytes.
MOST_SCORES = 32 * 12001 ** 2
MOST_FLOPS = 1.18e12
MOST_BYTES = 7.5e9
MOST_RESIDENT = 9e9


def listed():
    return [
        # The smallest call: one new token of one sequence of a two-layer float32 decoder.
        dict(name="chunk_token_f32", kind="chunk", rope="d64_sections", dtype="f32", batch=1,
             layers=2, kv_heads=2, group=2, n_lo=1, n_hi=1, past_lo=299, past_hi=299, block=0),
        # A user's next turn: 48 text tokens after 1,152 cached ones, 8B-class decoder.
        dict(name="chunk_turn", kind="chunk", rope="d128_interleaved_24", dtype="bf16", batch=1,
             layers=2, kv_heads=8, group=4, n_lo=48, n_hi=48, past_lo=1152, past_hi=1152,
             block=0),
        # A serving step: 64 sequences in a paged cache, of which some decode a token and
        # some bring a piece of up to 256.
        dict(name="chunk_mixed_paged", kind="chunk", rope="d128_sections", dtype="bf16",
             batch=64, layers=2, kv_heads=4, group=7, n_lo=1, n_hi=256, past_lo=2400,
             past_hi=6000, block=16),
        # Prefill: 8 prompts of 2,560 tokens, 2,048 of them visual.
        dict(name="prompt_batch", kind="chunk", rope="d128_interleaved", dtype="bf16", batch=8,
             layers=2, kv_heads=8, group=4, n_lo=2560, n_hi=2560, past_lo=0, past_hi=0, block=0),
        # Prefill of prompts of different lengths into a paged cache, one image each.
        dict(name="prompt_ragged_paged", kind="chunk", rope="d128_sections", dtype="bf16",
             batch=6, layers=2, kv_heads=4, group=7, n_lo=1661, n_hi=2545, past_lo=0, past_hi=0,
             block=16),
        # A long video prompt, one sequence.
        dict(name="prompt_long", kind="chunk", rope="d128_interleaved_24", dtype="bf16", batch=1,
             layers=1, kv_heads=8, group=4, n_lo=12001, n_hi=12001, past_lo=0, past_hi=0,
             block=0),
        # Prefill of the small float32 decoder: two prompts around an image.
        dict(name="prompt_f32", kind="chunk", rope="d64_sections", dtype="f32", batch=2,
             layers=2, kv_heads=2, group=2, n_lo=300, n_hi=777, past_lo=0, past_hi=0, block=0),
        # The keys' weights after one decoded token of 32 sequences.
        dict(name="weights_token", kind="weights", rope="d128_interleaved", dtype="bf16",
             batch=32, layers=2, kv_heads=8, group=4, n_lo=1, n_hi=1, past_lo=2755,
             past_hi=4255, block=0, window=0, accumulate=True),
        # The weights that the last 32 tokens of 16 paged prompts give.
        dict(name="weights_window_paged", kind="weights", rope="d128_sections", dtype="bf16",
             batch=16, layers=2, kv_heads=4, group=7, n_lo=64, n_hi=200, past_lo=2400,
             past_hi=6000, block=16, window=32, accumulate=False),
        # The weights from every token of 4 prompts.
        dict(name="weights_prompt", kind="weights", rope="d128_interleaved", dtype="bf16",
             batch=4, layers=2, kv_heads=8, group=4, n_lo=2560, n_hi=2560, past_lo=0, past_hi=0,
             block=0, window=0, accumulate=False),
        # One sequence of an 8B-class decoder cut back from 1,152 to 768 slots, every layer.
        dict(name="evict_one", kind="evict", rope="d128_interleaved_24", dtype="bf16", batch=1,
             layers=36, kv_heads=8, len_lo=1152, len_hi=1152, budget=768, first=4, last=64,
             block=0),
        # 16 paged sequences, those above 2,048 slots cut back to as many.
        dict(name="evict_paged", kind="evict", rope="d128_sections", dtype="bf16", batch=16,
             layers=28, kv_heads=4, len_lo=1800, len_hi=6000, budget=2048, first=16, last=256,
             block=16),
    ]


# ------------------------------------------------------------------ drawn cases
def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_one(rng):
    kind = rng.choice(["chunk", "chunk", "chunk", "weights", "weights", "evict"])
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    rope = rng.choice(sorted(r for r in ROPES if ROPES[r][0] == (64 if rng.random() < 0.25 else 128)))
    case = dict(kind=kind, rope=rope, dtype=dtype, kv_heads=rng.choice([1, 2, 3, 4, 4, 5, 6, 8, 8, 8]),
                block=rng.choice([0, 0, 0, 0, 16, 16, 32, 64, 8, 24]))
    if kind == "evict":
        lo = _log_int(rng, 40, 6000)
        hi = int(lo * rng.uniform(1.0, 2.5))
        budget = max(24, int(hi * rng.uniform(0.25, 0.95)))
        case.update(batch=_log_int(rng, 1, 48), layers=_log_int(rng, 1, 64), len_lo=lo, len_hi=hi,
                    budget=budget, first=rng.choice([0, 1, 4, 16]),
                    last=rng.choice([0, 1, budget // 8, budget // 3]))
        if case["first"] + case["last"] > budget:
            case["last"] = 0
        return case
    shape = rng.choice(["token", "turn", "mixed", "prompt", "prompt"])
    if shape == "token":
        n_lo = n_hi = 1
    elif shape == "turn":
        n_lo = _log_int(rng, 2, 200)
        n_hi = int(n_lo * rng.uniform(1.0, 2.0))
    elif shape == "mixed":
        n_lo, n_hi = 1, _log_int(rng, 16, 512)
    else:
        n_lo = _log_int(rng, 16, 8000)
        n_hi = int(n_lo * rng.uniform(1.0, 2.0))
    p_lo = 0 if shape == "prompt" else _log_int(rng, 16, 6000)
    case.update(batch=_log_int(rng, 1, 64), layers=rng.choice([1, 2, 3]),
                group=rng.choice([1, 2, 3, 4, 4, 5, 6, 7, 8, 8]), n_lo=n_lo, n_hi=n_hi,
                past_lo=p_lo, past_hi=int(p_lo * rng.uniform(1.0, 2.5)))
    if kind == "weights":
        case.update(window=rng.choice([0, 0, 1, 16, 32, 64]), accumulate=rng.random() < 0.5)
    return case


def draw(rng):
    while True:
        case = _draw_one(rng)
        w = work(case)
        # (float32 products cost 16 times as much as bf16 ones)
        flops = w["flops"] * (16 if case["dtype"] == "f32" else 1)
        if (w["bytes"] <= MOST_BYTES and flops <= MOST_FLOPS and _scores(case) <= MOST_SCORES
                and _resident(case) <= MOST_RESIDENT):
            return case


# ------------------------------------------------------- what a case consists of
def _elem(case):
    return 4 if case["dtype"] == "f32" else 2


def _resident(case):
    row = case["layers"] * case["kv_heads"] * ROPES[case["rope"]][0] * _elem(case) * 2
    if case["kind"] == "evict":
        return case["batch"] * (case["len_hi"] + 64) * row
    return case["batch"] * (case["past_hi"] + case["n_hi"] + 64) * row


def _scores(case):
    if case["kind"] == "evict":
        return 0
    return case["batch"] * case["kv_heads"] * case["group"] * case["n_hi"] * (case["past_hi"] + case["n_hi"])


def _layout(case):
    """A case's lengths: they depend on the case alone (their order comes from the seed), so
    that its work is the same for every seed."""
    rng = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    B = case["batch"]
    if case["kind"] == "evict":
        return {"lens": [rng.randint(case["len_lo"], case["len_hi"]) for _ in range(B)]}
    n = [_log_int(rng, case["n_lo"], case["n_hi"]) for _ in range(B)]
    past = [rng.randint(case["past_lo"], case["past_hi"]) for _ in range(B)]
    return {"n": n, "lens": [a + b for a, b in zip(n, past)]}


class _Inputs:
    """Tensors of one case and seed, made on the GPU."""

    def __init__(self, case, seed):
        self.case, self.dev = case, torch.device("cuda")
        self.rng = np.random.default_rng([int(seed), 23])
        self.gen = torch.Generator(device=self.dev)
        self.gen.manual_seed(int(seed))
        self.dtype = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
        self.head_dim, self.sections, self.interleaved, self.theta = ROPES[case["rope"]]
        self.scale = self.head_dim ** -0.5
        B = case["batch"]
        lay = _layout(case)
        order = self.rng.permutation(B)
        self.lens = np.array(lay["lens"])[order]
        self.cache_len = self.ints(self.lens)
        self.cache(self.lens)
        if case["kind"] == "evict":
            self.capacity = self.cap
            # Weights as attention leaves them: a few large, most small, none negative.
            w = torch.rand((B, case["kv_heads"], self.cap), generator=self.gen, device=self.dev)
            self.weights = w.pow_(8)
            return
        n = np.array(lay["n"])[order]
        self.n = n
        self.off = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
        self.q_off = self.ints(self.off)
        T, Hq, D = int(self.off[-1]), case["kv_heads"] * case["group"], self.head_dim
        self.q = torch.randn((T, Hq, D), generator=self.gen, device=self.dev, dtype=self.dtype)
        # Positions: text counts on; two thirds of a prompt are an image, a grid 48 wide.
        pos = np.zeros((T, 3), np.int32)
        for b in range(B):
            i, m, past = int(self.off[b]), int(n[b]), int(self.lens[b] - n[b])
            pos[i:i + m] = past + np.arange(m)[:, None]
            if past == 0 and m >= 96:
                v0, nv = m // 6, m * 2 // 3
                grid = np.arange(nv)
                pos[i + v0:i + v0 + nv] = v0 + np.stack([0 * grid, grid // 48, grid % 48], axis=1)
                pos[i + v0 + nv:i + m] = v0 + max(48, -(-nv // 48)) + np.arange(m - v0 - nv)[:, None]
        self.pos = self.ints(pos)

    def ints(self, a, dtype=np.int32):
        return torch.from_numpy(np.ascontiguousarray(a, dtype=dtype)).to(self.dev)

    def cache(self, lens):
        """Contiguous or paged cache; keys with four channels per head eight times as large,
        as the keys of rotary decoders have outlier channels."""
        c, D = self.case, self.head_dim
        B, NL, H = c["batch"], c["layers"], c["kv_heads"]
        self.table = None
        if c["block"]:
            need = [-(-int(n) // c["block"]) for n in lens]
            pool = self.rng.permutation(sum(need)).astype(np.int32)
            table = np.full((B, max(need)), -1, np.int32)
            at = 0
            for b, k in enumerate(need):
                table[b, :k] = pool[at:at + k]
                at += k
            self.table_host, self.table = table, self.ints(table)
            shape, head_axis = (NL, sum(need), c["block"], H, D), 3
            self.cap = max(need) * c["block"]
        else:
            self.cap = int(max(lens)) + 32
            shape, head_axis = (B, NL, H, self.cap, D), 2
        scale = torch.ones(H, D, dtype=self.dtype)
        for h in range(H):
            scale[h, self.rng.choice(D, 4, replace=False).tolist()] = 8.0
        view = [1] * 5
        view[head_axis], view[-1] = H, D
        new = lambda: torch.randn(shape, generator=self.gen, device=self.dev, dtype=self.dtype)
        self.cache_k = new().mul_(scale.to(self.dev).view(view))
        self.cache_v = new()


def prepare(case, seed):
    x = _Inputs(case, seed)
    if case["kind"] == "weights":
        # What the program has from its attention of these tokens.
        x.lse = _lse(x, _padded(x))
        x.weights = None
        if case["accumulate"]:
            x.start = torch.rand((case["batch"], case["kv_heads"], x.cap), generator=x.gen, device=x.dev)
            x.weights = x.start.clone()
    x.layer = case["layers"] - 1
    if own:
        import paper_2606_26631_amd as prcr
        x.rope = prcr.Rope(x.head_dim, x.sections, x.interleaved, x.theta)
        x.store = prcr.Cache(x.cache_k, x.cache_v, x.table)
    return x


def run(x):
    return _own(x) if own else _plain(x)


def _own(x):
    import paper_2606_26631_amd as prcr
    c = x.case
    if c["kind"] == "chunk":
        return prcr.chunk_attention(x.rope, x.store, x.layer, x.q, x.q_off, x.pos, x.cache_len)
    if c["kind"] == "weights":
        return prcr.key_weights(x.rope, x.store, x.layer, x.q, x.q_off, x.pos, x.cache_len, x.lse,
                                window=c["window"] or None, weights=x.weights,
                                accumulate=c["accumulate"])
    new_len, kept, weights = prcr.evict(x.store, x.cache_len, x.weights, c["budget"], c["first"], c["last"])
    return new_len, kept, weights, x.cache_k, x.cache_v


# ------------------------------------------------------------------- plain form
def _axes(x):
    """Axis (0 = t, 1 = h, 2 = w) of each rotary pair."""
    i = torch.arange(x.head_dim // 2, device=x.dev)
    st, sh, sw = x.sections
    if x.interleaved:
        a = torch.where((i % 3 == 1) & (i < 3 * sh), 1, 0)
        return torch.where((i % 3 == 2) & (i < 3 * sw), 2, a)
    return (i >= st).long() + (i >= st + sh).long()


def _rotated(x):
    """The queries, rotated in 64 bits and rounded once to the stored type (as the cached keys
    were), in 32 bits."""
    D = x.head_dim
    inv = x.theta ** (-2.0 * torch.arange(D // 2, dtype=torch.float64, device=x.dev) / D)
    ang = (x.pos.double()[:, _axes(x)] * inv)[:, None, :]
    lo, hi = x.q.double().chunk(2, dim=-1)
    y = torch.cat([lo * ang.cos() - hi * ang.sin(), hi * ang.cos() + lo * ang.sin()], dim=-1)
    if x.dtype == torch.bfloat16:
        # (by way of float32 it would be rounded twice)
        m, e = torch.frexp(y)
        y = torch.ldexp(torch.round(m * 256), e - 8)
    return y.float()


def _rows(x, cached):
    """A layer's cached rows, [B, H, most keys, D] in 32 bits."""
    most = int(x.lens.max())
    if x.table is None:
        return cached[:, x.case["layers"] - 1, :, :most].float()
    r = cached[x.case["layers"] - 1][x.table.clamp(min=0).long()].flatten(1, 2)[:, :most]
    return r.transpose(1, 2).float()


def _padded(x):
    """What all of the plain form goes by: (row of each sequence's i-th token [B, N], whether
    there is one, each such token's scores [B, H, G, N, L] with -inf at what it does not see)."""
    c = x.case
    B, H, G, N = c["batch"], c["kv_heads"], c["group"], int(x.n.max())
    off = x.q_off.long()
    i = torch.arange(N, device=x.dev)
    live = i < (off[1:] - off[:-1])[:, None]
    row = torch.where(live, off[:-1, None] + i, 0)
    q = _rotated(x)[row].view(B, N, H, G, -1).permute(0, 2, 3, 1, 4).reshape(B, H, G * N, -1)
    k = _rows(x, x.cache_k)
    s = torch.matmul(q, k.transpose(2, 3)).mul_(x.scale).view(B, H, G, N, -1)
    first = (x.cache_len - (x.q_off[1:] - x.q_off[:-1]))[:, None, None]
    sees = torch.arange(k.shape[2], device=x.dev) <= first + i[:, None]
    s.masked_fill_(~(sees & live[:, :, None])[:, None, None], -math.inf)
    return row, live, s


def _packed(padded, live):
    """[B, H, G, N, ...] to the packed tokens' [T, H * G, ...]."""
    t = padded.permute(0, 3, 1, 2, *range(4, padded.dim()))
    return t[live].flatten(1, 2)


def _lse(x, padded):
    _, live, s = padded
    m = s.amax(-1, keepdim=True).clamp(min=-3e38)
    return _packed((s - m).exp_().sum(-1).log_() + m.squeeze(-1), live).contiguous()


def _plain(x):
    c = x.case
    if c["kind"] == "evict":
        return _plain_evict(x)
    row, live, s = _padded(x)
    B, H, G, N, L = s.shape
    if c["kind"] == "chunk":
        m = s.amax(-1, keepdim=True).clamp(min=-3e38)
        e = s.sub_(m).exp_()
        l = e.sum(-1)
        o = torch.matmul(e.view(B, H, G * N, L), _rows(x, x.cache_v)).view(B, H, G, N, -1)
        o = o / l.unsqueeze(-1)
        return _packed(o, live).to(x.dtype), _packed(l.log() + m.squeeze(-1), live)
    lse = x.lse[row].view(B, N, H, G).permute(0, 2, 3, 1)
    n = (x.q_off[1:] - x.q_off[:-1])[:, None]
    used = live & (torch.arange(N, device=x.dev) >= n - (c["window"] or N))
    w = s.sub_(lse.unsqueeze(-1)).exp_().mul_(used[:, None, None, :, None]).sum((2, 3))
    if c["accumulate"]:
        x.weights[:, :, :L] += w
        return x.weights
    full = torch.zeros((B, H, x.cap), device=x.dev)
    full[:, :, :L] = w
    return full


def _plain_evict(x):
    c = x.case
    B, H, K = c["batch"], c["kv_heads"], c["budget"]
    j = torch.arange(x.cap, device=x.dev)
    n = x.cache_len[:, None]
    score = x.weights.double().sum(1).float()
    fixed = (j < c["first"]) | (j >= n - c["last"]) | (n <= K)
    score = torch.where(fixed, math.inf, score).masked_fill(j >= n, -math.inf)
    kept = score.sort(dim=1, descending=True, stable=True).indices[:, :K]
    new_len = n.clamp(max=K)
    kept = torch.where(j[:kept.shape[1]] < new_len, kept, x.cap).sort(dim=1).values
    kept = torch.nn.functional.pad(kept, (0, K - kept.shape[1]), value=x.cap)
    live = kept < x.cap
    src = torch.where(live, kept, 0)
    weights = torch.zeros_like(x.weights)
    most = min(K, x.cap)
    weights[:, :, :most] = (x.weights.gather(2, src[:, None].expand(B, H, K)) * live[:, None])[:, :, :most]
    b = torch.arange(B, device=x.dev)[:, None].expand(B, K)[live]
    frm, to = src[live], torch.arange(K, device=x.dev).expand(B, K)[live]
    if x.table is None:
        x.cache_k[b, :, :, to] = x.cache_k[b, :, :, frm]
        x.cache_v[b, :, :, to] = x.cache_v[b, :, :, frm]
    else:
        bs, t = c["block"], x.table.long()
        fb, tb = t[b, frm // bs], t[b, to // bs]
        x.cache_k[:, tb, to % bs] = x.cache_k[:, fb, frm % bs]
        x.cache_v[:, tb, to % bs] = x.cache_v[:, fb, frm % bs]
    return (new_len[:, 0].int(), torch.where(live, kept, -1).int(), weights, x.cache_k, x.cache_v)


# ------------------------------------------------------------------------- work
def work(case):
    D, s, H = ROPES[case["rope"]][0], _elem(case), case["kv_heads"]
    lay = _layout(case)
    table = sum(-(-n // case["block"]) for n in lay["lens"]) * 4 if case["block"] else 0
    B = case["batch"]
    if case["kind"] == "evict":
        # The kept rows but the first ones move: read and written, keys and values.
        moved = sum(case["budget"] - case["first"] for n in lay["lens"] if n > case["budget"])
        kept = sum(min(n, case["budget"]) for n in lay["lens"])
        return {"bytes": moved * case["layers"] * H * D * 4 * s + sum(lay["lens"]) * H * 4
                + kept * (H + 1) * 4 + table + 8 * B, "flops": 0}
    G = case["group"]
    T, keys = sum(lay["n"]), sum(lay["lens"])
    if case["kind"] == "weights" and case["window"]:
        n = [min(a, case["window"]) for a in lay["n"]]
    else:
        n = lay["n"]
    rows = sum(n)
    seen = sum(a * (b - a) + a * (a + 1) // 2 for a, b in zip(n, lay["lens"]))
    if case["kind"] == "chunk":
        return {"bytes": keys * H * D * 2 * s + T * H * G * (D * 2 * s + 4) + T * 12 + table + 8 * B,
                "flops": seen * H * G * D * 4}
    return {"bytes": keys * H * (D * s + (8 if case["accumulate"] else 4))
            + rows * (H * G * (D * s + 4) + 12) + table + 8 * B, "flops": seen * H * G * D * 2}


# ------------------------------------------------------------- 64-bit reference
def _bf16_nearest(y):
    """float64 array to the nearest bfloat16 (ties to even), as float64."""
    m, e = np.frexp(y)
    return np.ldexp(np.rint(np.ldexp(m, 8)), e - 8)


def _exact_queries(x):
    """Rotated queries [T, Hq, D] (float64) as the definition has them: complex pairs turned by
    their angles, rounded once to the stored type."""
    D, P = x.head_dim, x.head_dim // 2
    st, sh, sw = x.sections
    axis = [(1 if i % 3 == 1 and i < 3 * sh else 2 if i % 3 == 2 and i < 3 * sw else 0) if x.interleaved
            else (0 if i < st else 1 if i < st + sh else 2) for i in range(P)]
    freq = torch.tensor([x.theta ** (-2.0 * i / D) for i in range(P)], dtype=torch.float64, device=x.dev)
    turn = x.pos.double()[:, torch.tensor(axis, device=x.dev)] * freq
    z = torch.complex(x.q[..., :P].double(), x.q[..., P:].double())
    z = z * torch.polar(torch.ones_like(turn), turn)[:, None, :]
    y = torch.cat([z.real, z.imag], dim=-1)
    if x.dtype == torch.bfloat16:
        return torch.from_numpy(_bf16_nearest(y.cpu().numpy())).to(x.dev)
    return y.float().double()


def _exact_rows(x, cached, b, h, n):
    """Slots 0..n-1 of one sequence and KV head, [n, D] in float64."""
    layer = x.case["layers"] - 1
    if x.table is None:
        return cached[b, layer, h, :n].double()
    slots = np.arange(n)
    blk = torch.from_numpy(x.table_host[b, slots // x.case["block"]].astype(np.int64)).to(x.dev)
    return cached[layer, blk, torch.from_numpy(slots % x.case["block"]).to(x.dev), h].double()


def exact(case, seed):
    x = prepare(case, seed)
    if case["kind"] == "evict":
        return _exact_evict(x)
    B, H, G, D = case["batch"], case["kv_heads"], case["group"], x.head_dim
    q = _exact_queries(x)
    T = q.shape[0]
    chunk = case["kind"] == "chunk"
    out = torch.zeros((T, H * G, D), dtype=torch.float64, device=x.dev) if chunk else None
    lse = torch.zeros((T, H * G), dtype=torch.float64, device=x.dev) if chunk else None
    w = None if chunk else torch.zeros((B, H, x.cap), dtype=torch.float64, device=x.dev)
    if not chunk and case["accumulate"]:
        w += x.start.double()
    for b in range(B):
        n, m, r0 = int(x.lens[b]), int(x.n[b]), int(x.off[b])
        if not chunk and case["window"]:
            r0, m = r0 + max(0, m - case["window"]), min(m, case["window"])
        hidden = torch.arange(n, device=x.dev)[None, :] > (n - m + torch.arange(m, device=x.dev))[:, None]
        for h in range(H):
            k = _exact_rows(x, x.cache_k, b, h, n)
            v = _exact_rows(x, x.cache_v, b, h, n) if chunk else None
            for g in range(G):
                qh = h * G + g
                s = (q[r0:r0 + m, qh] @ k.T) * x.scale
                s[hidden] = -math.inf
                if chunk:
                    lse[r0:r0 + m, qh] = s.logsumexp(1)
                    out[r0:r0 + m, qh] = s.softmax(1) @ v
                else:
                    w[b, h, :n] += (s - x.lse[r0:r0 + m, qh].double()[:, None]).exp().sum(0)
    return (out, lse) if chunk else w


def _exact_evict(x):
    """The kept slots, the weights and the caches, one sequence at a time."""
    c = x.case
    B, K, bs = c["batch"], c["budget"], c["block"]
    w = x.weights.cpu().numpy()
    score = w.astype(np.float64).sum(axis=1).astype(np.float32)
    kept = np.full((B, K), -1, np.int32)
    weights = np.zeros(w.shape, np.float64)
    new_len = np.minimum(x.lens, K)
    ck, cv = x.cache_k.clone(), x.cache_v.clone()
    for b in range(B):
        n = int(x.lens[b])
        keep = np.arange(n)
        if n > K:
            between = np.arange(c["first"], n - c["last"])
            best = np.lexsort((between, -score[b, between]))[:K - c["first"] - c["last"]]
            keep = np.sort(np.concatenate([np.arange(c["first"]), between[best], np.arange(n - c["last"], n)]))
        kept[b, :len(keep)] = keep
        weights[b, :, :len(keep)] = w[b][:, keep]
        to = np.arange(len(keep))
        idx = lambda a: torch.from_numpy(a.astype(np.int64)).to(x.dev)
        for new, old in ((ck, x.cache_k), (cv, x.cache_v)):
            if bs:
                t = x.table_host[b]
                new[:, idx(t[to // bs]), idx(to % bs)] = old[:, idx(t[keep // bs]), idx(keep % bs)]
            else:
                new[b][:, :, :len(keep)] = old[b][:, :, idx(keep)]
    # (moved rows are the stored ones, bit for bit: their values in 64 bits are the same numbers)
    return (x.ints(new_len), x.ints(kept), torch.from_numpy(weights).to(x.dev), ck, cv)
