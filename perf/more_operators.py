"""The decoder cache in 8 bits, as cases that can be timed and compared: writing it (a prompt's
or a decoded token's keys and values, revisited tokens), reading it back, and a decoded token's
attention over it.

A cache row (one slot, layer and KV head) is head_dim codes, e4m3 or int8, and one float32
scale.  With x the row that a cache of the inputs' type would hold (keys rotated in double and
rounded once to that type, values as they are) and Q = 448 (e4m3) or 127 (int8), in float32:

    scale = max(max |x_i| / Q, 2^-126),   code_i = nearest(x_i * (1 / scale)), ties to even

and the row stands for code_i * scale.  A program appends each layer's rows as the model makes
them (quant_append), appends revisited visual tokens in all layers (quant_rebind_inject), attends
with every decoded token (quant_decode_attention), and reads a layer back where an operator on
several tokens needs it in the model's type (quant_read).  Shapes are those of workloads.py and
bench.py: 28 layers x 4 KV heads x 7 and 36 layers x 8 KV heads x 4 query heads, head_dim 128,
bf16, and a small float32 decoder of head_dim 64.
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
LARGEST = {"e4m3": 448.0, "i8": 127.0}     # the largest code
# Bounds of a drawn case: the largest listed ones' traffic and resident bytes.
MOST_BYTES = 7.2e8
MOST_RESIDENT = 5.2e9


def listed():
    return [
        # The smallest call: one decoded token of a small float32 decoder, after 299 others.
        dict(name="append_token_f32", kind="append", rope="d64_sections", dtype="f32", code="e4m3",
             batch=1, layers=2, kv_heads=2, n_lo=1, n_hi=1, past_lo=299, past_hi=299, block=0),
        # A serving step: one decoded token of each of 64 paged sequences.
        dict(name="append_step_paged", kind="append", rope="d128_sections", dtype="bf16",
             code="e4m3", batch=64, layers=2, kv_heads=4, n_lo=1, n_hi=1, past_lo=2911,
             past_hi=6511, block=16),
        # Prefill of one layer: 8 prompts of 2,560 tokens, 2,048 of them visual.
        dict(name="append_prompts", kind="append", rope="d128_interleaved", dtype="bf16",
             code="e4m3", batch=8, layers=2, kv_heads=8, n_lo=2560, n_hi=2560, past_lo=0, past_hi=0,
             block=0),
        # The next turns of six paged sequences, text and an image each: written in int8, and the
        # layer read back for these tokens' attention.
        dict(name="append_read_turns_i8", kind="append", rope="d128_sections", dtype="bf16",
             code="i8", batch=6, layers=2, kv_heads=4, n_lo=361, n_hi=1783, past_lo=900, past_hi=2545,
             block=16),
        # One sequence's layer read back before a turn of a few tokens.
        dict(name="read_one_i8", kind="read", rope="d128_interleaved_24", dtype="bf16", code="i8",
             batch=1, layers=2, kv_heads=8, len_lo=1152, len_hi=1152, block=0),
        # A serving batch's layer read back: 64 paged sequences of mixed length.
        dict(name="read_paged", kind="read", rope="d128_sections", dtype="bf16", code="e4m3",
             batch=64, layers=2, kv_heads=4, len_lo=2912, len_hi=6512, block=16),
        # One sequence of an 8B-class decoder revisits 32 visual tokens.
        dict(name="rebind_8b_k32", kind="rebind", rope="d128_interleaved_24", dtype="bf16",
             code="e4m3", batch=1, layers=36, kv_heads=8, visual=768, k_lo=32, k_hi=32, len_lo=1024,
             len_hi=1024, block=0),
        # Serving: 16 paged sequences revisit 512 of 2,304 visual tokens each.
        dict(name="rebind_paged", kind="rebind", rope="d128_sections", dtype="bf16", code="e4m3",
             batch=16, layers=28, kv_heads=4, visual=2304, k_lo=512, k_hi=512, len_lo=2400,
             len_hi=6000, block=16),
        # One sequence's decoded token, one layer: 32 query heads over 8 KV heads.
        dict(name="decode_one", kind="decode", rope="d128_interleaved_24", dtype="bf16", code="e4m3",
             batch=1, layers=2, kv_heads=8, group=4, len_lo=1152, len_hi=1152, block=0),
        # A serving step of 32 sequences, one layer, contiguous.
        dict(name="decode_batch", kind="decode", rope="d128_interleaved", dtype="bf16", code="e4m3",
             batch=32, layers=2, kv_heads=8, group=4, len_lo=2756, len_hi=4256, block=0),
        # The same of 64 sequences in a paged int8 cache, 28 query heads over 4 KV heads.
        dict(name="decode_paged_i8", kind="decode", rope="d128_sections", dtype="bf16", code="i8",
             batch=64, layers=2, kv_heads=4, group=7, len_lo=2912, len_hi=6512, block=16),
        # One long video, float32 queries: the cache's length shared out over the chip.
        dict(name="decode_long", kind="decode", rope="d128_interleaved_24", dtype="f32", code="e4m3",
             batch=1, layers=1, kv_heads=8, group=4, len_lo=120001, len_hi=120001, block=0),
    ]


# ------------------------------------------------------------------ drawn cases
def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_one(rng):
    kind = rng.choice(["append", "append", "read", "rebind", "decode", "decode", "decode"])
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    rope = rng.choice(sorted(r for r in ROPES if ROPES[r][0] == (64 if rng.random() < 0.25 else 128)))
    case = dict(kind=kind, rope=rope, dtype=dtype, code=rng.choice(["e4m3", "i8"]),
                kv_heads=rng.choice([1, 2, 3, 4, 4, 5, 6, 8, 8, 8]),
                block=rng.choice([0, 0, 0, 0, 16, 16, 32, 64, 8, 24]))
    case.update(batch=_log_int(rng, 1, 64), layers=rng.choice([1, 2, 3]))
    if kind == "append":
        n_lo = rng.choice([1, _log_int(rng, 2, 200), _log_int(rng, 16, 4000)])
        p_lo = rng.choice([0, _log_int(rng, 1, 6000)])
        case.update(n_lo=n_lo, n_hi=1 if n_lo == 1 else int(n_lo * rng.uniform(1.0, 2.5)), past_lo=p_lo,
                    past_hi=int(p_lo * rng.uniform(1.0, 2.5)))
    elif kind == "rebind":
        visual = _log_int(rng, 36, 4608)
        hi = _log_int(rng, 4, min(1024, visual))
        lo = _log_int(rng, 40, 6000)
        case.update(code="e4m3", layers=_log_int(rng, 2, 64), visual=visual,
                    k_lo=max(1, int(hi * rng.choice([1.0, 1.0, 0.6, 0.1]))), k_hi=hi, len_lo=lo,
                    len_hi=int(lo * rng.uniform(1.0, 2.5)))
    else:
        lo = _log_int(rng, 16, 6000)
        if kind == "decode" and rng.random() < 0.2:
            lo, case["batch"] = _log_int(rng, 6000, 48000), _log_int(rng, 1, 4)
        case.update(len_lo=lo, len_hi=int(lo * rng.uniform(1.0, 2.5)))
        if kind == "decode":
            case["group"] = rng.choice([1, 2, 3, 4, 4, 5, 6, 7, 8, 8])
    return case


def draw(rng):
    while True:
        case = _draw_one(rng)
        if work(case)["bytes"] <= MOST_BYTES and _resident(case) <= MOST_RESIDENT:
            return case


# ------------------------------------------------------- what a case consists of
def _elem(case):
    return 4 if case["dtype"] == "f32" else 2


def _longest(case):
    if case["kind"] == "append":
        return case["past_hi"] + case["n_hi"]
    return case["len_hi"] + (case["k_hi"] if case["kind"] == "rebind" else 0)


def _resident(case):
    D, H = ROPES[case["rope"]][0], case["kv_heads"]
    cache = case["batch"] * (_longest(case) + 64) * case["layers"] * H * 2 * (D + 4)
    rows = 0
    if case["kind"] == "append":
        rows = case["batch"] * case["n_hi"]
    elif case["kind"] == "read":
        rows = case["batch"] * case["len_hi"]
    elif case["kind"] == "rebind":
        rows = case["batch"] * case["visual"] * case["layers"]
    return cache + rows * H * D * 2 * _elem(case)


def _layout(case):
    """A case's lengths: they depend on the case alone (their order comes from the seed), so
    that its work is the same for every seed."""
    rng = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    B = case["batch"]
    if case["kind"] == "append":
        n = [_log_int(rng, case["n_lo"], case["n_hi"]) for _ in range(B)]
        past = [rng.randint(case["past_lo"], case["past_hi"]) for _ in range(B)]
        return {"n": n, "past": past, "lens": [a + b for a, b in zip(n, past)]}
    lay = {"lens": [rng.randint(case["len_lo"], case["len_hi"]) for _ in range(B)]}
    if case["kind"] == "rebind":
        lay["k"] = [rng.randint(case["k_lo"], case["k_hi"]) for _ in range(B)]
    return lay


class _Inputs:
    """Tensors of one case and seed, made on the GPU."""

    def __init__(self, case, seed):
        self.case, self.dev = case, torch.device("cuda")
        self.rng = np.random.default_rng([int(seed), 29])
        self.gen = torch.Generator(device=self.dev)
        self.gen.manual_seed(int(seed))
        self.dtype = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
        self.head_dim, self.sections, self.interleaved, self.theta = ROPES[case["rope"]]
        self.layer, self.scale = case["layers"] - 1, self.head_dim ** -0.5
        lay = _layout(case)
        order = self.rng.permutation(case["batch"])
        getattr(self, "_" + case["kind"])({k: np.array(v)[order] for k, v in lay.items()})

    def _append(self, lay):
        c, D = self.case, self.head_dim
        B, H, n, past = c["batch"], c["kv_heads"], lay["n"], lay["past"]
        self.n, self.past, self.lens = n, past, lay["lens"]
        S = int(n.max())
        self.raw_k = self.keys((B, S, H, D), 2)
        self.raw_v = self.normal((B, S, H, D))
        # Text counts on; two thirds of a prompt or turn are an image, a grid 48 wide.
        s = np.arange(S)
        pos = np.repeat((past[:, None] + s)[:, :, None], 3, axis=2)
        for b in range(B):
            m = int(n[b])
            if m >= 96:
                v0, nv = m // 6, m * 2 // 3
                g = np.arange(nv)
                pos[b, v0:v0 + nv] = past[b] + v0 + np.stack([0 * g, g // 48, g % 48], axis=1)
                pos[b, v0 + nv:] = past[b] + v0 + max(48, -(-nv // 48)) + np.arange(S - v0 - nv)[:, None]
        self.pos, self.n_tokens, self.start = self.ints(pos), self.ints(n), self.ints(past)
        self.cache_len = self.ints(self.lens)
        self.cache(self.lens)

    def _read(self, lay):
        self.lens = lay["lens"]
        self.cache_len = self.ints(self.lens)
        self.cache(self.lens)

    def _rebind(self, lay):
        c, D = self.case, self.head_dim
        B, M, NL, H, k = c["batch"], c["visual"], c["layers"], c["kv_heads"], lay["k"]
        self.lens = lay["lens"]
        self.mem_k, self.mem_v = self.keys((B, M, NL, H, D), 3), self.normal((B, M, NL, H, D))
        self.coords = self.ints(np.zeros((B, M, 3)))
        self.n_visual = self.ints(np.full(B, M))
        off = np.concatenate([[0], np.cumsum(k)])
        idx = np.concatenate([np.sort(self.rng.choice(M, int(m), replace=False)) for m in k])
        # New positions as reassignment makes them: real numbers in a short stretch before the
        # next text position.
        at = np.repeat(self.lens, k)[:, None]
        self.new_pos = torch.from_numpy(at - 2 + 3 * self.rng.random((len(idx), 3))).to(self.dev)
        self.sel_off, self.sel_idx, self.k_of = self.ints(off), self.ints(idx), k
        self.cache_len = self.ints(self.lens)
        self.cache(self.lens + k)

    def _decode(self, lay):
        c = self.case
        self.lens = lay["lens"]
        self.q = self.normal((c["batch"], c["kv_heads"] * c["group"], self.head_dim))
        self.cache_len = self.ints(self.lens)
        self.q_pos = self.ints(self.lens + self.rng.integers(0, 40, c["batch"]))
        self.cache(self.lens)

    def ints(self, a, dtype=np.int32):
        return torch.from_numpy(np.ascontiguousarray(a, dtype=dtype)).to(self.dev)

    def normal(self, shape):
        return torch.randn(shape, generator=self.gen, device=self.dev, dtype=self.dtype)

    def keys(self, shape, head_axis):
        """Keys: four channels of a head are four times as large, as those of rotary decoders
        have outlier channels."""
        H, D = self.case["kv_heads"], self.head_dim
        scale = torch.ones(H, D, dtype=self.dtype)
        for h in range(H):
            scale[h, self.rng.choice(D, 4, replace=False).tolist()] = 4.0
        view = [1] * len(shape)
        view[head_axis], view[-1] = H, D
        return self.normal(shape).mul_(scale.to(self.dev).view(view))

    def cache(self, lens):
        """The 8-bit cache with room for `lens` slots.  What is in it: quantised rows as above where
        the case reads them, any finite codes where it only writes."""
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
            shape, scales, head_axis = (NL, sum(need), c["block"], H, D), (NL, sum(need), H, c["block"]), 3
            self.cap = max(need) * c["block"]
        else:
            self.cap = int(max(lens)) + 32
            shape, scales, head_axis = (B, NL, H, self.cap, D), (B, NL, H, self.cap), 2
        kind = torch.float8_e4m3fn if c["code"] == "e4m3" else torch.int8
        if c["kind"] == "rebind":
            new = lambda: (torch.randint(0, 120, shape, generator=self.gen, device=self.dev, dtype=torch.uint8)
                           .view(kind), torch.rand(scales, generator=self.gen, device=self.dev))
            self.k, self.k_scale = new()
            self.v, self.v_scale = new()
            return
        # (a layer of it is quantised; the others hold the same)
        one = (B, 1, H, self.cap, D) if self.table is None else (1,) + shape[1:]
        layers = 1 if self.table is None else 0

        def made(rows):
            code, scale = _quantised(rows.float(), c["code"])
            if self.table is not None:
                scale = scale.transpose(2, 3)
            spread = lambda t: t.expand(*[NL if i == layers else n for i, n in enumerate(t.shape)]).contiguous()
            return spread(code.view(torch.uint8)).view(kind), spread(scale)

        self.k, self.k_scale = made(self.keys(one, head_axis))
        self.v, self.v_scale = made(self.normal(one))


def prepare(case, seed):
    x = _Inputs(case, seed)
    if own:
        import paper_2606_26631_amd as prcr
        x.rope = prcr.Rope(x.head_dim, x.sections, x.interleaved, x.theta)
        x.store = prcr.QuantCache(x.k, x.v, x.k_scale, x.v_scale, x.table)
        if case["kind"] == "rebind":
            x.mem = prcr.Memory(x.mem_k, x.mem_v, x.coords, x.n_visual)
    if case["kind"] == "read" or (case["kind"] == "append" and case["code"] == "i8"):
        # Where a layer is read back to: what lies behind a sequence's length stays.
        shape = (case["batch"], 1, case["kv_heads"], x.cap, x.head_dim)
        x.read_k, x.read_v = (torch.zeros(shape, device=x.dev, dtype=x.dtype) for _ in range(2))
    return x


def run(x):
    return _own(x) if own else _plain(x)


def _own(x):
    import paper_2606_26631_amd as prcr
    kind = x.case["kind"]
    if kind == "decode":
        return prcr.quant_decode_attention(x.rope, x.store, x.layer, x.q, x.q_pos, x.cache_len)
    if kind == "rebind":
        prcr.quant_rebind_inject(x.rope, x.mem, x.sel_off, x.sel_idx, x.new_pos, x.store, x.cache_len)
        return x.k, x.v, x.k_scale, x.v_scale
    if kind == "append":
        prcr.quant_append(x.rope, x.store, x.layer, x.raw_k, x.raw_v, x.pos, x.n_tokens, x.start)
        if x.case["code"] == "e4m3":
            return x.k, x.v, x.k_scale, x.v_scale
    k, v = prcr.quant_read(x.store, x.layer, x.cache_len, x.dtype, k=x.read_k, v=x.read_v)
    return k, v, x.k_scale, x.v_scale


# ------------------------------------------------------------------- plain form
def _quantised(rows, code):
    """(codes, scales) of float32 rows [..., D]."""
    most = rows.abs().amax(-1)
    scale = (most.double() / LARGEST[code]).float().clamp(min=2.0 ** -126)
    y = rows * scale.double().reciprocal().float().unsqueeze(-1)
    return y.to(torch.float8_e4m3fn) if code == "e4m3" else y.round().to(torch.int8), scale


def _axes(x):
    """Axis (0 = t, 1 = h, 2 = w) of each rotary pair."""
    i = torch.arange(x.head_dim // 2, device=x.dev)
    st, sh, sw = x.sections
    if x.interleaved:
        a = torch.where((i % 3 == 1) & (i < 3 * sh), 1, 0)
        return torch.where((i % 3 == 2) & (i < 3 * sw), 2, a)
    return (i >= st).long() + (i >= st + sh).long()


def _turned(x, rows, pos):
    """rows [n, ..., D] rotated in 64 bits at pos [n, 3]."""
    D = x.head_dim
    inv = x.theta ** (-2.0 * torch.arange(D // 2, dtype=torch.float64, device=x.dev) / D)
    ang = pos.double()[:, _axes(x)] * inv
    ang = ang.view(ang.shape[0], *[1] * (rows.dim() - 2), -1)
    lo, hi = rows.double().chunk(2, dim=-1)
    return torch.cat([lo * ang.cos() - hi * ang.sin(), hi * ang.cos() + lo * ang.sin()], dim=-1)


def _stored(x, y):
    """64-bit rows rounded once to the inputs' type, in 32 bits."""
    if x.dtype == torch.bfloat16:
        # (by way of float32 it would be rounded twice)
        m, e = torch.frexp(y)
        y = torch.ldexp(torch.round(m * 256), e - 8)
    return y.float()


def _cached(x, codes, scales):
    """A layer's cached rows, [B, H, capacity, D] in 32 bits (any block's where the table has none)."""
    if x.table is None:
        return codes[:, x.layer].float() * scales[:, x.layer].unsqueeze(-1)
    t = x.table.clamp(min=0).long()
    r = codes.view(torch.uint8)[x.layer][t].view(codes.dtype).float()
    r = r * scales[x.layer][t].transpose(2, 3).unsqueeze(-1)
    return r.flatten(1, 2).transpose(1, 2)


def _plain(x):
    c = x.case
    kind = c["kind"]
    if kind == "decode":
        return _plain_decode(x)
    if kind == "rebind":
        b = torch.repeat_interleave(torch.arange(c["batch"], device=x.dev),
                                    (x.sel_off[1:] - x.sel_off[:-1]).long())
        j = torch.arange(len(b), device=x.dev) - x.sel_off.long()[b]
        slot, m = x.cache_len.long()[b] + j, x.sel_idx.long()
        k, v = _stored(x, _turned(x, x.mem_k[b, m], x.new_pos)), x.mem_v[b, m].float()
        _write(x, x.k, x.k_scale, k, b, slot)
        _write(x, x.v, x.v_scale, v, b, slot)
        return x.k, x.v, x.k_scale, x.v_scale
    if kind == "append":
        s = torch.arange(x.raw_k.shape[1], device=x.dev)
        b, s = (s < x.n_tokens[:, None]).nonzero(as_tuple=True)
        slot = x.start.long()[b] + s
        k, v = _stored(x, _turned(x, x.raw_k[b, s], x.pos[b, s])), x.raw_v[b, s].float()
        _write(x, x.k, x.k_scale, k, b, slot, x.layer)
        _write(x, x.v, x.v_scale, v, b, slot, x.layer)
        if c["code"] == "e4m3":
            return x.k, x.v, x.k_scale, x.v_scale
    live = (torch.arange(x.cap, device=x.dev) < x.cache_len[:, None])[:, None, :, None]
    for to, codes, scales in ((x.read_k, x.k, x.k_scale), (x.read_v, x.v, x.v_scale)):
        to[:, 0] = torch.where(live, _cached(x, codes, scales).to(x.dtype), to[:, 0])
    return x.read_k, x.read_v, x.k_scale, x.v_scale


def _write(x, codes, scales, rows, b, slot, layer=None):
    """Rows [n, (layers,) H, D] quantised into slots `slot` of sequences b."""
    code, scale = _quantised(rows, x.case["code"])
    code, to = code.view(torch.uint8), codes.view(torch.uint8)
    if x.table is None:
        at = slice(None) if layer is None else layer
        to[b, at, :, slot] = code
        scales[b, at, :, slot] = scale
        return
    blk, off = x.table.long()[b, slot // x.case["block"]], slot % x.case["block"]
    if layer is None:
        to[:, blk, off] = code.transpose(0, 1)
        scales[:, blk, :, off] = scale
    else:
        to[layer, blk, off] = code
        scales[layer, blk, :, off] = scale


def _plain_decode(x):
    c = x.case
    B, H, G = c["batch"], c["kv_heads"], c["group"]
    q = _turned(x, x.q, x.q_pos[:, None].expand(B, 3)).mul_(x.scale).float().view(B, H, G, -1)
    s = torch.matmul(q, _cached(x, x.k, x.k_scale).transpose(2, 3))
    hidden = torch.arange(s.shape[-1], device=x.dev) >= x.cache_len[:, None]
    s.masked_fill_(hidden[:, None, None], -math.inf)
    e = s.sub_(s.amax(-1, keepdim=True)).exp_()
    o = torch.matmul(e, _cached(x, x.v, x.v_scale)) / e.sum(-1, keepdim=True)
    return o.view(B, H * G, -1)


# ------------------------------------------------------------------------- work
def work(case):
    D, s, H, B = ROPES[case["rope"]][0], _elem(case), case["kv_heads"], case["batch"]
    lay = _layout(case)
    lens = [a + b for a, b in zip(lay["lens"], lay["k"])] if case["kind"] == "rebind" else lay["lens"]
    table = sum(-(-n // case["block"]) for n in lens) * 4 if case["block"] else 0
    coded, plain = 2 * H * (D + 4), 2 * H * D * s         # bytes of a slot's rows in one layer
    if case["kind"] == "decode":
        return {"bytes": sum(lens) * coded + table + 8 * B + B * H * case["group"] * D * (s + 4),
                "flops": sum(lens) * H * case["group"] * D * 4}
    if case["kind"] == "read":
        return {"bytes": sum(lens) * (coded + plain) + table + 4 * B, "flops": sum(lens) * H * D * 2}
    if case["kind"] == "rebind":
        n = sum(lay["k"])
        return {"bytes": n * case["layers"] * (coded + plain) + n * 36 + table + 12 * B,
                "flops": n * case["layers"] * H * D * 7}
    n = sum(lay["n"])
    w = {"bytes": n * (coded + plain + 12) + table + 8 * B, "flops": n * H * D * 7}
    if case["code"] == "i8":
        w["bytes"] += sum(lens) * (coded + plain)
        w["flops"] += sum(lens) * H * D * 2
    return w


# ------------------------------------------------------------- 64-bit reference
def _nearest(y, fraction, least):
    """float64 array to the nearest number of so many fraction bits and that least exponent, ties
    to even."""
    _, e = np.frexp(y)
    step = np.ldexp(1.0, np.maximum(e - 1, least) - fraction)
    return np.rint(y / step) * step


def _exact_turned(x, rows, pos):
    """Rows [n, ..., D] at pos [n, 3]: complex pairs turned by their angles, float64."""
    D, P = x.head_dim, x.head_dim // 2
    st, sh, sw = x.sections
    axis = [(1 if i % 3 == 1 and i < 3 * sh else 2 if i % 3 == 2 and i < 3 * sw else 0) if x.interleaved
            else (0 if i < st else 1 if i < st + sh else 2) for i in range(P)]
    freq = torch.tensor([x.theta ** (-2.0 * i / D) for i in range(P)], dtype=torch.float64, device=x.dev)
    turn = pos.double()[:, torch.tensor(axis, device=x.dev)] * freq
    z = torch.complex(rows[..., :P].double(), rows[..., P:].double())
    u = torch.polar(torch.ones_like(turn), turn)
    z = z * u.view(u.shape[0], *[1] * (rows.dim() - 2), P)
    return torch.cat([z.real, z.imag], dim=-1).cpu().numpy()


def _exact_codes(x, y):
    """Codes and scales of rows (float64, before their rounding to the inputs' type)."""
    y = _nearest(y, 7, -126) if x.dtype == torch.bfloat16 else y.astype(np.float32).astype(np.float64)
    scale = np.maximum(np.abs(y).max(axis=-1) / LARGEST[x.case["code"]], 2.0 ** -126)
    y = y / scale[..., None]
    return _nearest(y, 3, -6) if x.case["code"] == "e4m3" else np.rint(y), scale


def _exact_place(x, b, slots):
    """Index of a sequence's slots: (sequence, slot), or (block, offset)."""
    if x.table is None:
        return b, torch.from_numpy(slots).to(x.dev)
    bs = x.case["block"]
    return (torch.from_numpy(x.table_host[b, slots // bs].astype(np.int64)).to(x.dev),
            torch.from_numpy(slots % bs).to(x.dev))


def _exact_layer(x, codes, scales, b, n):
    """Slots 0..n-1 of a sequence in the case's layer: [H, n, D] float64."""
    i, j = _exact_place(x, b, np.arange(n))
    if x.table is None:
        return codes[b, x.layer, :, :n].double() * scales[b, x.layer, :, :n, None].double()
    c = codes[x.layer].view(torch.uint8)[i, j].view(codes.dtype).double()
    return (c * scales[x.layer][i, :, j].double()[..., None]).transpose(0, 1)


def _exact_store(x, codes, scales, b, slots, rows):
    """Rows [n, (layers,) H, D] (float64) of one sequence into float64 caches."""
    code, scale = (torch.from_numpy(t).to(x.dev) for t in _exact_codes(x, rows))
    i, j = _exact_place(x, b, slots)
    if code.dim() == 3:
        code, scale = code[:, None], scale[:, None]
        layers = slice(x.layer, x.layer + 1)
    else:
        layers = slice(None)
    if x.table is None:
        codes[b, layers][:, :, j] = code.permute(1, 2, 0, 3)
        scales[b, layers][:, :, j] = scale.permute(1, 2, 0)
    else:
        codes[layers][:, i, j] = code.transpose(0, 1)
        scales[layers].transpose(2, 3)[:, i, j] = scale.transpose(0, 1)


def exact(case, seed):
    x = prepare(case, seed)
    kind, B, H = case["kind"], case["batch"], case["kv_heads"]
    if kind == "decode":
        G, D = case["group"], x.head_dim
        q = torch.from_numpy(_exact_turned(x, x.q, x.q_pos[:, None].expand(B, 3))).to(x.dev).view(B, H, G, D)
        out = torch.empty((B, H, G, D), dtype=torch.float64, device=x.dev)
        for b in range(B):
            n = int(x.lens[b])
            k, v = _exact_layer(x, x.k, x.k_scale, b, n), _exact_layer(x, x.v, x.v_scale, b, n)
            for h in range(H):
                out[b, h] = (q[b, h] @ k[h].T * x.scale).softmax(1) @ v[h]
        return out.view(B, H * G, D)
    if kind == "rebind" and work(case)["bytes"] > 4e8:
        return None                              # (the rows in 64 bits pass through the host)
    if kind != "read":
        k, v, ks, vs = x.k.double(), x.v.double(), x.k_scale.double(), x.v_scale.double()
        at = 0
        for b in range(B):
            if kind == "rebind":
                m = int(x.k_of[b])
                pick = x.sel_idx[at:at + m].long()
                rk, rv, pos, first = x.mem_k[b, pick], x.mem_v[b, pick], x.new_pos[at:at + m], int(x.lens[b])
                at += m
            else:
                m = int(x.n[b])
                rk, rv, pos, first = x.raw_k[b, :m], x.raw_v[b, :m], x.pos[b, :m], int(x.past[b])
            slots = first + np.arange(m)
            _exact_store(x, k, ks, b, slots, _exact_turned(x, rk, pos))
            _exact_store(x, v, vs, b, slots, rv.double().cpu().numpy())
        if kind == "rebind" or case["code"] == "e4m3":
            return k, v, ks, vs
        x.k, x.v, x.k_scale, x.v_scale = k, v, ks, vs
    rk, rv = x.read_k.double(), x.read_v.double()
    for b in range(B):
        n = int(x.lens[b])
        rk[b, 0, :, :n] = _exact_layer(x, x.k, x.k_scale, b, n)
        rv[b, 0, :, :n] = _exact_layer(x, x.v, x.v_scale, b, n)
    return rk, rv, x.k_scale.double(), x.v_scale.double()
