"""What the operators on the cache in 8 bits refuse, on the host, before any HIP call: every call here has
placeholder pointers, or tensors on the host, and must return or raise its error."""
import ctypes

import pytest
import torch

import paper_2606_26631_amd as prcr
from paper_2606_26631_amd.binding import CCache, CMem, CQuantCache, CRope
from test_abi import host_only

NULL, SHAPE, DTYPE, ALIGN, UNSUPPORTED, ALIAS = 1, 2, 3, 4, 6, 7
NAMES = ["k", "v", "ks", "vs", "table", "raw_k", "raw_v", "pos", "n", "start", "err", "q", "q_pos", "len", "out", "ws", "mem_k",
         "mem_v", "coords", "n_visual", "v_slot", "off", "idx", "new_pos", "new_len", "slots", "out_k", "out_v"]
AT = {n: (i + 1) << 40 for i, n in enumerate(NAMES)}
ref = lambda x: None if x is None else ctypes.byref(x)


def rope(D=128, sections=(16, 24, 24), inter=0, theta=1e6):
    return CRope(D, (ctypes.c_int32 * 3)(*sections), inter, theta)


def cache(s_max=512, code=0, paged=0, bs=16, max_blocks=32, n_blocks=100, **kw):
    a = {n: AT[n] for n in ("k", "v", "ks", "vs", "table")} | kw
    return CQuantCache(CCache(paged, a["k"], a["v"], 0 if paged == 1 else s_max, a["table"] if paged else None, bs, max_blocks, n_blocks),
                       a["ks"], a["vs"], code)


def memory(**kw):
    a = dict(k=AT["mem_k"], v=AT["mem_v"], n_visual=AT["n_visual"], batch=2, M=100, NL=3, H=4, D=128, dtype=1, v_slot=None) | kw
    return CMem(a["k"], a["v"], AT["coords"], a["n_visual"], a["batch"], a["M"], a["NL"], a["H"], a["D"], a["dtype"], a["v_slot"])


def call(fn, **kw):
    a = dict(rope=rope(), cache=cache(), dtype=1, batch=2, n_layers=3, H=4, layer=1, S=10, D=128, Hq=28, scale=0.1, total_k=9,
             bytes=1 << 40, mem=memory(), s_out=512) | {n: AT[n] for n in NAMES} | kw
    L = prcr.lib()
    if fn == "append":
        return L.prcr_quant_append(ref(a["rope"]), ref(a["cache"]), a["dtype"], a["batch"], a["n_layers"], a["H"], a["layer"],
                                   a["raw_k"], a["raw_v"], a["S"], a["pos"], a["n"], a["start"], a["err"], None)
    if fn == "read":
        return L.prcr_quant_read(ref(a["cache"]), a["dtype"], a["batch"], a["n_layers"], a["H"], a["D"], a["layer"], a["len"],
                                 a["out_k"], a["out_v"], a["s_out"], a["err"], None)
    if fn == "decode":
        return L.prcr_quant_decode_attention(ref(a["rope"]), ref(a["cache"]), a["dtype"], a["batch"], a["n_layers"], a["H"], a["layer"],
                                             a["q"], a["Hq"], a["q_pos"], a["len"], a["scale"], a["out"], a["ws"], a["bytes"],
                                             a["err"], None)
    return L.prcr_quant_rebind_inject(ref(a["rope"]), ref(a["mem"]), a["off"], a["idx"], a["total_k"], a["new_pos"], ref(a["cache"]),
                                      a["len"], a["new_len"], a["slots"], a["err"], None)


CACHES = [
    (None, NULL), (cache(k=None), NULL), (cache(v=None), NULL), (cache(ks=None), NULL), (cache(vs=None), NULL),
    (cache(paged=1, table=None), NULL), (cache(code=2), DTYPE), (cache(code=-1), DTYPE), (cache(paged=2), SHAPE), (cache(0), SHAPE),
    (cache((1 << 30) + 1), SHAPE), (cache(paged=1, bs=0), SHAPE), (cache(paged=1, max_blocks=0), SHAPE),
    (cache(paged=1, n_blocks=0), SHAPE), (cache(paged=1, max_blocks=1 << 30), SHAPE), (cache(k=AT["k"] + 8), ALIGN),
    (cache(v=AT["v"] + 4), ALIGN), (cache(ks=AT["ks"] + 2), ALIGN), (cache(vs=AT["vs"] + 1), ALIGN),
    (cache(paged=1, table=AT["table"] + 2), ALIGN)]


@host_only
@pytest.mark.parametrize("fn", ["append", "read", "decode", "rebind"])
@pytest.mark.parametrize("i", range(len(CACHES)))
def test_caches(fn, i):
    c, want = CACHES[i]
    assert call(fn, cache=c) == want


SHAPES = [(dict(dtype=2), DTYPE), (dict(dtype=-1), DTYPE), (dict(batch=0), SHAPE), (dict(batch=65536), SHAPE), (dict(n_layers=0), SHAPE),
          (dict(H=0), SHAPE), (dict(H=65536), SHAPE), (dict(layer=-1), SHAPE), (dict(layer=3), SHAPE), (dict(err=AT["err"] + 2), ALIGN),
          (dict(n_layers=1 << 30, layer=0), SHAPE)]


@host_only
@pytest.mark.parametrize("fn", ["append", "read", "decode"])
@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_shapes(fn, i):
    kw, want = SHAPES[i]
    assert call(fn, **kw) == want


@host_only
@pytest.mark.parametrize("fn", ["append", "decode", "rebind"])
@pytest.mark.parametrize("r,want", [(None, NULL), (rope(sections=(16, 24, 23)), SHAPE), (rope(theta=-1.0), SHAPE), (rope(inter=2), SHAPE),
                                    (rope(32, (16, 0, 0)), UNSUPPORTED), (rope(sections=(32, 16, 16)), UNSUPPORTED)])
def test_ropes(fn, r, want):
    assert call(fn, rope=r) == want


@host_only
@pytest.mark.parametrize("kw,want", [
    (dict(raw_k=None), NULL), (dict(raw_v=None), NULL), (dict(pos=None), NULL), (dict(n=None), NULL), (dict(start=None), NULL),
    (dict(S=0), SHAPE), (dict(S=1 << 30), SHAPE), (dict(raw_k=AT["raw_k"] + 8), ALIGN), (dict(raw_v=AT["raw_v"] + 2), ALIGN),
    (dict(pos=AT["pos"] + 2), ALIGN), (dict(n=AT["n"] + 1), ALIGN), (dict(start=AT["start"] + 2), ALIGN),
    (dict(raw_k=AT["k"]), ALIAS), (dict(raw_v=AT["v"] + 16), ALIAS), (dict(pos=AT["ks"]), ALIAS), (dict(n=AT["vs"] + 4), ALIAS),
    (dict(start=AT["k"] + 64), ALIAS), (dict(cache=cache(v=AT["k"])), ALIAS), (dict(cache=cache(vs=AT["ks"] + 4)), ALIAS),
    (dict(cache=cache(ks=AT["k"])), ALIAS), (dict(cache=cache(paged=1, table=AT["v"])), ALIAS)])
def test_append(kw, want):
    assert call("append", **kw) == want


@host_only
@pytest.mark.parametrize("kw,want", [
    (dict(len=None), NULL), (dict(out_k=None), NULL), (dict(out_v=None), NULL), (dict(s_out=0), SHAPE), (dict(s_out=(1 << 30) + 1), SHAPE),
    (dict(D=96), UNSUPPORTED), (dict(out_k=AT["out_k"] + 8), ALIGN), (dict(len=AT["len"] + 2), ALIGN), (dict(out_k=AT["out_v"] + 16), ALIAS),
    (dict(out_k=AT["k"]), ALIAS), (dict(out_v=AT["vs"]), ALIAS), (dict(out_v=AT["len"]), ALIAS),
    (dict(cache=cache(paged=1), out_k=AT["table"]), ALIAS)])
def test_read(kw, want):
    assert call("read", **kw) == want


@host_only
@pytest.mark.parametrize("kw,want", [
    (dict(q=None), NULL), (dict(q_pos=None), NULL), (dict(len=None), NULL), (dict(out=None), NULL), (dict(ws=None), NULL),
    (dict(Hq=27), SHAPE), (dict(Hq=36), SHAPE), (dict(Hq=0), SHAPE), (dict(bytes=1000), SHAPE), (dict(scale=float("nan")), SHAPE),
    (dict(scale=float("inf")), SHAPE), (dict(scale=-3e38), SHAPE), (dict(q=AT["q"] + 8), ALIGN), (dict(q_pos=AT["q_pos"] + 2), ALIGN),
    (dict(len=AT["len"] + 1), ALIGN), (dict(out=AT["out"] + 2), ALIGN), (dict(ws=AT["ws"] + 2), ALIGN), (dict(out=AT["q"]), ALIAS),
    (dict(out=AT["len"]), ALIAS), (dict(ws=AT["k"]), ALIAS), (dict(out=AT["ws"] + 64), ALIAS), (dict(ws=AT["ks"]), ALIAS),
    (dict(cache=cache(paged=1), ws=AT["table"]), ALIAS)])
def test_decode(kw, want):
    assert call("decode", **kw) == want


@host_only
@pytest.mark.parametrize("kw,want", [
    (dict(mem=None), NULL), (dict(mem=memory(k=None)), NULL), (dict(mem=memory(n_visual=None)), NULL), (dict(mem=memory(v=None)), NULL),
    (dict(off=None), NULL), (dict(idx=None), NULL), (dict(new_pos=None), NULL), (dict(len=None), NULL), (dict(mem=memory(dtype=3)), DTYPE),
    (dict(mem=memory(batch=0)), SHAPE), (dict(mem=memory(M=0)), SHAPE), (dict(mem=memory(D=64)), SHAPE), (dict(total_k=-1), SHAPE),
    (dict(mem=memory(k=AT["mem_k"] + 8)), ALIGN), (dict(mem=memory(v=None, v_slot=AT["v_slot"] + 2)), ALIGN),
    (dict(off=AT["off"] + 2), ALIGN), (dict(idx=AT["idx"] + 2), ALIGN), (dict(new_pos=AT["new_pos"] + 4), ALIGN),
    (dict(len=AT["len"] + 2), ALIGN), (dict(new_len=AT["new_len"] + 2), ALIGN), (dict(slots=AT["slots"] + 4), ALIGN),
    (dict(new_len=AT["len"]), ALIAS), (dict(new_len=AT["off"] + 8), ALIAS), (dict(slots=AT["new_pos"]), ALIAS),
    (dict(mem=memory(k=AT["k"])), ALIAS), (dict(cache=cache(vs=AT["mem_v"])), ALIAS), (dict(slots=AT["new_len"]), ALIAS),
    (dict(mem=memory(v=None, v_slot=AT["slots"])), ALIAS)])
def test_rebind(kw, want):
    assert call("rebind", **kw) == want


@host_only
def test_workspace_size():
    L, n = prcr.lib(), ctypes.c_size_t()
    f = L.prcr_quant_decode_workspace_size
    assert f(ctypes.byref(cache()), 2, 28, 4, 128, None) == NULL
    assert f(None, 2, 28, 4, 128, ctypes.byref(n)) == NULL
    assert f(ctypes.byref(cache(code=9)), 2, 28, 4, 128, ctypes.byref(n)) == DTYPE
    assert f(ctypes.byref(cache()), 2, 27, 4, 128, ctypes.byref(n)) == SHAPE
    assert f(ctypes.byref(cache()), 2, 28, 4, 96, ctypes.byref(n)) == UNSUPPORTED
    assert f(ctypes.byref(cache()), 2, 28, 4, 128, ctypes.byref(n)) == 0 and n.value >= 2 * 28 * 130 * 4


# ------------------------------------------------------------------ the Python classes
def host_cache(kind=torch.int8, **kw):
    """A cache on the host (nothing is launched on it)."""
    c = prcr.QuantCache.__new__(prcr.QuantCache)
    c.k = c.v = torch.zeros(1, 2, 1, 8, 64, dtype=torch.uint8).view(kind)
    c.k_scale = c.v_scale = torch.zeros(1, 2, 1, 8)
    c.block_table, c.paged, c.device = None, False, c.k.device
    return c


@pytest.mark.parametrize("n", [2 ** 32, 2 ** 31, -2 ** 31 - 1, 10 ** 30])
def test_numbers_beyond_32_bits(n):
    r, c = prcr.Rope(64, (32, 0, 0)), host_cache()
    for f in (lambda: prcr.quant_append(r, c, n, None, None, None, None, None),
              lambda: prcr.quant_read(c, n, None, torch.float32),
              lambda: prcr.quant_decode_attention(r, c, n, None, None, None),
              lambda: prcr.quant_decode_workspace_bytes(c, n)):
        with pytest.raises(ValueError, match="32 bits"):
            f()


@pytest.mark.parametrize("dtype", [torch.float16, torch.float64, torch.int8, None, "bf16"])
def test_read_types(dtype):
    with pytest.raises(ValueError, match="element type"):
        prcr.quant_read(host_cache(), 0, None, dtype)


def test_tensors_on_the_host_are_refused():
    c, s = torch.zeros(1, 2, 1, 8, 64, dtype=torch.int8), torch.zeros(1, 2, 1, 8)
    with pytest.raises(ValueError, match="GPU"):
        prcr.QuantCache(c, c, s, s)
    r = prcr.Rope(64, (32, 0, 0))
    for f in (lambda: prcr.quant_append(r, host_cache(), 0, torch.zeros(1, 1, 1, 64), None, None, None, None),
              lambda: prcr.quant_read(host_cache(), 0, torch.zeros(1, dtype=torch.int32), torch.float32),
              lambda: prcr.quant_decode_attention(r, host_cache(), 0, torch.zeros(1, 1, 64), None, None)):
        with pytest.raises(ValueError, match="GPU"):
            f()
