"""What the operators on several tokens per sequence refuse, on the host, before any HIP call:
every call here has placeholder pointers and must return its error code."""
import ctypes

import pytest

import paper_2606_26631_amd as prcr
from paper_2606_26631_amd.binding import CCache, CMem, CRope
from test_abi import host_only

pytestmark = host_only

NULL, SHAPE, DTYPE, ALIGN, UNSUPPORTED, ALIAS = 1, 2, 3, 4, 6, 7
MB = 1 << 20
AT = {n: (i + 1) << 40 for i, n in enumerate(
    ["k", "v", "table", "q", "q_off", "q_len", "q_pos", "cache_len", "out", "lse", "ws", "err", "weights", "new_len",
     "kept", "new_weights", "v_slot"])}


def rope(D=128, sections=(16, 24, 24), inter=0, theta=1e6):
    return CRope(D, (ctypes.c_int32 * 3)(*sections), inter, theta)


def contiguous(s_max=512, **kw):
    return CCache(0, kw.get("k", AT["k"]), kw.get("v", AT["v"]), s_max, None, 0, 0, 0)


def paged(bs=16, max_blocks=32, n_blocks=100, table=AT["table"]):
    return CCache(1, AT["k"], AT["v"], 0, table, bs, max_blocks, n_blocks)


def attend(fn, **kw):
    a = dict(rope=rope(), cache=contiguous(), dtype=1, batch=2, n_layers=3, n_kv_heads=4, layer=1, n_q_heads=28,
             total_q=10, scale=0.1, window=0, accumulate=0, bytes=1 << 33)
    a |= {n: AT[n] for n in ("q", "q_off", "q_len", "q_pos", "cache_len", "out", "lse", "ws", "err", "weights")}
    a |= kw
    ref = lambda x: None if x is None else ctypes.byref(x)
    head = [ref(a["rope"]), ref(a["cache"]), a["dtype"], a["batch"], a["n_layers"], a["n_kv_heads"], a["layer"], a["q"],
            a["n_q_heads"], a["q_off"], a["q_len"], a["total_q"], a["q_pos"], a["cache_len"]]
    L = prcr.lib()
    if fn == "chunk":
        return L.prcr_chunk_attention(*head, a["scale"], a["out"], a["lse"], a["ws"], a["bytes"], a["err"], None)
    return L.prcr_key_weights(*head, a["lse"], a["window"], a["scale"], a["accumulate"], a["weights"], a["ws"], a["bytes"],
                              a["err"], None)


BOTH = [
    (dict(rope=None), NULL), (dict(cache=None), NULL), (dict(q=None), NULL), (dict(q_off=None), NULL),
    (dict(q_pos=None), NULL), (dict(cache_len=None), NULL), (dict(cache=contiguous(k=None)), NULL),
    (dict(cache=contiguous(v=None)), NULL), (dict(cache=paged(table=None)), NULL),
    (dict(dtype=2), DTYPE), (dict(dtype=-1), DTYPE),
    (dict(batch=0), SHAPE), (dict(batch=65536), SHAPE), (dict(n_kv_heads=0), SHAPE), (dict(n_q_heads=27), SHAPE),
    (dict(n_q_heads=0), SHAPE), (dict(total_q=-1), SHAPE), (dict(total_q=1 << 26), SHAPE), (dict(layer=-1), SHAPE),
    (dict(layer=3), SHAPE), (dict(n_layers=0), SHAPE), (dict(scale=float("nan")), SHAPE), (dict(scale=float("inf")), SHAPE),
    (dict(cache=contiguous(0)), SHAPE), (dict(cache=contiguous((1 << 30) + 1)), SHAPE), (dict(cache=paged(bs=0)), SHAPE),
    (dict(cache=paged(max_blocks=1 << 30)), SHAPE), (dict(cache=paged(n_blocks=0)), SHAPE),
    (dict(rope=rope(sections=(16, 24, 23))), SHAPE), (dict(rope=rope(theta=-1.0)), SHAPE),
    (dict(rope=rope(32, (16, 0, 0))), UNSUPPORTED), (dict(rope=rope(sections=(32, 16, 16))), UNSUPPORTED),
    (dict(q=AT["q"] + 8), ALIGN), (dict(q_off=AT["q_off"] + 2), ALIGN), (dict(q_len=AT["q_len"] + 1), ALIGN),
    (dict(q_pos=AT["q_pos"] + 2), ALIGN), (dict(cache_len=AT["cache_len"] + 1), ALIGN), (dict(ws=AT["ws"] + 8), ALIGN),
    (dict(err=AT["err"] + 2), ALIGN), (dict(lse=AT["lse"] + 2), ALIGN), (dict(cache=contiguous(k=AT["k"] + 8)), ALIGN),
]


@pytest.mark.parametrize("fn", ["chunk", "weights"])
@pytest.mark.parametrize("case", range(len(BOTH)))
def test_both(fn, case):
    kw, want = BOTH[case]
    assert attend(fn, **kw) == want


@pytest.mark.parametrize("kw,want", [
    (dict(out=None), NULL), (dict(ws=None), NULL), (dict(bytes=0), SHAPE), (dict(out=AT["out"] + 8), ALIGN),
    (dict(out=AT["q"]), ALIAS), (dict(out=AT["k"] + 16), ALIAS), (dict(lse=AT["out"] + 256), ALIAS),
    (dict(ws=AT["v"]), ALIAS), (dict(lse=AT["q_off"] + 8), ALIAS), (dict(out=AT["cache_len"] - 16), ALIAS),
    (dict(cache=paged(max_blocks=256), ws=AT["table"] + 128), ALIAS), (dict(out=AT["q_pos"]), ALIAS), (dict(lse=AT["q_len"]), ALIAS)])
def test_chunk(kw, want):
    kw = dict(total_q=10, cache=contiguous(4096)) | kw   # (few rows, many slots: the keys are split)
    assert attend("chunk", **kw) == want


@pytest.mark.parametrize("kw,want", [
    (dict(weights=None), NULL), (dict(lse=None), NULL), (dict(ws=None), NULL), (dict(window=-1), SHAPE),
    (dict(bytes=10 * 28 * 256 - 1), SHAPE), (dict(weights=AT["weights"] + 2), ALIGN), (dict(weights=AT["lse"]), ALIAS),
    (dict(weights=AT["q"]), ALIAS), (dict(weights=AT["k"]), ALIAS), (dict(ws=AT["q"] + 16), ALIAS),
    (dict(weights=AT["cache_len"]), ALIAS), (dict(ws=AT["weights"] + 64), ALIAS)])
def test_weights(kw, want):
    assert attend("weights", **kw) == want


def test_nothing_to_do():
    """No rows: nothing is launched, and the rows' pointers may be missing."""
    assert attend("chunk", total_q=0, q=None, q_pos=None, out=None, ws=None, lse=None) == 0
    assert attend("weights", total_q=0, q=None, q_pos=None, lse=None, ws=None, accumulate=1) == 0


def evict(**kw):
    a = dict(cache=contiguous(), dtype=1, batch=2, n_layers=3, n_kv_heads=4, head_dim=128, budget=100, first=4, last=20,
             mem=None, bytes=1 << 33)
    a |= {n: AT[n] for n in ("cache_len", "weights", "new_len", "kept", "new_weights", "ws", "err")}
    a |= kw
    ref = lambda x: None if x is None else ctypes.byref(x)
    return prcr.lib().prcr_evict(ref(a["cache"]), a["dtype"], a["batch"], a["n_layers"], a["n_kv_heads"], a["head_dim"],
                                 a["cache_len"], a["weights"], a["budget"], a["first"], a["last"], a["new_len"], a["kept"],
                                 a["new_weights"], ref(a["mem"]), a["ws"], a["bytes"], a["err"], None)


def memory(batch=2, max_visual=9, v=None, v_slot=AT["v_slot"]):
    return CMem(AT["q"], v, AT["q_pos"], AT["q_len"], batch, max_visual, 3, 4, 128, 1, v_slot)


@pytest.mark.parametrize("kw,want", [
    (dict(cache=None), NULL), (dict(cache_len=None), NULL), (dict(weights=None), NULL), (dict(new_len=None), NULL),
    (dict(kept=None), NULL), (dict(ws=None), NULL), (dict(mem=memory(v_slot=None)), NULL), (dict(dtype=5), DTYPE),
    (dict(batch=0), SHAPE), (dict(n_layers=0), SHAPE), (dict(budget=0), SHAPE), (dict(first=-1), SHAPE),
    (dict(last=-1), SHAPE), (dict(first=50, last=51), SHAPE), (dict(first=2 ** 31 - 1, last=2 ** 31 - 1), SHAPE),
    (dict(bytes=2 * 513 * 4 - 1), SHAPE), (dict(mem=memory(batch=3)), SHAPE), (dict(mem=memory(max_visual=0)), SHAPE),
    (dict(head_dim=96), UNSUPPORTED), (dict(ws=AT["ws"] + 4), ALIGN), (dict(weights=AT["weights"] + 2), ALIGN),
    (dict(kept=AT["kept"] + 2), ALIGN), (dict(mem=memory(v_slot=AT["v_slot"] + 2)), ALIGN),
    (dict(kept=AT["cache_len"]), ALIAS), (dict(new_weights=AT["weights"]), ALIAS), (dict(new_len=AT["cache_len"] + 4), ALIAS),
    (dict(weights=AT["k"]), ALIAS), (dict(cache=contiguous(v=AT["k"])), ALIAS), (dict(ws=AT["kept"]), ALIAS),
    (dict(cache=paged(), kept=AT["table"]), ALIAS), (dict(mem=memory(v_slot=AT["cache_len"])), ALIAS)])
def test_evict(kw, want):
    assert evict(**kw) == want


@pytest.mark.parametrize("kw", [dict(budget=(1 << 30) + 1), dict(budget=2 ** 31 - 1),
                                dict(mem=memory(max_visual=(1 << 30) + 1)), dict(mem=memory(max_visual=2 ** 31 - 1))])
def test_evict_counts_beyond_the_largest(kw):
    """Counts that a loop's 32-bit index could run past."""
    assert evict(bytes=1 << 40, **kw) == SHAPE
    n = ctypes.c_size_t()
    if "budget" in kw:
        assert prcr.lib().prcr_evict_workspace_size(ctypes.byref(contiguous()), 2, kw["budget"], ctypes.byref(n)) == SHAPE


@pytest.mark.parametrize("fn", ["chunk", "weights"])
@pytest.mark.parametrize("scale", [3e38, -3e38])
def test_scale_without_a_finite_base_two_form(fn, scale):
    assert attend(fn, scale=scale) == SHAPE


def test_workspace_sizes():
    L, n = prcr.lib(), ctypes.c_size_t()
    c, p = contiguous(), paged()
    assert L.prcr_chunk_workspace_size(ctypes.byref(c), 2, 10, 28, 4, 128, None) == NULL
    assert L.prcr_chunk_workspace_size(None, 2, 10, 28, 4, 128, ctypes.byref(n)) == NULL
    assert L.prcr_key_weights_workspace_size(ctypes.byref(c), 7, 2, 10, 28, 4, 128, 0, ctypes.byref(n)) == DTYPE
    assert L.prcr_chunk_workspace_size(ctypes.byref(c), 2, 10, 27, 4, 128, ctypes.byref(n)) == SHAPE
    assert L.prcr_chunk_workspace_size(ctypes.byref(c), 2, 10, 28, 4, 96, ctypes.byref(n)) == UNSUPPORTED
    assert L.prcr_key_weights_workspace_size(ctypes.byref(c), 1, 2, 10, 28, 4, 128, -1, ctypes.byref(n)) == SHAPE
    assert L.prcr_key_weights_workspace_size(ctypes.byref(c), 1, 2, 10, 28, 4, 128, 0, ctypes.byref(n)) == 0
    assert n.value >= 10 * 28 * 256
    assert L.prcr_evict_workspace_size(ctypes.byref(c), 2, 0, ctypes.byref(n)) == SHAPE
    assert L.prcr_evict_workspace_size(ctypes.byref(p), 2, 100, ctypes.byref(n)) == 0
    assert n.value == 2 * (100 * 8 + 513 * 4)
