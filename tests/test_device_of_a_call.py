"""Every call is made with its tensors' GPU as the current one: torch's default stream is given to the C interface as a
null pointer, which stands for the current device's.  On the host, by the Python path, with the C library and torch's
notion of a current GPU replaced (the tensors are the host's, and nothing is launched)."""
import contextlib

import pytest
import torch

import paper_2606_26631_amd as prcr
from paper_2606_26631_amd import binding
from test_gpu_native_calls import _Declines

B, M, NL, H, D, S = 2, 6, 2, 1, 64, 32


class Gpu:
    """The current device, and the C calls made meanwhile."""

    def __init__(self):
        self.current, self.calls = ["another GPU"], []

    @contextlib.contextmanager
    def device(self, d):
        self.current.append(d)
        yield
        self.current.pop()

    def __getattr__(self, name):                # the C library's functions
        if name.endswith("_size"):
            return getattr(self.lib, name)

        def call(*args):
            self.calls.append((name, self.current[-1], args[-1].value))
            return 0
        return call


@pytest.fixture
def gpu(monkeypatch):
    g = Gpu()
    g.lib = binding.lib()
    stream = type("Stream", (), {"cuda_stream": 0})
    monkeypatch.setattr(binding, "lib", lambda: g)
    monkeypatch.setattr(binding, "_NATIVE", _Declines())
    monkeypatch.setattr(binding, "_need", lambda *a, **k: None)
    monkeypatch.setattr(torch.cuda, "device", g.device)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda d=None: stream())
    return g


def calls():
    ints = lambda *s: torch.zeros(s, dtype=torch.int32)
    rows = lambda *s: torch.zeros(s)
    rope = prcr.Rope(D, (8, 12, 12))
    mem = prcr.Memory(rows(B, M, NL, H, D), rows(B, M, NL, H, D), ints(B, M, 3), ints(B))
    cache = prcr.Cache(rows(B, NL, H, S, D), rows(B, NL, H, S, D))
    codes = lambda: torch.zeros(B, NL, H, S, D, dtype=torch.int8)
    cache8 = prcr.QuantCache(codes(), codes(), rows(B, NL, H, S), rows(B, NL, H, S))
    sel = (ints(B + 1), ints(3))
    new_pos = torch.zeros(3, 3, dtype=torch.float64)
    k, q = rows(B, 4, H, D), rows(B, 2, D)
    rows_of = (q, ints(B + 1), ints(B, 3), ints(B))
    return {
        "prcr_store_raw": lambda: prcr.store_raw(mem, 0, k, k, ints(B, M)),
        "prcr_reassign_coords": lambda: prcr.reassign_coords(mem, *sel, ints(B)),
        "prcr_rebind_inject": lambda: prcr.rebind_inject(rope, mem, *sel, new_pos, cache, ints(B)),
        "prcr_revisit": lambda: prcr.revisit(rope, mem, *sel, ints(B), cache, ints(B)),
        "prcr_prefill_capture": lambda: prcr.prefill_capture(rope, mem, 0, k, k, ints(B, 4, 3), ints(B), ints(B, 4), cache,
                                                             ints(B)),
        "prcr_decode_attention": lambda: prcr.decode_attention(rope, cache, 0, q, ints(B), ints(B)),
        "prcr_decode_attention_static": lambda: prcr.decode_attention_static(rope, cache, 0, q, ints(B), ints(B)),
        "prcr_chunk_attention": lambda: prcr.chunk_attention(rope, cache, 0, *rows_of),
        "prcr_key_weights": lambda: prcr.key_weights(rope, cache, 0, *rows_of, rows(B, 2)),
        "prcr_evict": lambda: prcr.evict(cache, ints(B), rows(B, H, S), 4),
        "prcr_quant_append": lambda: prcr.quant_append(rope, cache8, 0, k, k, ints(B, 4, 3), ints(B), ints(B)),
        "prcr_quant_rebind_inject": lambda: prcr.quant_rebind_inject(rope, mem, *sel, new_pos, cache8, ints(B)),
        "prcr_quant_read": lambda: prcr.quant_read(cache8, 0, ints(B), torch.float32),
        "prcr_quant_decode_attention": lambda: prcr.quant_decode_attention(rope, cache8, 0, q, ints(B), ints(B)),
    }


def test_the_tensors_gpu_is_current_in_every_call(gpu):
    todo = calls()
    for name, call in todo.items():
        call()
        assert gpu.calls[-1] == (name, torch.device("cpu"), None), gpu.calls[-1]
    assert len(gpu.calls) == len(todo) and gpu.current == ["another GPU"]
    # (Every C call on a stream is among them.)
    on_stream = {n for n in dir(prcr) if callable(getattr(prcr, n)) and not n.endswith("bytes")}
    on_stream -= {"Cache", "Memory", "Rope", "QuantCache", "PrcrError", "lib"}
    assert {f"prcr_{n}" for n in on_stream} == set(todo)


def test_a_cache_on_another_device_than_the_memory_is_refused(gpu):
    """(The meta device stands for another GPU.)"""
    ints = lambda *s: torch.zeros(s, dtype=torch.int32)
    rope, rows = prcr.Rope(D, (8, 12, 12)), torch.zeros(B, M, NL, H, D)
    mem = prcr.Memory(rows, rows, ints(B, M, 3), ints(B))
    far = lambda *s, dtype=torch.float32: torch.zeros(s, dtype=dtype, device="meta")
    sel, new_pos, k = (ints(B + 1), ints(3)), torch.zeros(3, 3, dtype=torch.float64), torch.zeros(B, 4, H, D)
    cache = prcr.Cache(far(B, NL, H, S, D), far(B, NL, H, S, D))
    cache8 = prcr.QuantCache(*(far(B, NL, H, S, D, dtype=torch.int8) for _ in range(2)), *(far(B, NL, H, S) for _ in range(2)))
    for call in (lambda: prcr.rebind_inject(rope, mem, *sel, new_pos, cache, ints(B)),
                 lambda: prcr.revisit(rope, mem, *sel, ints(B), cache, ints(B)),
                 lambda: prcr.prefill_capture(rope, mem, 0, k, k, ints(B, 4, 3), ints(B), ints(B, 4), cache, ints(B)),
                 lambda: prcr.quant_rebind_inject(rope, mem, *sel, new_pos, cache8, ints(B)),
                 lambda: prcr.evict(cache, ints(B), far(B, H, S), 4, mem=mem)):
        with pytest.raises(ValueError, match="is on .*, expected"):
            call()
    assert not gpu.calls
