"""The attention calls refuse a rope whose head_dim is not the cache's: the C calls take the length of the
cache's rows from the rope alone."""
import pytest
import torch

import paper_2606_26631_amd as prcr
from paper_2606_26631_amd import binding
from test_gpu_native_calls import _Declines

B, NL, H, S = 2, 1, 2, 32
ROPES = {64: (64, (8, 12, 12)), 128: (128, (16, 24, 24))}


def calls(rope, cache, q, q3, off, pos, pos3, lens, lse):
    return {
        "decode_attention": lambda: prcr.decode_attention(rope, cache, 0, q, pos, lens),
        "decode_attention_static": lambda: prcr.decode_attention_static(rope, cache, 0, q, pos, lens),
        "chunk_attention": lambda: prcr.chunk_attention(rope, cache, 0, q3, off, pos3, lens),
        "key_weights": lambda: prcr.key_weights(rope, cache, 0, q3, off, pos3, lens, lse),
    }


def inputs(D, device, cache):
    ints = lambda *a: torch.tensor(a, dtype=torch.int32, device=device)
    q = torch.zeros(B, 2 * H, D, device=device)
    return (cache, q, q.clone(), ints(0, 1, 2), ints(3, 4), torch.zeros(2, 3, dtype=torch.int32, device=device),
            ints(20, 9), torch.zeros(2, 2 * H, device=device))


NAMES = ["decode_attention", "decode_attention_static", "chunk_attention", "key_weights"]


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("rope_dim,D", [(128, 64), (64, 128)])
def test_refused_before_anything_else(name, paged, rope_dim, D):
    cache = prcr.Cache.__new__(prcr.Cache)      # (on the host: nothing is launched on it)
    cache.k = cache.v = torch.zeros((NL, 4, 16, H, D) if paged else (B, NL, H, S, D))
    cache.block_table = torch.zeros(B, 2, dtype=torch.int32) if paged else None
    cache.paged, cache.device = paged, cache.k.device
    with pytest.raises(ValueError, match="rope head_dim differs"):
        calls(prcr.Rope(*ROPES[rope_dim]), *inputs(D, "cpu", cache))[name]()


@pytest.mark.gpu
@pytest.mark.parametrize("name", NAMES)
def test_refused_by_both_routes(monkeypatch, name):
    """(With a rope shorter than the rows, which stay within the cache's memory whatever is called.)"""
    print("rope of another head_dim", name, flush=True)
    cache = prcr.Cache(*(torch.zeros(B, NL, H, S, 128, device="cuda") for _ in range(2)))
    x = inputs(128, "cuda", cache)
    native = binding._native()
    for route in (native, _Declines()):
        monkeypatch.setattr(binding, "_NATIVE", route)
        calls(prcr.Rope(*ROPES[128]), *x)[name]()
        with pytest.raises(ValueError, match="rope head_dim differs"):
            calls(prcr.Rope(*ROPES[64]), *x)[name]()
