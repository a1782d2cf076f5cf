"""The two host routes of the operators on several tokens per sequence: the native module's call and the
Python path give the same bits, on the current stream and on another one, and what one refuses the
other refuses with the same error."""
import numpy as np
import pytest
import torch

import paper_2606_26631_amd as prcr
from gpu_util import DEV, to_dev
from paper_2606_26631_amd import binding
from test_gpu_chunk import Inputs
from test_gpu_native_calls import _Declines

B, H, G, D = 3, 2, 3, 64


def setup(block):
    x = Inputs("bf16", D, H, G, [9, 0, 40], [60, 7, 90], block, seed=3, cap=96)
    x.c = x.cache()
    x.a = x.args(x.c)
    x.n = to_dev(np.array([5, 0, 40], np.int32))
    cap = 96 if x.table is None else x.table.shape[1] * block
    x.w = torch.rand((B, H, cap), device=DEV, generator=torch.Generator(DEV).manual_seed(1))
    x.err = torch.zeros(1, dtype=torch.int32, device=DEV)
    x.mem = prcr.Memory(torch.zeros((B, 4, 2, H, D), dtype=torch.bfloat16, device=DEV), None,
                        torch.zeros((B, 4, 3), dtype=torch.int32, device=DEV), to_dev(np.full(B, 4, np.int32)),
                        to_dev(np.arange(B * 4, dtype=np.int32).reshape(B, 4) * 5))
    x.lse = torch.zeros((x.q.shape[0], H * G), device=DEV)
    return x


def calls(x, stream):
    e = dict(err=x.err, stream=stream)
    lens = x.a[6]
    return [
        ("chunk_attention", lambda: prcr.chunk_attention(*x.a, **e)),
        ("chunk_attention", lambda: prcr.chunk_attention(*x.a, q_len=x.n, scale=-0.3, **e)),
        ("key_weights", lambda: prcr.key_weights(*x.a, x.lse, **e)),
        ("key_weights", lambda: prcr.key_weights(*x.a, x.lse, q_len=x.n, window=4, scale=0.2, weights=x.w, accumulate=True, **e)),
        ("evict", lambda: prcr.evict(x.c, lens, x.w, 50, 3, 9, mem=x.mem, **e)),
        ("evict", lambda: prcr.evict(x.c, lens, x.w, 20, **e)),
    ]


@pytest.mark.gpu
@pytest.mark.parametrize("block", [0, 16])
def test_both_routes_give_the_same(monkeypatch, block):
    native, side, got = binding._native(), torch.cuda.Stream(), []
    for route in ("native", "python"):
        taken = []

        class Recorder:
            def __getattr__(self, name):
                def call(*args):
                    out = getattr(native, name)(*args)
                    taken.append((name, out is not None))
                    return out
                return call

        monkeypatch.setattr(binding, "_NATIVE", Recorder() if route == "native" else _Declines())
        for stream in (None, side):
            x = setup(block)
            torch.cuda.synchronize()
            outs = []
            for name, call in calls(x, stream):
                print(route, name, block, flush=True)
                r = call()
                torch.cuda.synchronize()
                r = [r] if not isinstance(r, tuple) else list(r)
                if name == "chunk_attention":    # (rows of no sequence are not written)
                    rows = torch.cat([torch.arange(5), torch.arange(9, 49)])
                    r = [t[rows.to(DEV)] for t in r]
                outs += [t.clone() for t in r]
            got.append(outs + [x.c.k, x.c.v, x.w, x.mem.v_slot, x.err])
        if route == "native":
            assert len(taken) == 12 and all(t for _, t in taken), taken
    for other in got[1:]:
        assert len(other) == len(got[0])
        for a, b in zip(got[0], other):
            assert a.dtype == b.dtype and torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


@pytest.mark.gpu
def test_refusals_are_the_same_on_both_routes(monkeypatch):
    """Every call is refused on the host, before a launch."""
    x = setup(0)
    rope, c, layer, q, off, pos, lens = x.a
    small = torch.zeros(8, dtype=torch.uint8, device=DEV)
    other = prcr.Memory(x.mem.k[:2], None, x.mem.coords[:2], x.mem.n_visual[:2], x.mem.v_slot[:2])
    wide = prcr.Cache(torch.zeros((1, 1, 1, 4400, D), dtype=torch.bfloat16, device=DEV),
                      torch.zeros((1, 1, 1, 4400, D), dtype=torch.bfloat16, device=DEV))
    one = to_dev(np.array([0, 2], np.int32))
    bad = [
        lambda: prcr.chunk_attention(rope, c, 2, q, off, pos, lens),
        lambda: prcr.chunk_attention(rope, c, 2 ** 32, q, off, pos, lens),
        lambda: prcr.chunk_attention(rope, c, 0, q.float(), off, pos, lens),
        lambda: prcr.chunk_attention(rope, c, 0, q[:, :5].contiguous(), off, pos, lens),
        lambda: prcr.chunk_attention(rope, c, 0, q.transpose(0, 1), off, pos, lens),
        lambda: prcr.chunk_attention(rope, c, 0, q, off[:-1], pos, lens),
        lambda: prcr.chunk_attention(rope, c, 0, q, off, pos[:-1], lens),
        lambda: prcr.chunk_attention(rope, c, 0, q, off, pos, lens.long()),
        lambda: prcr.chunk_attention(rope, c, 0, q, off, pos, lens, q_len=lens[:1]),
        lambda: prcr.chunk_attention(rope, c, 0, q, off, pos, lens, out=q),
        lambda: prcr.chunk_attention(rope, c, 0, q, off, pos, lens, lse=x.lse.half()),
        lambda: prcr.chunk_attention(rope, c, 0, q, off, pos, lens, scale=float("nan")),
        lambda: prcr.chunk_attention(prcr.Rope(128, (16, 24, 24)), c, 0, q, off, pos, lens),
        lambda: prcr.chunk_attention(rope, wide, 0, q[:2], one, pos[:2], lens[:1], workspace=small),
        lambda: prcr.key_weights(*x.a, x.lse, window=0),
        lambda: prcr.key_weights(*x.a, x.lse, window=-3),
        lambda: prcr.key_weights(*x.a, x.lse, window=2 ** 32 + 3),
        lambda: prcr.key_weights(*x.a, x.lse, accumulate=True),
        lambda: prcr.key_weights(*x.a, x.lse[:-1]),
        lambda: prcr.key_weights(*x.a, x.lse, weights=x.w[:, :, :-1]),
        lambda: prcr.key_weights(*x.a, x.lse, workspace=small),
        lambda: prcr.evict(c, lens, x.w, 0),
        lambda: prcr.evict(c, lens, x.w, 10, 6, 5),
        lambda: prcr.evict(c, lens, x.w, 10, -1),
        lambda: prcr.evict(c, lens, x.w, 2 ** 32 + 5),
        lambda: prcr.evict(c, lens, x.w, 10, 2 ** 32 - 4, 3),
        lambda: prcr.evict(c, lens, x.w.double(), 10),
        lambda: prcr.evict(c, lens, x.w, 10, new_weights=x.w),
        lambda: prcr.evict(c, lens, x.w, 10, kept=torch.zeros((B, 9), dtype=torch.int32, device=DEV)),
        lambda: prcr.evict(c, lens, x.w, 10, mem=other),
        lambda: prcr.evict(c, lens, x.w, 10, workspace=small),
    ]
    native = binding._native()
    for i, call in enumerate(bad):
        print("refusal", i, flush=True)
        said = []
        for route in (native, _Declines()):
            monkeypatch.setattr(binding, "_NATIVE", route)
            try:
                call()
                said.append(None)
            except Exception as e:      # noqa: BLE001 - whatever it is, it has to be the same
                said.append((type(e), str(e)))
        assert said[0] == said[1] and said[0] is not None, (i, said)
    torch.cuda.synchronize()


def test_native_module_declines_what_is_no_tensor_and_leaves_no_error():
    n = binding._native()
    for name, count in (("chunk_attention", 14), ("key_weights", 16), ("evict", 13)):
        for arg in (None, 1, "pcr", torch.zeros(2, 2), object(), prcr.Rope(64, (8, 12, 12))):
            assert getattr(n, name)(*[arg] * count) is None
        with pytest.raises(TypeError):
            getattr(n, name)(None)
