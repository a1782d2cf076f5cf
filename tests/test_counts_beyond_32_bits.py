"""Counts that do not fit the C interface's 32 bits are refused by the Python path, which takes every
call with such a number, and never wrapped round to another one.  (The checks come before those
of the tensors, so that these calls need none on a GPU.)"""
from types import SimpleNamespace

import pytest
import torch

import paper_2606_26631_amd as prcr

BIG = [2 ** 32, 2 ** 32 + 3, 2 ** 31, -2 ** 31 - 1, 10 ** 30]
ROPE = prcr.Rope(64, (32, 0, 0))
K = torch.zeros(1, 2, 1, 8, 64)


def cache(k=K, table=None):
    c = prcr.Cache.__new__(prcr.Cache)       # (on the host: nothing is launched on it)
    c.k, c.v, c.block_table, c.paged, c.device = k, k, table, table is not None, k.device
    return c


CALLS = {
    "layer": lambda n: [
        lambda: prcr.store_raw(None, n, None, None, None),
        lambda: prcr.prefill_capture(ROPE, None, n, None, None, None, None, None, None, None),
        lambda: prcr.decode_attention(ROPE, cache(), n, None, None, None),
        lambda: prcr.decode_attention_static(ROPE, cache(), n, None, None, None),
        lambda: prcr.chunk_attention(ROPE, cache(), n, None, None, None, None),
        lambda: prcr.key_weights(ROPE, cache(), n, None, None, None, None, None)],
    "l_ext": lambda n: [
        lambda: prcr.reassign_coords(None, None, None, None, "pcr", n),
        lambda: prcr.revisit(ROPE, None, None, None, None, None, None, "pcr", n)],
    "window": lambda n: [
        lambda: prcr.key_weights(ROPE, cache(), 0, None, None, None, None, None, window=n),
        lambda: prcr.key_weights_workspace_bytes(cache(), 4, 1, window=n)],
    "total_q": lambda n: [lambda: prcr.chunk_workspace_bytes(cache(), n, 1),
                          lambda: prcr.key_weights_workspace_bytes(cache(), n, 1)],
    "n_q_heads": lambda n: [lambda: prcr.chunk_workspace_bytes(cache(), 4, n),
                            lambda: prcr.key_weights_workspace_bytes(cache(), 4, n),
                            lambda: prcr.decode_workspace_bytes(cache(), 1, n)],
    "batch": lambda n: [lambda: prcr.decode_workspace_bytes(cache(), n, 1)],
    "budget": lambda n: [lambda: prcr.evict(cache(), None, None, n), lambda: prcr.evict_workspace_bytes(cache(), n)],
    "keep_first": lambda n: [lambda: prcr.evict(cache(), None, None, 4, n)],
    "keep_last": lambda n: [lambda: prcr.evict(cache(), None, None, 4, 0, n)],
    "sections": lambda n: [lambda: prcr.Rope(64, (32, n, 0)).inv_freq(), lambda: prcr.Rope(64, (n, 0, 0)).to_c()],
    "head_dim": lambda n: [lambda: prcr.Rope(n, (32, 0, 0)).to_c()],
}


@pytest.mark.parametrize("n", BIG)
@pytest.mark.parametrize("what", sorted(CALLS))
def test_refused(what, n):
    for call in CALLS[what](n):
        with pytest.raises(ValueError, match=f"{what} .*32 bits"):
            call()


@pytest.mark.parametrize("n", [2 ** 31 - 1, -2 ** 31])
@pytest.mark.parametrize("what", ["layer", "window", "budget", "l_ext"])
def test_the_largest_are_left_to_the_other_checks(what, n):
    for call in CALLS[what](n):
        try:
            call()
        except Exception as e:
            assert "32 bits" not in str(e)


def test_sizes_of_tensors():
    """A table wider, or a selection longer, than 2^31 (of memory that is never touched)."""
    wide = torch.empty(1, dtype=torch.int32).expand(1, 2 ** 32 + 3)
    with pytest.raises(ValueError, match="32 bits"):
        cache(table=wide).to_c()
    m = SimpleNamespace(k=K)
    k = SimpleNamespace(shape=(1, 2 ** 32 + 9, 1, 1, 64), data_ptr=lambda: 0, dtype=torch.float32)
    m.v, m.coords, m.n_visual, m.v_slot, m.k = None, K, K, K, k
    with pytest.raises(ValueError, match="32 bits"):
        prcr.Memory.to_c(m)
