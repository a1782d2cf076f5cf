"""Scales and codes of the cache in 8 bits for every finite float32 as a row's largest magnitude, bit for bit as the
format's divisions give them: the kernel takes the quotient and the inverse without a division.  A row's other elements
lie next to borders between codes: an inverse that is one unit off (put into the plain form) changes a code in 97.7 to
100 % of the rows, in either direction."""
import pytest
import torch

import paper_2606_26631_amd as prcr
from gpu_util import DEV
from quant_ref import CODES, LARGEST, quantised32

pytestmark = pytest.mark.gpu

D, ROWS = 64, 1 << 21                        # rows of one call's keys, and of its values
FINITE = 0x7F800000                          # float32 magnitudes, as bits


def borders(kind):
    """The numbers halfway between neighbouring codes, where a code depends on the inverse's last bit."""
    if kind == torch.int8:
        return torch.arange(127, dtype=torch.float32) + 0.5
    codes = torch.arange(0x7F, dtype=torch.uint8).view(kind).float()
    return (codes[1:] + codes[:-1]) / 2


def quantised(x, most, kind):
    """The format in float32.  (A quotient of two float32 numbers in double, rounded to float32, is the float32 quotient:
    double has more than twice its bits and two; smaller numbers than the smallest scale are not told apart.)"""
    scale = (most.double() / LARGEST[kind]).float().clamp(min=2.0 ** -126)
    y = x * scale.double().reciprocal().float()[:, None]
    return (y.round() if kind == torch.int8 else y).to(kind), scale


@pytest.mark.parametrize("kind", sorted(CODES))
def test_every_largest_magnitude(kind):
    print(f"scales of every largest magnitude, {kind}", flush=True)
    kind = CODES[kind]
    between = borders(kind).to(DEV)
    store = [torch.zeros((1, 1, 1, ROWS, D), dtype=torch.uint8, device=DEV).view(kind) for _ in range(2)]
    scales = [torch.zeros((1, 1, 1, ROWS), device=DEV) for _ in range(2)]
    cache = prcr.QuantCache(*store, *scales)
    rope, err = prcr.Rope(D, (8, 12, 12)), torch.zeros(1, dtype=torch.int32, device=DEV)
    pos = torch.zeros((1, ROWS, 3), dtype=torch.int32, device=DEV)      # (keys are not turned)
    count, start = (torch.tensor([n], dtype=torch.int32, device=DEV) for n in (ROWS, 0))
    gen = torch.Generator(device=DEV).manual_seed(1)

    def rows(first):
        """Rows whose largest magnitudes are the numbers from `first` on, the others next to codes' borders."""
        most = torch.arange(first, first + ROWS, device=DEV).clamp(max=FINITE - 1).int().view(torch.float32)
        pick = torch.randint(len(between), (D,), generator=gen, device=DEV)
        sign = torch.randint(2, (D,), generator=gen, device=DEV) * 2.0 - 1.0
        at = int(torch.randint(D, (1,), generator=gen, device=DEV))
        scale = (most.double() / LARGEST[kind]).float().clamp(min=2.0 ** -126)
        x = torch.minimum(between[pick] * scale[:, None], most[:, None]) * sign
        x[:, at] = most * sign[at]
        return x, most

    wrong = torch.zeros((), dtype=torch.int64, device=DEV)
    for first in range(0, FINITE, 2 * ROWS):
        made = [rows(first), rows(first + ROWS)]
        prcr.quant_append(rope, cache, 0, *(x.view(1, ROWS, 1, D) for x, _ in made), pos, count, start, err=err)
        for (x, most), codes, got in zip(made, store, scales):
            code, scale = quantised(x, most, kind)
            wrong += (got[0, 0, 0].view(torch.int32) != scale.view(torch.int32)).sum()
            wrong += (codes[0, 0, 0].float() != code.float()).sum()
        if first % (256 * ROWS) == 0:           # the form used here is the tests' own
            for x, most in made:
                c, s = quantised(x[:1000], most[:1000], kind)
                code, scale = quantised32(x[:1000].cpu().numpy(), kind)
                assert (c.float().cpu().numpy() == code).all() and (s.cpu().numpy() == scale).all()
    assert int(wrong) == 0 and int(err.item()) == 0
