"""CPU-only: what rounding to 8-bit floats again, along the other way, changes, and what is said of it."""

import re

import torch

import f8_reference as ref
from paper_1803_03288_amd import layers


def stated():
    """The bound that ``linear_f8_backward`` states, a part of a block's largest value."""
    return 2.0 ** int(re.search(r"values of 2\^(-\d+) of a block's", " ".join(layers.linear_f8_backward.__doc__.split())).group(1))


def again(x):
    """The values that blocks of rows keep of values that blocks of columns have kept."""
    q, scale, _ = ref.blocks(x)
    kept = q * scale
    q, scale, _ = ref.blocks(ref.along(kept))
    return kept, ref.along(q * scale)


def test_the_largest_value_that_changes():
    """A block whose largest is 240 keeps the scale 1; 1.875 * 2^-7, exact in its own row, is 2^-14 of that and between two values of the type."""
    x = torch.zeros(128, 1)
    x[0], x[1] = 240.0, 1.875 * 2.0 ** -7
    kept, now = again(x)
    assert torch.equal(kept, x.double())                    # (a scale for each row)
    assert float(now[1]) == 2.0 ** -6 and float(now[0]) == 240.0
    assert float(x[1] / x[0]) <= stated()


def test_nothing_above_the_bound_changes():
    """All values of the types, down to far below their block's largest, beside every largest value that a block can have."""
    for _, _, bits in ref.F8.values():
        ms = torch.arange(2 ** bits, 2 ** (bits + 1)).double() / 2 ** bits
        for top in ms:
            values = torch.unique((ms[:, None] * 2.0 ** torch.arange(-30.0, 1.0)[None]).flatten().double())
            values = values[values <= top]
            x = torch.zeros(128, len(values), dtype=torch.float64)
            x[0], x[1] = top, values                        # columns: blocks of rows
            q, scale, _ = ref.blocks(ref.along(x))
            off = (q * scale)[:, 1] != values
            assert off.any() and float((values[off] / top).max()) <= stated()
