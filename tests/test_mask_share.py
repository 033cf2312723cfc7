"""The share of elements that a mask drops, as include/sr.h states it."""
import math
import os
import re

import numpy as np
import pytest
import torch

import paper_2605_05802_amd as sr
from paper_2605_05802_amd.build import INCLUDE
from test_decoder_rows import mask_words, rng


def stated(p):
    """The header's own expression for D, evaluated."""
    text = open(os.path.join(INCLUDE, "sr.h")).read()
    expression = re.search(r"^ \* +D = (.*)$", text, re.M).group(1)
    return eval(expression.replace("65536 p", "65536 * p"), {"min": min, "round": lambda x: math.floor(x + 0.5), "p": float(np.float32(p))})


SHARES = [0.0, 2.0 ** -18, 2.0 ** -17, 1e-5, 0.1, 0.5, 0.9, 0.999, 1 - 2.0 ** -16, 1 - 2.0 ** -17, 1 - 2.0 ** -20, 1 - 2.0 ** -24]


@pytest.mark.parametrize("p", SHARES)
def test_what_is_kept_has_a_factor(p):
    """Every p that is taken has one: what is kept is multiplied by 65536 / (65536 - D)."""
    assert 0 <= stated(p) < 65536 and abs(stated(p) / 65536 - p) <= 2.0 ** -16


@pytest.mark.gpu
@pytest.mark.parametrize("p", SHARES)
def test_masks_of_every_share(p):
    """Powers of two for values: products with the factor are exact where it is one, else within a rounding of it and one of the product."""
    rows, width = 1000, 1000
    x = 2.0 ** torch.randint(-3, 4, (rows, width), generator=rng(1), device="cuda").float()
    out = torch.empty_like(x)
    sr.sr_dropout(x, out, sr.Dropout(p, 12, mask=3))
    D = stated(p)
    words = mask_words(12, 3, np.arange(rows * width // 4, dtype=np.uint64))
    k = torch.from_numpy(words.view("<u2").reshape(rows, width) >= D).cuda()
    assert torch.equal(out != 0, k) and (p < 0.99999 or 0 < int(k.sum()) < 100)
    want = x.double() * k * (65536.0 / (65536 - D))
    assert bool(((out.double() - want).abs() <= 2.0 ** -23 * want).all())
