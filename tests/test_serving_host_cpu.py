"""The serving step's host side where it is easily got wrong: ends of schedules, sizes, kinds of tensors."""
import math

import numpy as np
import pytest

from paper_2604_26557_amd import binding as kv


@pytest.mark.parametrize("base,trained,ends", [(10000.0, 65536, (40, 65)), (10000.0, 131072, (45, 70)), (10000.0, 4096, (20, 46)), (1.0e6, 32768, (23, 40)),
                                               (10000.0, 64, (0, 17)), (1.5, 1 << 20, (127, 127))])
def test_rope_table_by_index_past_the_last_pair(base, trained, ends):
    """The mixture of KV_ROPE_INDEX ends where t = low even if no pair is there: the last pairs keep their share of the plain frequency.  An end outside 0 .. rot_dim - 1
    is moved there."""
    n, rot, factor, low, high = 32, 128, 4.0, 1.0, 32.0
    at = lambda t: 64 * math.log(trained / (t * 2 * math.pi)) / math.log(base)  # noqa: E731
    first, last = min(max(math.floor(at(high)), 0), 127), min(max(math.ceil(at(low)), 0), 127)
    assert (first, last) == ends
    i = np.arange(64)
    keep = 1 - np.clip((i - first) / max(last - first, 1e-3), 0, 1)
    f = base ** (-i / 64)
    f = f * keep + f / factor * (1 - keep)
    a = np.arange(n)[:, None] * f
    got = kv.kv_rope_table(n, rot, base, kv.KV_ROPE_INDEX, factor, trained, low, high).numpy().astype(np.float64)
    # an angle below 32 in 53 bits, then 24
    assert np.abs(got - np.stack([np.cos(a), np.sin(a)], -1)).max() <= 2.0 ** -24 + 1e-13
    # and the last pair's angle by itself: sines of small angles, relative to a rounding
    assert np.abs(np.arcsin(got[1, 63, 1]) / f[63] - 1) <= 2.0 ** -22
