"""Attention of drafted tokens over a cache: results of 16 bits, and corners of its arithmetic."""
import numpy as np
import pytest
import torch

from paper_2604_26557_amd import binding as kv
from servecase import FORMATS, UNIT, Cache, attention_bound, random_parents

pytestmark = pytest.mark.gpu

DTYPES = [torch.float16, torch.bfloat16]


def rows(shape, dtype, seed, scale=1.0):
    return torch.from_numpy(np.random.default_rng(seed).standard_normal(shape).astype(np.float32) * scale).to(dtype)


def check_same(c, q, parents, got, **how):
    """A 16-bit result against 64 bits: the bound of 32-bit arithmetic, what the parts of a probability lose (2^-22 and 2^-16 of it, in numerator and sum), and
    one rounding.  A probability rounded to 16 bits misses it: 2^-11 and 2^-8 of each."""
    out, weight, spread = c.expected(q, parents, **how)
    g = got.double().cpu().numpy()
    tol = attention_bound(out, weight, spread, max(c.lens) + 256, c.dtype, True)
    tol = tol + 2 * (2.0 ** -22 if c.dtype == torch.float16 else 2.0 ** -16) * weight
    tol = tol * (1 + UNIT[c.dtype]) + UNIT[c.dtype] * np.abs(out) + (2.0 ** -25 if c.dtype == torch.float16 else 0)   # fp16 results may be subnormal
    err = np.abs(g - out)
    assert np.isfinite(g).all()
    assert (err <= tol).all(), (err.max(), (err / tol).max())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("fmt", list(FORMATS))
@pytest.mark.parametrize("D,H,G,lens,trees", [(64, 2, 1, [600, 33], [1, 1]), (128, 1, 4, [1500], [7]), (256, 2, 3, [90, 257], [5, 9]), (128, 1, 20, [700], [16])])
def test_16_bit_results_are_rounded_once(dtype, fmt, D, H, G, lens, trees):
    """As decode attention's: probabilities and their sums have more bits than the result."""
    parents = [random_parents(np.random.default_rng(D), n) for n in trees]
    c = Cache(lens, H, D, dtype, fmt, seed=D + G, extra=max(trees), n_q_heads=H * G)
    q = rows((sum(trees), H * G, D), dtype, 41).cuda()
    for n_splits in (0, 1, 3):
        check_same(c, q, parents, c.attend(q, parents, kv.KV_OUT_SAME, n_splits))
