"""Attention of drafted tokens with 32 and 64 query rows a workgroup, against a plain 64-bit form: every format, type and kind of result, layouts, masks, splits."""
import itertools

import numpy as np
import pytest
import torch

from paper_2604_26557_amd import binding as kv
from servecase import FORMATS, UNIT, attention_bound, random_parents, sees
from treeshapes import LAYOUTS, SHAPES, WideCache, without_a_context, words_of

pytestmark = pytest.mark.gpu

DTYPES = [torch.float16, torch.bfloat16]
OUTS = [kv.KV_OUT_F32, kv.KV_OUT_SAME]


def make(D, nb, which, fmt, dtype, layout, kind, seed):
    """(cache, q, masks, splits) of a batch; kind: trees, a causal chain, or any mask (rows that see nothing among them)."""
    H, G, lens, drafted, splits = SHAPES[D, nb][which] if kind == "tree" or which == 0 else without_a_context(SHAPES[D, nb][which])[0]
    rng = np.random.default_rng(seed)
    c = WideCache(lens, H, D, G, dtype, fmt, layout, max(drafted), seed)
    q = torch.from_numpy(rng.standard_normal((sum(drafted), H * G, D)).astype(np.float32) * 1.5).to(dtype).cuda()
    if kind == "any":
        masks = [rng.random((n, n)) < 0.3 for n in drafted]
        for m in masks:
            m[1::5] = False
    else:
        masks = [np.tril(np.ones((n, n), dtype=bool)) if kind == "chain" else sees(random_parents(rng, n)) for n in drafted]
    return c, q, masks, splits


def run(c, q, masks, out_dtype, n_splits, chain=False):
    return c.attend(q, [[-1] * len(m) for m in masks], out_dtype, n_splits, mask=None if chain else words_of(masks))


def tolerance(c, want, out_dtype):
    """The bound of 32-bit arithmetic; with 16-bit results also what the parts of a probability lose, in numerator and sum, and one rounding."""
    out, weight, spread = want
    tol = attention_bound(out, weight, spread, max(c.lens) + 256, c.dtype, True)
    if out_dtype == kv.KV_OUT_SAME:
        tol = tol + 2 * (2.0 ** -22 if c.dtype == torch.float16 else 2.0 ** -16) * weight
        tol = tol * (1 + UNIT[c.dtype]) + UNIT[c.dtype] * np.abs(out) + (2.0 ** -25 if c.dtype == torch.float16 else 0)
    return tol


def check(c, want, got, out_dtype, rows=slice(None)):
    g = got.double().cpu().numpy()
    err, tol = np.abs(g - want[0])[rows], tolerance(c, want, out_dtype)[rows]
    assert np.isfinite(g[rows]).all() and (err <= tol).all(), (err.max(), (err / tol).max())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("fmt", list(FORMATS))
@pytest.mark.parametrize("which", [0, 1, 2])
@pytest.mark.parametrize("D,nb", list(SHAPES))
def test_wide_attention(D, nb, which, fmt, dtype):
    """Trees, in a layout that goes round with format, type and batch; both kinds of result, each number of splits."""
    i = which + 2 * list(FORMATS).index(fmt) + DTYPES.index(dtype) + nb // 2
    c, q, masks, splits = make(D, nb, which, fmt, dtype, LAYOUTS[i % 5], "tree", 100 + i)
    want = c.expected64(q, masks)
    for od, n in itertools.product(OUTS, splits):
        check(c, want, run(c, q, masks, od, n), od)


@pytest.mark.parametrize("fmt", list(FORMATS))
@pytest.mark.parametrize("kind", ["any", "chain"])
@pytest.mark.parametrize("D,nb", list(SHAPES))
def test_wide_attention_masks(D, nb, fmt, kind):
    """Masks that are no tree, with rows that see nothing where there is no context; a causal chain without a mask."""
    c, q, masks, splits = make(D, nb, 2, fmt, DTYPES[(D + nb) % 4 // 2], LAYOUTS[1], kind, 7 + D)
    b = c.lens.index(0)
    first = sum(len(m) for m in masks[:b])
    empty = [first + i for i, r in enumerate(masks[b]) if not r.any()]
    assert len(empty) > 2 or kind == "chain"
    want = c.expected64(q, masks)
    for od, n in itertools.product(OUTS, splits):
        got = run(c, q, masks, od, n, kind == "chain")
        check(c, want, got, od)
        assert (got[empty] == 0).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("fmt", list(FORMATS))
@pytest.mark.parametrize("D,nb", list(SHAPES))
def test_wide_attention_and_values_that_are_not_finite(D, nb, fmt, dtype):
    """In rows past the drafted tokens, in drafted tokens that no row sees, and in one that a single row sees: that row alone is not finite."""
    c, q, masks, splits = make(D, nb, 0, fmt, dtype, LAYOUTS[0], "any", 11 + D)
    want = c.expected64(q, masks)
    at = np.cumsum([0] + [len(m) for m in masks])
    bad = np.zeros(len(q), dtype=bool)
    for b, m in enumerate(masks):
        if len(m) == 0:
            continue
        m[:, 0] = False                       # seen by none
        if b % 2 == 0 and len(m) > 6:
            m[:, 3] = False
            m[5, 3] = True                    # by one
            bad[at[b] + 5] = True
        for slot in [c.lens[b]] + ([c.lens[b] + 3] if b % 2 == 0 and len(m) > 6 else []) + list(range(c.lens[b] + len(m), c.rows)):
            for kind in "kv":
                if fmt == "16":
                    c.dev[kind][b, :, slot, 5] = [float("nan"), float("inf"), float("-inf")][slot % 3] if kind == "v" else float("nan")
                else:
                    c.dev[kind + "_scale"][b, :, slot, D // 64] = 255
    want = c.expected64(q, masks)             # of the finite values, which what is seen has but for the rows that are bad
    for od, n in itertools.product(OUTS, splits):
        got = run(c, q, masks, od, n)
        check(c, want, got, od, ~bad)
        assert torch.isnan(got[torch.from_numpy(bad).cuda()]).all()


@pytest.mark.parametrize("fmt", list(FORMATS))
@pytest.mark.parametrize("D,nb", list(SHAPES))
def test_wide_attention_steep_scores(D, nb, fmt):
    """Scores of a spread of a dozen and more: references move again and again, and few tokens take nearly all."""
    c, q, masks, splits = make(D, nb, 1, fmt, torch.bfloat16, LAYOUTS[1], "tree", 13 + D)
    q[:] = (q.float() * 8).to(q.dtype)
    want = c.expected64(q, masks)
    assert 2 * want[2].max() * 2.0 ** -24 < 0.05   # the bound's first order holds
    for n in splits:
        check(c, want, run(c, q, masks, kv.KV_OUT_F32, n), kv.KV_OUT_F32)


def test_wide_runs_give_the_same_bits():
    c, q, masks, _ = make(128, 4, 2, "fp8", torch.bfloat16, LAYOUTS[1], "tree", 17)
    first = run(c, q, masks, kv.KV_OUT_SAME, 2)
    for _ in range(5):
        assert torch.equal(run(c, q, masks, kv.KV_OUT_SAME, 2), first)


@pytest.mark.parametrize("od", OUTS)
@pytest.mark.parametrize("pad", [1, 2, 3, 4])
@pytest.mark.parametrize("D,nb", list(SHAPES) + [(64, 1), (128, 1), (256, 1)])
def test_results_at_any_stride(D, nb, pad, od):
    """Results whose rows start at odd elements have the bits of those side by side, and nothing between them is written."""
    if nb == 1:
        c = WideCache([300, 40, 0], 2, D, 3, torch.bfloat16, "fp8", LAYOUTS[1], 5, 19)
        masks, splits = [sees(random_parents(np.random.default_rng(n), n)) for n in (5, 1, 3)], (1, 2)
        q = torch.from_numpy(np.random.default_rng(3).standard_normal((9, 6, D)).astype(np.float32)).to(torch.bfloat16).cuda()
    else:
        c, q, masks, splits = make(D, nb, 2, "fp8", torch.bfloat16, LAYOUTS[1], "tree", 19)
    words, parents = words_of(masks), [[-1] * len(m) for m in masks]
    for n in splits + (1,):
        want = c.attend(q, parents, od, n, mask=words)
        wide = torch.full((len(q), q.shape[1], D + pad), 7, dtype=want.dtype, device="cuda")
        c.attend(q, parents, od, n, mask=words, out=wide[..., :D])
        assert torch.equal(wide[..., :D], want) and (wide[..., D:] == 7).all()
