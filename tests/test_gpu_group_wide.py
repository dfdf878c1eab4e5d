"""kv_group_attn's kernels of 32 and 64 query rows a workgroup, and of prefixes of many rows beside sequences of few, against 64-bit forms. That these batches take them is checked without a GPU."""
import numpy as np
import pytest
import torch

from paper_2604_26557_amd import binding as kv
from servecase import FORMATS
from widecase import SHAPES, Wide, shape_of

pytestmark = pytest.mark.gpu

DTYPES = [torch.float16, torch.bfloat16]
KEYS = list(SHAPES)
NAMES = ["-".join(map(str, k)) for k in KEYS]
SHAPED = (dict(), dict(cap=12.0), dict(slopes=True), dict(cap=12.0, slopes=True))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("fmt", list(FORMATS))
@pytest.mark.parametrize("key", KEYS, ids=NAMES)
def test_wide_kernels(key, fmt, dtype):
    """Each with results of 32 and of 16 bits, plain, capped and biased; row blocks that are filled in part, sequences without new tokens."""
    for pow2, layout in ((0, "paged"), (1, "bhsd")):
        if pow2 and shape_of(key, fmt, 1) is shape_of(key, fmt, 0):
            break
        b = Wide(key[0], shape_of(key, fmt, pow2), dtype, fmt, layout, seed=pow2)
        for kw in SHAPED[pow2::2] + (SHAPED[:1] if pow2 else SHAPED[3:]):
            b.shape(**kw)
            b.check(b.run())
            b.check(b.run(kv.KV_OUT_SAME), False)


@pytest.mark.parametrize("key", KEYS, ids=NAMES)
def test_wide_kernels_of_windows_and_trees(key):
    """Windows that begin in the prefix and in a sequence's own tokens; trees of new tokens."""
    n = KEYS.index(key)
    fmt, dtype = (list(FORMATS) * 2)[n % 3], DTYPES[n % 2]
    fmt = "16" if fmt == "fp8" and key == (256, "apart", 1, 2) else fmt
    for tree, windows in ((False, (7, 90)), (True, (0, 40))):
        b = Wide(key[0], shape_of(key, fmt, n % 2), dtype, fmt, "paged", seed=n, tree=tree, bt=(16, 24)[n % 2])
        for i, window in enumerate(windows):
            b.shape(window=window, **SHAPED[(n + i) % 4])
            b.check(b.run())
            b.check(b.run(kv.KV_OUT_SAME), False)


@pytest.mark.parametrize("value,kind", [(float("nan"), "k"), (float("inf"), "v")])
@pytest.mark.parametrize("key", KEYS, ids=NAMES)
def test_wide_kernels_of_values_that_are_not_finite(key, value, kind):
    """Rows that see one have it in their results, the others what they had, whatever workgroup they share: rows are gone over one by one."""
    n = KEYS.index(key)
    s = shape_of(key, "16", n % 2)
    b = Wide(key[0], s, DTYPES[n % 2], "16", ("paged", "bhsd")[n % 2], seed=n).shape(window=9, **SHAPED[n % 4])
    hit = np.zeros(b.tok_first[-1], dtype=bool)
    places = []   # (sequence in whose place, token)
    for g, P in enumerate(b.prefix):   # of a prefix: those near its end see it
        places.append((b.first[g], P - 6))
    seqs = [i for i, t in enumerate(b.news) if t > 0]
    for i in (seqs[0], seqs[-1]):      # own tokens, the first new one among them
        places.append((i, b.lens[i]))
    for i, j in places:
        at, r = b.c.place(i, j)
        b.c.dev[kind][at, :, r, 5] = value
    for i, t in enumerate(b.news):
        a, shared = b.shared(i)
        seen = b.seen(i)
        for k, j in places:
            if (k == a and j < shared) or (k == i and j >= shared):
                hit[b.tok_first[i]:b.tok_first[i] + t] |= seen[:, j]
    assert hit.any() and not hit.all()
    if b.prefix:   # and a follower's place of the prefix, which nobody reads
        at, r = b.c.place(b.first[0] + 1, 3)
        b.c.dev[kind][at, :, r, 5] = value
    for od in (kv.KV_OUT_F32, kv.KV_OUT_SAME):
        got = b.run(od)
        b.check(got, od == kv.KV_OUT_F32, rows=~hit)
        bad = got[torch.from_numpy(hit).cuda()]
        assert torch.isnan(bad).all() if kind == "k" else (~torch.isfinite(bad[..., 5])).all() and torch.isfinite(bad[..., :5]).all() and torch.isfinite(bad[..., 6:]).all()


@pytest.mark.parametrize("key", [k for k in KEYS if k[0] == 128], ids=[n for n in NAMES if n.startswith("128")])
def test_wide_kernels_of_negative_scales_and_strided_results(key):
    b = Wide(128, shape_of(key, "16", 0), torch.bfloat16, "16", "paged", seed=3).shape(cap=9.0)
    n, hq = b.tok_first[-1], b.H * b.G
    buf = torch.full((n + 2, hq + 1, 131), 9.0, device="cuda")
    out = buf[:n, 1:, 2:130]
    got = b.attend(kv.KV_OUT_F32, b.splits, scale=-0.11, out=out)
    b.check(got, scale=-0.11)
    assert (buf[n:] == 9).all() and (buf[:, 0] == 9).all() and (buf[:, :, :2] == 9).all() and (buf[:, :, 130:] == 9).all()
