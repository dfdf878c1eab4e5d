"""The serving step's operators against plain 64-bit forms: rotary positions, rows into and out of a cache of 16, 8 or 4 bits, and
attention of drafted tokens over it."""
import itertools

import numpy as np
import pytest
import torch

from paper_2604_26557_amd import binding as kv
from servecase import FORMATS, UNIT, Cache, attention_bound, pack_codes, random_parents, ref_quantise, ref_rope, ref_values, sees, unpack_codes

pytestmark = pytest.mark.gpu

DTYPES = [torch.float16, torch.bfloat16]


def rows(shape, dtype, seed, scale=1.0):
    return torch.from_numpy(np.random.default_rng(seed).standard_normal(shape).astype(np.float32) * scale).to(dtype)


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def same(a, b):
    """Equal as values, NaN to NaN."""
    a, b = np.asarray(a, dtype=np.float64), np.asarray(b, dtype=np.float64)
    return np.array_equal(a, b, equal_nan=True)


# ------------------------------------------------------------------------------------------ rotary positions
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("style", [kv.KV_ROPE_HALF, kv.KV_ROPE_PAIRS])
@pytest.mark.parametrize("n,heads,D,rot", [(1, 1, 64, 64), (7, 5, 128, 128), (33, 32, 128, 64), (3, 7, 80, 32), (5, 3, 96, 48), (130, 9, 256, 256), (1, 6, 16, 16)])
@pytest.mark.parametrize("transposed", [False, True])
def test_rope(dtype, style, n, heads, D, rot, transposed):
    x = rows((n, heads, D), dtype, 1)
    pos = np.random.default_rng(2).integers(0, 5000, n).astype(np.int32)
    table = kv.kv_rope_table(5000, rot)
    rope = kv.Rope(table.cuda(), style)
    out = torch.full_like(x, 9).cuda()
    kv.kv_rope(rope, i32(pos.tolist()), x.cuda(), out, transposed=transposed)
    want = ref_rope(x.double().numpy(), table.numpy(), pos, rot, style, transposed)
    # three roundings to 24 bits of terms up to twice the pair's size, and one to 16 bits (subnormals: half of the smallest)
    got = out.double().cpu().numpy()
    size = np.abs(x.double().numpy()).max()
    tol = UNIT[dtype] * np.abs(want) + 3 * 2.0 ** -24 * 2 * size
    assert (np.abs(got - want) <= tol).all()
    assert same(got[..., rot:], x.double().numpy()[..., rot:])


@pytest.mark.parametrize("style", [kv.KV_ROPE_HALF, kv.KV_ROPE_PAIRS])
def test_rope_strides_and_in_place(style):
    """Heads of a wider row (q, k and v of a token side by side), one head's rows far apart, in place and not."""
    buf = rows((11, 12, 128), torch.bfloat16, 3).cuda()
    rope, pos = kv.Rope(kv.kv_rope_table(64, 64).cuda(), style), i32(list(range(20, 31)))
    x = buf[:, 2:9]
    want = torch.empty((11, 7, 128), dtype=torch.bfloat16, device="cuda")
    kv.kv_rope(rope, pos, x, want)
    heads_first = torch.zeros((7, 11, 128), dtype=torch.bfloat16, device="cuda")
    kv.kv_rope(rope, pos, x, heads_first.transpose(0, 1))
    assert torch.equal(heads_first.transpose(0, 1), want)
    kept = buf.clone()
    kv.kv_rope(rope, pos, x, x)
    assert torch.equal(buf[:, 2:9], want)
    assert torch.equal(buf[:, :2], kept[:, :2]) and torch.equal(buf[:, 9:], kept[:, 9:])


def test_rope_gradient_against_differences():
    """d/dx sum(w * rope(x)) = rope transposed of w, compared with differences of the 64-bit form."""
    table = kv.kv_rope_table(100, 32, magnitude=1.25)
    x, w = rows((4, 2, 64), torch.float16, 4), rows((4, 2, 64), torch.float16, 5)
    pos = np.array([0, 1, 50, 99])
    for style in (kv.KV_ROPE_HALF, kv.KV_ROPE_PAIRS):
        grad = torch.empty_like(w).cuda()
        kv.kv_rope(kv.Rope(table.cuda(), style), i32(pos.tolist()), w.cuda(), grad, transposed=True)
        g = grad.double().cpu().numpy()
        x64, w64 = x.double().numpy(), w.double().numpy()
        loss = lambda z: (w64 * ref_rope(z, table.numpy(), pos, 32, style)).sum()  # noqa: E731
        for idx in itertools.product(range(4), range(2), (0, 1, 15, 16, 17, 31, 32, 63)):
            step = np.zeros_like(x64)
            step[idx] = 2.0 ** -10
            diff = (loss(x64 + step) - loss(x64 - step)) / 2.0 ** -9   # the form is linear: no error of truncation
            assert abs(diff - g[idx]) <= 2.0 ** -11 * abs(diff) + 2.0 ** -20


def test_rope_turned_back_and_positions_outside():
    x = rows((6, 3, 64), torch.bfloat16, 6)
    rope = kv.Rope(kv.kv_rope_table(10, 32).cuda())
    out = torch.zeros_like(x).cuda()
    kv.kv_rope(rope, i32([0, 9, 10, -1, 2**31 - 1, 5]), x.cuda(), out)
    bad = torch.isnan(out[..., :32].float()).all(-1).all(-1).cpu()
    assert bad.tolist() == [False, False, True, True, True, False]
    assert torch.equal(out[..., 32:].cpu(), x[..., 32:]) and torch.equal(out[0].cpu(), x[0])
    back = torch.zeros_like(out)
    kv.kv_rope(rope, i32([0, 9, 0, 0, 0, 5]), out, back, transposed=True)
    for i in (0, 1, 5):   # two roundings to 8 bits of values up to twice as large
        assert (back[i].cpu().double() - x[i].double()).abs().max() <= 4 * UNIT[torch.bfloat16] * x[i].double().abs().max()
    kv.kv_rope(rope, i32([]), x.cuda()[:0], out[:0])


# ------------------------------------------------------------------------------------------ rows in and out
def write_case(dtype, fmt, layout, style, n, H, D, rot, seed=7, bt=16, lens=(40, 3, 25)):
    c = Cache(lens, H, D, dtype, fmt, layout, bt=bt, seed=seed, extra=n)
    rng = np.random.default_rng(seed + 1)
    seq = rng.integers(0, len(lens), n)
    slots, seen = [], set()
    for b in seq:   # distinct places anywhere in the capacity
        while True:
            s = int(rng.integers(0, lens[b] + n))
            if (b, s) not in seen:
                break
        seen.add((b, s))
        slots.append(s)
    return c, seq.tolist(), slots, rows((n, H, D), dtype, seed + 2), rows((n, H, D), dtype, seed + 3)


def snapshot(c):
    return {k: v.clone() for k, v in c.dev.items()}


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("fmt", list(FORMATS))
@pytest.mark.parametrize("layout,bt", [("bhsd", 0), ("paged", 16), ("paged", 7)])
@pytest.mark.parametrize("n,H,D,rot,style", [(1, 1, 32, 0, 0), (9, 3, 64, 64, kv.KV_ROPE_HALF), (37, 8, 128, 64, kv.KV_ROPE_PAIRS),
                                             (20, 2, 96, 16, kv.KV_ROPE_HALF), (5, 5, 256, 256, kv.KV_ROPE_PAIRS), (6, 2, 128, 48, kv.KV_ROPE_HALF)])
def test_cache_write_and_read(dtype, fmt, layout, bt, n, H, D, rot, style):
    """Codes, scales and untouched rows bit for bit (V; K without rotation), rotated K to a rounding; then the same rows read back."""
    c, seq, slots, k, v = write_case(dtype, fmt, layout, style, n, H, D, rot, bt=bt or 16)
    before = snapshot(c)
    table = kv.kv_rope_table(300, rot) if rot else None
    rope = kv.Rope(table.cuda(), style) if rot else None
    pos = np.random.default_rng(8).integers(0, 300, n).astype(np.int32)
    kv.kv_cache_write(c.plan, c.view, c.blocks, 0, k.cuda(), v.cuda(), i32(seq), i32(slots), rope, i32(pos.tolist()) if rot else None)
    if rot:   # the rotation alone, which test_rope compares with 64 bits; the write rounds it in the same places
        kr = torch.empty_like(k).cuda()
        kv.kv_rope(rope, i32(pos.tolist()), k.cuda(), kr)
        kr = kr.cpu()
    else:
        kr = k
    places = [c.place(b, s) for b, s in zip(seq, slots)]
    want = {}
    for kind, x in (("k", kr), ("v", v)):
        if fmt == "16":
            got = torch.stack([c.dev[kind][i, :, r] for i, r in places]).cpu()
            assert torch.equal(got.view(torch.int16), x.view(torch.int16))
            want[kind] = x.double().numpy()
        else:
            code, scale = ref_quantise(x.double().numpy(), fmt, dtype == torch.float16)
            got = torch.stack([c.dev[kind][i, :, r] for i, r in places]).cpu().numpy()
            gots = torch.stack([c.dev[kind + "_scale"][i, :, r] for i, r in places]).cpu().numpy()
            assert np.array_equal(gots, scale)
            assert np.array_equal(unpack_codes(got, fmt), code)
            want[kind] = ref_values(code, scale, fmt)
    for name, t in c.dev.items():   # nothing else was written
        keep = torch.ones(t.shape[:1] + t.shape[2:3], dtype=torch.bool)
        for i, r in places:
            keep[i, r] = False
        m = keep[:, None, :, None].expand(t.shape).cuda()
        assert torch.equal(t[m], before[name][m])
    ko, vo = torch.full_like(k, 5).cuda(), torch.full_like(v, 5).cuda()
    kv.kv_cache_read(c.plan, c.view, c.blocks, 0, i32(seq), i32(slots), ko, vo)
    assert same(ko.double().cpu(), want["k"]) and same(vo.double().cpu(), want["v"])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
def test_every_scale_and_code(dtype, fmt):
    """Rows whose blocks go through all magnitudes of the type, ties between codes, zeros of both signs, infinities and NaNs."""
    raw = np.arange(65536, dtype=np.uint16)
    bits = np.random.default_rng(1).permutation(raw).reshape(-1, 32)
    near = raw.reshape(-1, 32)                       # neighbours: one exponent per block
    ties = np.stack([np.arange(32) * 0.25 * 2.0 ** e for e in range(-14, 12)]).astype(np.float32)
    t = torch.cat([torch.from_numpy(np.concatenate([bits, near]).view(np.int16).copy()).view(dtype), torch.from_numpy(ties).to(dtype), -torch.from_numpy(ties).to(dtype),
                   torch.zeros((4, 32), dtype=dtype)])
    t = torch.cat([t, torch.zeros((-len(t)) % 4, 32, dtype=dtype)]).view(-1, 1, 128)
    n = t.shape[0]
    c = Cache([n], 1, 128, dtype, fmt, seed=3)
    kv.kv_cache_write(c.plan, c.view, c.blocks, 0, t.cuda(), t.flip(0).contiguous().cuda(), i32([0] * n), i32(list(range(n))))
    code, scale = ref_quantise(t.double().numpy(), fmt, dtype == torch.float16)
    assert np.array_equal(c.dev["k_scale"][0, 0].cpu().numpy(), scale[:, 0])
    got = unpack_codes(c.dev["k"][0, 0].cpu().numpy(), fmt)
    fine = np.repeat(scale[:, 0] != 255, 32, -1)
    assert np.array_equal(got[fine], code[:, 0][fine])
    ko, vo = torch.zeros_like(t).cuda(), torch.zeros_like(t).cuda()
    kv.kv_cache_read(c.plan, c.view, c.blocks, 0, i32([0] * n), i32(list(range(n))), ko, vo)
    want = ref_values(code, scale, fmt)
    assert same(ko.double().cpu(), want)              # every value is a number of the type: nothing is rounded
    assert torch.equal(vo.flip(0).view(torch.int16)[~vo.flip(0).isnan()], ko.view(torch.int16)[~ko.isnan()])


@pytest.mark.parametrize("fmt", list(FORMATS))
@pytest.mark.parametrize("layout", ["bhsd", "paged"])
def test_rows_without_a_place_are_skipped(fmt, layout):
    c = Cache([20, 9], 2, 64, torch.float16, fmt, layout, seed=5)
    if layout == "paged":
        c.table[1, 0] = 10 ** 6
        c.table[0, 1] = -1
    before = snapshot(c)
    bad = [(-1, 0), (2, 0), (0, -1), (0, 10 ** 9), (2 ** 31 - 1, 3), (1, -2 ** 31), (0, 4096)]
    if layout == "paged":
        bad += [(1, 3), (0, 17)]
    else:
        bad += [(0, 20), (1, 20)]
    k = rows((len(bad), 2, 64), torch.float16, 6).cuda()
    seq, slot = i32([b for b, _ in bad]), i32([s for _, s in bad])
    kv.kv_cache_write(c.plan, c.view, c.blocks, 0, k, k, seq, slot)
    for name, t in c.dev.items():
        assert torch.equal(t, before[name])
    ko, vo = torch.full_like(k, 5), torch.full_like(k, 6)
    kv.kv_cache_read(c.plan, c.view, c.blocks, 0, seq, slot, ko, vo)
    assert (ko == 5).all() and (vo == 6).all()
    kv.kv_cache_write(c.plan, c.view, c.blocks, 0, k[:0], k[:0], seq[:0], slot[:0])


def test_write_strides_and_scale_orders():
    """K and V as parts of a wider row, scales of a token side by side over the heads."""
    n, H, D = 30, 4, 128
    c = Cache([30], H, D, torch.bfloat16, "fp8", seed=9, token_major_scales=True)
    assert c.dev["k_scale"].stride(2) == H * D // 32
    qkv = rows((n, 3 * H, D), torch.bfloat16, 10).cuda()
    k, v = qkv[:, H:2 * H], qkv[:, 2 * H:]
    order = np.random.default_rng(11).permutation(n).tolist()
    kv.kv_cache_write(c.plan, c.view, c.blocks, 0, k, v, i32([0] * n), i32(order))
    code, scale = ref_quantise(v.double().cpu().numpy(), "fp8", False)
    assert np.array_equal(c.dev["v"][0].cpu().numpy()[:, order].transpose(1, 0, 2), code)
    assert np.array_equal(c.dev["v_scale"][0].cpu().numpy()[:, order].transpose(1, 0, 2), scale)
    back = torch.zeros((H, n, 2, D), dtype=torch.bfloat16, device="cuda")   # a head's rows, K beside V
    ko, vo = back[:, :, 0].transpose(0, 1), back[:, :, 1].transpose(0, 1)
    kv.kv_cache_read(c.plan, c.view, c.blocks, 0, i32([0] * n), i32(order), ko, vo)
    assert same(vo.double().cpu(), ref_values(code, scale, "fp8"))


# ------------------------------------------------------------------------------------------ attention
def check(c, q, parents, got, f32, **how):
    out, weight, spread = c.expected(q, parents, **how)
    g = got.double().cpu().numpy()
    tol = attention_bound(out, weight, spread, max(c.lens) + 256, c.dtype, f32)
    err = np.abs(g - out)
    assert np.isfinite(g).all()
    assert (err <= tol).all(), (err.max(), (err / tol).max())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("fmt", list(FORMATS))
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("H,G", [(1, 1), (2, 4), (3, 7), (1, 16), (2, 20)])
def test_tree_attention_heads(dtype, fmt, D, H, G):
    lens = [100, 33]
    rng = np.random.default_rng(D + G)
    parents = [random_parents(rng, 6), random_parents(rng, 11)]
    c = Cache(lens, H, D, dtype, fmt, seed=D, extra=12, n_q_heads=H * G)
    q = rows((17, H * G, D), dtype, 20).cuda()
    for od in (kv.KV_OUT_F32, kv.KV_OUT_SAME):
        check(c, q, parents, c.attend(q, parents, od), od == kv.KV_OUT_F32)


@pytest.mark.parametrize("fmt", list(FORMATS))
@pytest.mark.parametrize("layout,bt", [("bhsd", 0), ("paged", 16), ("paged", 5), ("paged", 64), ("paged", 1)])
@pytest.mark.parametrize("lens,trees", [([0], [1]), ([1], [1]), ([0, 5], [0, 3]), ([15, 16, 17], [1, 1, 1]), ([31, 32, 33, 64], [2, 31, 1, 40]),
                                        ([700], [64]), ([129, 0, 513], [65, 20, 130]), ([300], [256]), ([2100, 40], [1, 1]), ([5000], [9])])
def test_tree_attention_lengths(fmt, layout, bt, lens, trees):
    rng = np.random.default_rng(sum(lens) + 3)
    parents = [random_parents(rng, n) for n in trees]
    c = Cache(lens, 2, 64, torch.bfloat16, fmt, layout, bt=bt or 16, seed=len(lens), extra=max(trees), n_q_heads=6)
    q = rows((sum(trees), 6, 64), torch.bfloat16, 21).cuda()
    for od in (kv.KV_OUT_F32, kv.KV_OUT_SAME):
        check(c, q, parents, c.attend(q, parents, od), od == kv.KV_OUT_F32)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("fmt", list(FORMATS))
@pytest.mark.parametrize("n_splits", [1, 2, 3, 7, 128])
def test_tree_attention_splits(dtype, fmt, n_splits):
    lens, trees = [1000, 3, 260], [5, 2, 17]
    rng = np.random.default_rng(n_splits)
    parents = [random_parents(rng, n) for n in trees]
    c = Cache(lens, 2, 128, dtype, fmt, "paged", seed=n_splits, extra=17, n_q_heads=8)
    q = rows((24, 8, 128), dtype, 22, 2.0).cuda()
    check(c, q, parents, c.attend(q, parents, kv.KV_OUT_F32, n_splits), True)
    small = torch.empty(16, dtype=torch.uint8, device="cuda")   # no room for partial results: nothing is split
    check(c, q, parents, c.attend(q, parents, kv.KV_OUT_F32, 0, ws=small), True)


@pytest.mark.parametrize("fmt", list(FORMATS))
def test_causal_chain_and_single_tokens(fmt):
    lens = [90, 200, 1]
    parents = [random_parents(None, n, tree=False) for n in (8, 1, 70)]
    c = Cache(lens, 2, 128, torch.float16, fmt, seed=4, extra=70, n_q_heads=2)
    q = rows((79, 2, 128), torch.float16, 23).cuda()
    check(c, q, parents, c.attend(q, parents, mask=None), True, chain=True)
    assert torch.equal(c.attend(q, parents, kv.KV_OUT_SAME, 1, mask=None), c.attend(q, parents, kv.KV_OUT_SAME, 1))   # the chain as a tree


@pytest.mark.parametrize("fmt", list(FORMATS))
@pytest.mark.parametrize("out_dtype", [kv.KV_OUT_F32, kv.KV_OUT_SAME])
def test_rows_that_see_nothing_and_any_mask(fmt, out_dtype):
    """Masks that are no tree: rows that see none, all, or only later tokens; without a context a row may be left empty."""
    rng = np.random.default_rng(6)
    lens, n = [0, 70], 67
    masks = [rng.random((n, n)) < 0.3 for _ in lens]
    masks[0][[0, 5, 66]] = False
    masks[1][[1, 2]] = False
    masks[0][7] = True
    c = Cache(lens, 2, 64, torch.bfloat16, fmt, seed=4, extra=n, n_q_heads=4)
    q = rows((2 * n, 4, 64), torch.bfloat16, 24).cuda()
    words = np.zeros((2 * n, 2), dtype=np.uint64)
    for i, row in enumerate(np.concatenate(masks)):
        for j in np.flatnonzero(row):
            words[i, j // 64] |= np.uint64(1) << np.uint64(j % 64)
    parents = [[-1] * n] * 2
    got = c.attend(q, parents, out_dtype, mask=torch.from_numpy(words.view(np.int64)).cuda())
    check(c, q, parents, got, out_dtype == kv.KV_OUT_F32, masks=masks)
    assert (got[[0, 5, 66]] == 0).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("fmt", list(FORMATS))
@pytest.mark.parametrize("kind,value", [("k", float("nan")), ("v", float("nan")), ("k", float("inf")), ("v", float("inf")), ("v", float("-inf"))])
def test_values_that_are_not_finite_where_no_row_sees_them(dtype, fmt, kind, value):
    """Behind the last drafted token, in drafted tokens of other branches, and in other sequences' rows."""
    lens, n = [50, 45], 9
    parents = [[-1, 0, 0, 1, 2, 3, 4, -1, 7]] * 2
    c = Cache(lens, 2, 64, dtype, fmt, seed=12, extra=40, n_q_heads=4)
    for b in range(2):
        for slot in range(lens[b] + n, c.rows):
            c.set_value(kind, b, slot, 3, value)
        c.set_value(kind, b, lens[b] + 4, 35, value)      # seen by tokens 4 and 6
        c.set_value(kind, b, lens[b] + 8, 40, value)      # seen by token 8
    q = rows((2 * n, 4, 64), dtype, 25).cuda()
    for od in (kv.KV_OUT_F32, kv.KV_OUT_SAME):
        got = c.attend(q, parents, od)
        out, weight, spread = c.expected(q, parents)
        hit = np.array([i % n in (4, 6, 8) for i in range(2 * n)])
        g = got.double().cpu().numpy()
        tol = attention_bound(out, weight, spread, 400, dtype, od == kv.KV_OUT_F32)
        assert (np.abs(g - out)[~hit] <= tol[~hit]).all()
        if kind == "v":   # only the columns of what is not finite
            fine = np.isfinite(out)
            assert np.array_equal(np.isfinite(g), fine) and (np.abs(g - out)[fine] <= tol[fine]).all()
            if fmt == "16":
                assert same(g[~fine], out[~fine])
        elif np.isnan(value) or fmt != "16":
            assert np.isnan(g[hit]).all()


def test_infinite_scores_of_one_sign():
    """A key of minus infinity times a positive query weighs nothing: the rest of the row is as if it was not there."""
    c = Cache([64], 1, 64, torch.bfloat16, "16", seed=13, extra=4, n_q_heads=2)
    c.set_value("k", 0, 10, 5, float("-inf"))
    q = rows((2, 2, 64), torch.bfloat16, 26).abs().cuda()
    parents = [[-1, 0]]
    got = c.attend(q, parents).double().cpu().numpy()
    want = c.expected(q, parents)[0]
    assert np.isfinite(want).all() and np.abs(got - want).max() <= 1e-4


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("big", [30.0, 1000.0])
def test_steep_and_large_scores(dtype, big):
    """Scores of hundreds to millions: one token takes nearly all, and which one depends on 32-bit scores being 32-bit scores."""
    c = Cache([500], 1, 128, dtype, "16", seed=14, extra=3, n_q_heads=4, scale=big if dtype == torch.bfloat16 else min(big, 200.0))
    q = rows((3, 4, 128), dtype, 27, big if dtype == torch.bfloat16 else min(big, 200.0)).cuda()
    parents = [[-1, -1, 0]]
    got = c.attend(q, parents).double().cpu().numpy()
    out, weight, spread = c.expected(q, parents)
    u = 2.0 ** -24
    # weights change by exp(the error of two scores): where that is not small, any mixture of the values is as good
    tol = weight * np.minimum(np.expm1(np.minimum(2 * spread[..., None] * u, 50)) + 64 * u, 1e30) + 1e-6 * big
    tol = np.where(2 * spread[..., None] * u > 0.5, 2 * np.abs(c.values["v"]).max(), tol)
    assert np.isfinite(got).all() and (np.abs(got - out) <= tol).all()


def test_attention_strides_scale_and_orders():
    """q as a part of a wider row, results by heads, a cache whose sequences and heads lie apart or turned round, another scale."""
    B, H, G, D, n = 2, 2, 3, 64, 5
    c = Cache([37, 80], H, D, torch.bfloat16, "fp8", seed=15, extra=8, n_q_heads=H * G, token_major_scales=True)
    for kind in ("k", "v"):   # [B, S, H, D] seen as [B, H, S, D], rows of twice the width
        t = c.dev[kind]
        wide = torch.zeros((t.shape[0], t.shape[2], t.shape[1], 2 * D), dtype=torch.uint8, device="cuda")
        wide[..., :D] = t.transpose(1, 2)
        c.dev[kind] = wide[..., :D].transpose(1, 2)
    k, v = ([c.dev[x].transpose(1, 2).as_strided(c.dev[x].shape[:1] + (c.dev[x].shape[1], c.dev[x].shape[2], D), c.dev[x].stride())] for x in ("k", "v"))
    k16, v16 = ([x[0].view(torch.int16)] for x in (k, v))
    c.view = kv.bhsd_view(k16, v16, c.lens, c.lens_dev)
    wide_q = rows((2 * n, 3 * H * G, D), torch.bfloat16, 28).cuda()
    q = wide_q[:, H * G:2 * H * G]
    by_head = torch.zeros((H * G, 2 * n, D), dtype=torch.float32, device="cuda")
    parents = [[-1, 0, 1, 0, 3]] * 2
    c.attend(q, parents, scale=0.2, out=by_head.transpose(0, 1))
    check(c, q, parents, by_head.transpose(0, 1), True, scale=0.2)


def test_offsets_beyond_32_bits():
    """Rows more than 4 GiB from the buffer's start, strided and paged."""
    D, far = 64, 5 << 30
    buf = torch.zeros(far + (1 << 20), dtype=torch.uint8, device="cuda")
    small = Cache([40], 1, D, torch.bfloat16, "fp8", seed=16, extra=4, n_q_heads=4)
    q = rows((4, 4, D), torch.bfloat16, 29).cuda()
    parents = [[-1, 0, 0, 2]]
    want = small.attend(q, parents, n_splits=1)
    n = small.rows
    # two sequences, the second one far away
    big = Cache([0, 40], 1, D, torch.bfloat16, "fp8", seed=16, extra=4, n_q_heads=4)
    k = buf.as_strided((2, 1, n, D), (far, n * D, D, 1))
    v = buf[n * D:].as_strided((2, 1, n, D), (far, n * D, D, 1))
    k[1], v[1] = small.dev["k"][0], small.dev["v"][0]
    big.dev["k_scale"][1], big.dev["v_scale"][1] = small.dev["k_scale"][0], small.dev["v_scale"][0]
    big.dev["k"], big.dev["v"] = k, v
    big.remake()
    assert torch.equal(big.attend(q, [[], parents[0]], n_splits=1), want)
    # written and read there
    kn = rows((1, 1, D), torch.bfloat16, 30).cuda()
    kv.kv_cache_write(big.plan, big.view, big.blocks, 0, kn, kn, i32([1]), i32([7]))
    ko, vo = torch.zeros_like(kn), torch.zeros_like(kn)
    kv.kv_cache_read(big.plan, big.view, big.blocks, 0, i32([1]), i32([7]), ko, vo)
    want_code, want_scale = ref_quantise(kn.double().cpu().numpy(), "fp8", False)
    assert same(ko.double().cpu(), ref_values(want_code, want_scale, "fp8")) and torch.equal(ko, vo)
    # tokens far apart
    s = 160 << 20
    k = buf.as_strided((1, 1, 33, D), (0, 0, s, 1))
    v = buf[D:].as_strided((1, 1, 33, D), (0, 0, s, 1))
    far_tokens = Cache([30], 1, D, torch.bfloat16, "fp8", seed=17, extra=3, n_q_heads=4)
    parents = [[-1, 0, 1]]
    want = far_tokens.attend(q[:3], parents, n_splits=1)
    k[0], v[0] = far_tokens.dev["k"][0], far_tokens.dev["v"][0]
    far_tokens.dev["k"], far_tokens.dev["v"] = k, v
    far_tokens.remake()
    assert torch.equal(far_tokens.attend(q[:3], parents, n_splits=1), want)
    # blocks of a pool beyond 4 GiB
    paged = Cache([40], 1, D, torch.bfloat16, "fp8", "paged", seed=18, extra=4, n_q_heads=4)
    parents = [[-1, 0, 0, 2]]
    want = paged.attend(q, parents, n_splits=1)
    n_pool, skip = far // (16 * D), (far - (1 << 20)) // (16 * D)
    pool_k = buf[:n_pool * 16 * D].view(n_pool, 1, 16, D)
    scales = torch.zeros((n_pool, 1, 16, D // 32), dtype=torch.uint8, device="cuda")
    m = paged.dev["k"].shape[0]
    pool_k[skip:skip + m], scales[skip:skip + m] = paged.dev["k"], paged.dev["k_scale"]
    keys_only = paged.dev["v"], paged.dev["v_scale"]
    paged.dev["v"][:], paged.dev["v_scale"][:] = paged.dev["k"], paged.dev["k_scale"]
    want = paged.attend(q, parents, n_splits=1)
    paged.table += skip
    paged.dev.update(k=pool_k, v=pool_k, k_scale=scales, v_scale=scales)
    paged.remake()
    assert torch.equal(paged.attend(q, parents, n_splits=1), want)
    del keys_only


def test_a_block_without_a_place_counts_as_unseen():
    """Ids outside the pool are skipped, as decode attention does."""
    c = Cache([64], 1, 64, torch.float16, "fp8", "paged", seed=19, extra=4, n_q_heads=2)
    q = rows((2, 2, 64), torch.float16, 31).cuda()
    c.table[0, 1] = -1
    got = c.attend(q, [[-1, 0]]).double().cpu().numpy()
    k, v = c.seq("k", 0, 66), c.seq("v", 0, 66)
    keep = np.r_[0:16, 32:66]
    x = q.double().cpu().numpy()
    for t, h in itertools.product(range(2), range(2)):
        idx = keep[keep <= 64 + t]
        s = k[0][idx] @ x[t, h] / 8
        p = np.exp(s - s.max())
        assert np.abs(got[t, h] - p @ v[0][idx] / p.sum()).max() <= 1e-5


def test_another_stream_and_graph():
    """The calls run on the stream they are given, and a graph of them replays with new contents."""
    c = Cache([100, 60], 2, 128, torch.bfloat16, "fp8", "paged", seed=20, extra=10, n_q_heads=8)
    parents = [[-1, 0, 0, 1], [-1, 0, 1]]
    n = 7
    table = kv.kv_rope_table(200, 128).cuda()
    rope = kv.Rope(table)
    first, first_dev = [0, 4, 7], i32([0, 4, 7])
    mask = torch.cat([kv.kv_tree_masks(p, 1)[0] for p in parents]).cuda()
    tree = kv.tree_batch(first, first_dev, mask)
    depth = [kv.kv_tree_masks(p, 1)[1].tolist() for p in parents]
    seq, slot = i32([0] * 4 + [1] * 3), i32([100, 101, 102, 103, 60, 61, 62])
    pos = i32([100 + d for d in depth[0]] + [60 + d for d in depth[1]])
    q, k, v = (torch.zeros((n, h, 128), dtype=torch.bfloat16, device="cuda") for h in (8, 2, 2))
    qr, out = torch.zeros_like(q), torch.zeros(q.shape, dtype=torch.float32, device="cuda")
    ws = torch.empty(kv.kv_tree_attn_workspace(c.plan, n, 200), dtype=torch.uint8, device="cuda")

    def step():
        kv.kv_rope(rope, pos, q, qr)
        kv.kv_cache_write(c.plan, c.view, c.blocks, 0, k, v, seq, slot, rope, pos)
        kv.kv_tree_attn(c.plan, c.view, c.blocks, 0, tree, qr, out, kv.KV_OUT_F32, 0, ws)

    def fill(seed):
        for i, t in enumerate((q, k, v)):
            t.copy_(rows(t.shape, torch.bfloat16, seed + i))

    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        fill(40)
        step()
        other = out.clone()
    s.synchronize()
    fill(40)
    step()
    torch.cuda.synchronize()
    assert torch.equal(other, out)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for seed in (50, 60, 70):
        fill(seed)
        out.fill_(3)
        g.replay()
        torch.cuda.synchronize()
        got = out.clone()
        step()
        torch.cuda.synchronize()
        assert torch.equal(got, out) and torch.isfinite(got).all()


def test_two_runs_give_the_same_bits():
    c = Cache([3000, 700], 2, 128, torch.bfloat16, "fp8", seed=21, extra=16, n_q_heads=8)
    parents = [random_parents(np.random.default_rng(1), 16), [-1]]
    q = rows((17, 8, 128), torch.bfloat16, 32).cuda()
    first = c.attend(q, parents)
    for _ in range(5):
        assert torch.equal(c.attend(q, parents), first)


@pytest.mark.parametrize("fmt,share", [("fp8", 2), ("fp4", 4)])
def test_example_of_a_serving_loop(fmt, share):
    """The operators together: drafts verified, accepted rows kept, the cache offloaded and reloaded as codes and scales."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "tree_step.py")
    spec = importlib.util.spec_from_file_location("tree_step", path)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    worst, moved, full = mod.main(layers=2, context=333, steps=4, fmt=fmt, say=lambda *a: None)
    # probabilities and results are rounded to 8 bits, the 32-bit form's operands are the same: two roundings of at most 2^-8 each
    assert worst <= 2 * 2.0 ** -8
    assert full / share < moved < full / share * 1.2   # scales are 1/32 of fp8 codes, 1/16 of fp4's; whole sectors


@pytest.mark.parametrize("fmt", ["16", "fp8"])
@pytest.mark.parametrize("D,H,G,layout,bt,lens,trees", [
    (128, 1, 40, "paged", 8, [90, 17], [7, 3]),           # blocks of half a group of 16 tokens, more heads than a row group
    (64, 2, 3, "paged", 48, [333, 1500], [5, 33]),        # blocks that are no power of two
    (256, 1, 8, "paged", 32, [4300], [30]),               # several rounds of a wavefront's look-ups: 32 steps of 128 tokens each
    (64, 1, 4, "paged", 16, [9000, 4095, 4097], [1, 2, 3]),
    (64, 3, 2, "bhsd", 0, [40 * i for i in range(20)], [1 + i % 5 for i in range(20)]),   # more sequences than the cut counts one by one
    (128, 2, 16, "bhsd", 0, [64] * 18, [9] * 18)])
def test_attention_blocks_groups_and_batches(fmt, D, H, G, layout, bt, lens, trees):
    rng = np.random.default_rng(len(lens))
    parents = [random_parents(rng, n) for n in trees]
    c = Cache(lens, H, D, torch.float16, fmt, layout, bt=bt or 16, seed=len(lens), extra=max(trees), n_q_heads=H * G)
    q = rows((sum(trees), H * G, D), torch.float16, 33).cuda()
    for n_splits in (0, 1):
        check(c, q, parents, c.attend(q, parents, kv.KV_OUT_F32, n_splits), True)


@pytest.mark.parametrize("stride", [(1 << 25) - 64, 1 << 25])
def test_tokens_as_far_apart_as_a_step_can_count(stride):
    """Either side of the token stride from which rows are looked up one by one: several steps of each wavefront."""
    D, n = 64, 300
    buf = torch.empty(stride * n + 2 * D, dtype=torch.uint8, device="cuda")
    c = Cache([n - 2], 1, D, torch.bfloat16, "fp8", seed=22, extra=2, n_q_heads=4)
    q = rows((2, 4, D), torch.bfloat16, 34).cuda()
    want = c.attend(q, [[-1, 0]], n_splits=1)
    for kind, at in (("k", 0), ("v", D)):
        far = buf[at:].as_strided((1, 1, n, D), (0, 0, stride, 1))
        far[0] = c.dev[kind][0]
        c.dev[kind] = far
    c.remake()
    assert torch.equal(c.attend(q, [[-1, 0]], n_splits=1), want)


@pytest.mark.parametrize("stride", [(1 << 28) - 4, 1 << 28])
def test_scales_of_a_block_as_far_apart_as_32_bits_count(stride):
    """Scales by tokens over all blocks: either side of what a block's offset holds."""
    D = 64
    c = Cache([100], 1, D, torch.bfloat16, "fp8", "paged", seed=23, extra=2, n_q_heads=4)
    q = rows((2, 4, D), torch.bfloat16, 35).cuda()
    want = c.attend(q, [[-1, 0]], n_splits=1)
    m, buf = c.dev["k_scale"].shape[0], torch.empty(stride * 16 + 4096, dtype=torch.uint8, device="cuda")
    for kind, at in (("k_scale", 0), ("v_scale", 2048)):
        far = buf[at:].as_strided((m, 1, 16, D // 32), (2, 2, stride, 1))
        far[:] = c.dev[kind]
        c.dev[kind] = far
    c.remake()
    assert torch.equal(c.attend(q, [[-1, 0]], n_splits=1), want)


@pytest.mark.parametrize("B", [63, 64, 65])
def test_ragged_batches_as_wide_as_a_wavefront(B):
    """Workgroups without work are left out of up to 64 sequences' launches, by sums over a wavefront's lanes."""
    rng = np.random.default_rng(B)
    lens, trees = rng.integers(0, 700, B).tolist(), rng.integers(0, 12, B).tolist()
    trees[0] = trees[-1] = 11
    trees[1] = trees[B // 2] = 0
    parents = [random_parents(rng, n) for n in trees]
    c = Cache(lens, 3, 64, torch.bfloat16, "fp8", "paged", seed=B, extra=12, n_q_heads=9)
    q = rows((sum(trees), 9, 64), torch.bfloat16, 36).cuda()
    for n_splits in (0, 1, 5):   # up to 33 rows: several row blocks
        check(c, q, parents, c.attend(q, parents, kv.KV_OUT_F32, n_splits), True)
