"""The serving step's host side: schedules of rotary frequencies, masks of trees, refusals (checked before anything is launched)."""
import ctypes as C
import math
import subprocess
import sys

import numpy as np
import pytest
import torch

from conftest import ROOT
from paper_2604_26557_amd import binding as kv

P = 1 << 20   # an address that is never read: a refused call launches nothing


# ------------------------------------------------------------------------------------------ rotary tables
def table_of(freqs, n_pos, magnitude=1.0):
    a = np.arange(n_pos)[:, None] * np.asarray(freqs)[None]
    return magnitude * np.stack([np.cos(a), np.sin(a)], -1)


def test_rope_table_plain_linear_and_base():
    n, rot = 500, 64
    f = 10000.0 ** (-np.arange(32) / 32)
    for kw, freqs, mag in ((dict(), f, 1), (dict(magnitude=1.5), f, 1.5), (dict(scaling=kv.KV_ROPE_LINEAR, factor=4.0), f / 4, 1)):
        got = kv.kv_rope_table(n, rot, **kw).numpy().astype(np.float64)
        # an angle below 500 rounded to 53 bits, and one rounding to 24
        assert np.abs(got - table_of(freqs, n, mag)).max() <= mag * (2.0 ** -24 + 500 * 2.0 ** -50)
    got = kv.kv_rope_table(n, rot, scaling=kv.KV_ROPE_BASE, factor=8.0).numpy().astype(np.float64)
    base = 10000.0 * 8 ** (64 / 62)
    assert np.abs(got - table_of(base ** (-np.arange(32) / 32), n)).max() <= 2.0 ** -24 + 1e-9
    # the longest wave is 8 times as long, the shortest as it was
    assert math.isclose(base ** (-31 / 32), 10000.0 ** (-31 / 32) / 8, rel_tol=1e-12)


def test_rope_table_by_wavelength_and_by_index():
    n, rot, trained, factor, low, high = 64, 128, 8192, 8.0, 1.0, 4.0
    f = 500000.0 ** (-np.arange(64) / 64)
    turns = trained * f / (2 * math.pi)
    keep = np.clip((turns - low) / (high - low), 0, 1)
    assert (keep == 1).any() and (keep == 0).any() and ((keep > 0) & (keep < 1)).any()
    got = kv.kv_rope_table(n, rot, 500000.0, kv.KV_ROPE_WAVELENGTH, factor, trained, low, high).numpy()
    assert np.abs(got - table_of(f * keep + f / factor * (1 - keep), n)).max() <= 2.0 ** -23
    low, high = 1.0, 32.0
    at = lambda t: 64 * math.log(trained / (t * 2 * math.pi)) / math.log(500000.0)  # noqa: E731
    first, last = math.floor(at(high)), math.ceil(at(low))
    keep = 1 - np.clip((np.arange(64) - first) / (last - first), 0, 1)
    got = kv.kv_rope_table(n, rot, 500000.0, kv.KV_ROPE_INDEX, factor, trained, low, high, 1.1).numpy()
    assert np.abs(got - table_of(f * keep + f / factor * (1 - keep), n, 1.1)).max() <= 1.1 * 2.0 ** -23


@pytest.mark.parametrize("kw", [dict(n_pos=0), dict(rot_dim=8), dict(rot_dim=24), dict(base=1.0), dict(base=float("nan")), dict(base=float("inf")), dict(scaling=5),
                                dict(scaling=-1), dict(scaling=kv.KV_ROPE_LINEAR, factor=0.5), dict(scaling=kv.KV_ROPE_LINEAR, factor=float("nan")),
                                dict(scaling=kv.KV_ROPE_WAVELENGTH, factor=2.0), dict(scaling=kv.KV_ROPE_WAVELENGTH, factor=2.0, trained_pos=10, low=4.0, high=1.0),
                                dict(scaling=kv.KV_ROPE_INDEX, factor=2.0, trained_pos=10, low=0.0), dict(magnitude=float("inf"))])
def test_rope_table_refusals(kw):
    with pytest.raises(kv.KVError) as e:
        kv.kv_rope_table(**{"n_pos": 4, "rot_dim": 32, **kw})
    assert e.value.code == kv.KV_EINVAL


def test_rope_table_too_small():
    d = kv.kv_rope_desc_t(4, 32, 0, 0, 10000.0, 1.0, 1.0, 4.0, 0.0)
    buf = (C.c_float * (4 * 32))()
    assert kv.lib().kv_rope_table(C.byref(d), buf, C.sizeof(buf) - 1) == kv.KV_ENOSPC
    assert kv.lib().kv_rope_table(C.byref(d), buf, C.sizeof(buf)) == kv.KV_OK and buf[0] == 1.0
    assert kv.lib().kv_rope_table(C.byref(d), None, 0) == kv.KV_EINVAL


# ------------------------------------------------------------------------------------------ trees
@pytest.mark.parametrize("n", [0, 1, 2, 63, 64, 65, 200, 256])
def test_tree_masks(n):
    rng = np.random.default_rng(n)
    parents = [int(rng.integers(-1, i)) for i in range(n)]
    masks, depths = kv.kv_tree_masks(parents, 4)
    for i in range(n):
        up, seen, depth = parents[i], {i}, 0
        while up >= 0:
            seen.add(up)
            up, depth = parents[up], depth + 1
        row = masks[i].numpy().view(np.uint64)
        assert {j for j in range(256) if int(row[j // 64]) >> (j % 64) & 1} == seen and depths[i] == depth


def test_tree_masks_refusals():
    for parents, words in (([0], 1), ([-2], 1), ([-1, 1], 1), ([-1] * 65, 1)):
        with pytest.raises(kv.KVError) as e:
            kv.kv_tree_masks(parents, words)
        assert e.value.code == kv.KV_ERANGE
    assert kv.lib().kv_tree_masks(None, 0, 1, None, None) == kv.KV_EINVAL
    assert kv.lib().kv_tree_masks((C.c_int32 * 1)(-1), 1, 0, None, None) == kv.KV_EINVAL
    assert kv.lib().kv_tree_masks((C.c_int32 * 1)(-1), 1, 1, None, None) == kv.KV_OK


# ------------------------------------------------------------------------------------------ refusals
def rope(**kw):
    return kv.kv_rope_t(**{**dict(table=P, n_pos=10, rot_dim=32, style=0), **kw})


@pytest.mark.parametrize("kw,rkw", [(dict(n_tok=-1), {}), (dict(n_heads=0), {}), (dict(head_dim=24), {}), (dict(head_dim=0), {}), (dict(dtype=2), {}), (dict(x=None), {}),
                                    (dict(out=None), {}), (dict(positions=None), {}), (dict(x=P + 8), {}), (dict(out=P + 2), {}), (dict(x_stride_t=4), {}),
                                    (dict(out_stride_h=-8), {}), (dict(x_stride_h=12), {}), (dict(out=P, out_stride_t=512), {}), ({}, dict(table=None)), ({}, dict(table=P + 4)),
                                    ({}, dict(n_pos=0)), ({}, dict(rot_dim=8)), ({}, dict(rot_dim=80)), ({}, dict(rot_dim=24)), ({}, dict(style=2))])
def test_rope_refusals(kw, rkw):
    a = dict(x=P, out=2 * P, x_stride_t=128, x_stride_h=64, out_stride_t=128, out_stride_h=64, positions=P, n_tok=1, n_heads=2, head_dim=64, dtype=0)
    a.update(kw)
    assert kv.lib().kv_rope(C.byref(rope(**rkw)), C.byref(kv.kv_rope_args_t(**a)), None) == kv.KV_EINVAL


def test_rope_of_nothing():
    a = kv.kv_rope_args_t(n_heads=2, head_dim=64)
    assert kv.lib().kv_rope(C.byref(rope()), C.byref(a), None) == kv.KV_OK
    assert kv.lib().kv_rope(None, C.byref(a), None) == kv.KV_EINVAL and kv.lib().kv_rope(C.byref(rope()), None, None) == kv.KV_EINVAL


class Fake:
    """A plan and a view of two sequences over addresses that are never read."""

    def __init__(self, D=64, H=2, Hq=4, paged=False, fmt=0, rows=100, **view):
        self.plan = kv.kv_layout_plan(1, H, Hq, D, [rows] * 2, kv.KV_F16, 512, 4096, kv.KV_PER_SEQ)
        self.ptr = (C.c_void_p * 1)(P)
        self.lens = (C.c_int32 * 2)(50, 60)
        row = D * (16, 8, 4)[fmt] // 16   # 16-bit elements
        v = kv.kv_view_t()
        v.layout, v.n_layers, v.k_layers, v.v_layers = int(paged), 1, self.ptr, self.ptr
        v.seq_lens_host, v.seq_lens_dev = self.lens, P
        if paged:
            v.block_tokens, v.n_pool_blocks, v.max_blocks_per_seq, v.block_table = 16, 20, 10, P
            v.layer_bytes = 20 * H * 16 * row * 2
        else:
            v.stride_b, v.stride_h, v.stride_s, v.s_alloc = H * rows * row, rows * row, row, rows
            v.layer_bytes = 2 * H * rows * row * 2
        for k, x in view.items():
            setattr(v, k, x)
        self.view = v
        zr = D // 32
        self.blocks = kv.kv_blocks_t(fmt, 1, self.ptr, self.ptr, 20 * H * 16 * zr if paged else 2 * H * rows * zr, H * (16 if paged else rows) * zr,
                                     (16 if paged else rows) * zr, zr) if fmt else None

    def refs(self):
        return self.plan.handle, C.byref(self.view), C.byref(self.blocks) if self.blocks else None

    def rows_call(self, name, layer=0, r=None, **kw):
        a = dict(k=P, v=P, k_stride_t=128, k_stride_h=64, v_stride_t=128, v_stride_h=64, tok_seq=P, tok_slot=P, n_tok=0)
        if name == "kv_cache_write":
            a.update(rope=C.pointer(r) if r is not None else None, positions=P)
        a.update(kw)
        t = kv.kv_write_args_t if name == "kv_cache_write" else kv.kv_read_args_t
        return getattr(kv.lib(), name)(*self.refs(), layer, C.byref(t(**a)), None)

    def attn(self, layer=0, first=(0, 0, 0), ws=P, **kw):
        f = (C.c_int32 * 3)(*first)
        a = dict(q=P, out=P, q_stride_t=256, q_stride_h=64, out_stride_t=256, out_stride_h=64, tok_first_host=f, tok_first_dev=P, mask=None, mask_words=0,
                 out_dtype=0, n_splits=0, scale=0.0)
        a.update(kw)
        return kv.lib().kv_tree_attn(*self.refs(), layer, C.byref(kv.kv_tree_args_t(**a)), ws, 1 << 20, None)


@pytest.mark.parametrize("name", ["kv_cache_write", "kv_cache_read"])
@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("fmt", [0, 1, 2])
def test_row_refusals(name, paged, fmt):
    ok = Fake(paged=paged, fmt=fmt)
    assert ok.rows_call(name) == kv.KV_OK   # no rows: nothing is launched
    for kw in (dict(n_tok=-1), dict(n_tok=1, k=None), dict(n_tok=1, v=None), dict(n_tok=1, tok_seq=None), dict(n_tok=1, tok_slot=None), dict(n_tok=1, k=P + 8),
               dict(n_tok=1, v=P + 2), dict(k_stride_t=4), dict(v_stride_h=-64)):
        assert ok.rows_call(name, **kw) == kv.KV_EINVAL, kw
    assert ok.rows_call(name, layer=1) == kv.KV_ERANGE and ok.rows_call(name, layer=-1) == kv.KV_ERANGE
    bad = [dict(layout=2), dict(k_layers=None), dict(layer_bytes=ok.view.layer_bytes - 1)]
    bad += [dict(block_table=None), dict(block_tokens=0), dict(n_pool_blocks=-1), dict(n_pool_blocks=21)] if paged else \
        [dict(stride_b=-8), dict(stride_h=4), dict(s_alloc=-1), dict(s_alloc=101), dict(stride_s=2 ** 40), dict(stride_b=2 ** 62), dict(seq_off_dev=P)]
    for kw in bad:
        rc = Fake(paged=paged, fmt=fmt, **kw).rows_call(name)
        assert rc in (kv.KV_EINVAL, kv.KV_ERANGE), kw
    null = (C.c_void_p * 1)(None)
    assert Fake(paged=paged, fmt=fmt, k_layers=null).rows_call(name) == kv.KV_EINVAL
    assert Fake(paged=paged, fmt=fmt, v_layers=(C.c_void_p * 1)(P + 8)).rows_call(name) == kv.KV_EINVAL
    if fmt:
        for key, value, rc in (("format", 3, kv.KV_EINVAL), ("format", 0, kv.KV_EINVAL), ("n_layers", 0, kv.KV_ERANGE), ("stride_b", -1, kv.KV_EINVAL),
                               ("layer_bytes", ok.blocks.layer_bytes - 1, kv.KV_ERANGE), ("k_scales", null, kv.KV_EINVAL), ("stride_s", 2 ** 61, kv.KV_ERANGE)):
            f = Fake(paged=paged, fmt=fmt)
            setattr(f.blocks, key, value)
            assert f.rows_call(name) == rc, key
    assert Fake(D=48, paged=paged, fmt=0).rows_call(name) == kv.KV_EINVAL
    if name == "kv_cache_write":
        assert ok.rows_call(name, r=rope()) == kv.KV_OK
        assert ok.rows_call(name, r=rope(rot_dim=80)) == kv.KV_EINVAL and ok.rows_call(name, r=rope(table=None)) == kv.KV_EINVAL
        assert ok.rows_call(name, r=rope(), n_tok=1, positions=None) == kv.KV_EINVAL
    assert getattr(kv.lib(), name)(None, None, None, 0, None, None) == kv.KV_EINVAL


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("fmt", [0, 1, 2])
def test_attention_refusals(paged, fmt):
    ok = Fake(paged=paged, fmt=fmt)
    assert ok.attn() == kv.KV_OK
    for kw in (dict(ws=None), dict(ws=P + 8), dict(tok_first_host=None), dict(tok_first_dev=None), dict(out_dtype=2), dict(n_splits=-1), dict(n_splits=129),
               dict(scale=float("nan")), dict(scale=float("inf")), dict(first=(1, 1, 1)), dict(first=(0, 2, 1)), dict(first=(0, 1, 1), q=None), dict(first=(0, 1, 1), out=None),
               dict(first=(0, 1, 1), q=P + 8), dict(first=(0, 1, 1), q_stride_t=4), dict(first=(0, 1, 1), out_stride_h=-1)):
        assert ok.attn(**kw) == kv.KV_EINVAL, kw
    for kw in (dict(layer=1), dict(layer=-1), dict(first=(0, 257, 257)), dict(first=(0, 65, 65), mask=P, mask_words=1), dict(first=(0, 1, 1), mask=P, mask_words=0),
               dict(first=(0, 0, 101))):   # the last: 60 + 101 rows in room for 100, or 160
        assert ok.attn(**kw) == kv.KV_ERANGE, kw
    assert Fake(paged=paged, fmt=fmt, D=96).attn() == kv.KV_EINVAL
    assert Fake(paged=paged, fmt=fmt, seq_lens_dev=None).attn() == kv.KV_EINVAL
    f = Fake(paged=paged, fmt=fmt)
    f.lens[0] = -1
    assert f.attn() == kv.KV_EINVAL
    f.lens[0] = 2 ** 31 - 1
    assert f.attn() == kv.KV_ERANGE
    if fmt:   # a row's scales are loaded at once
        f = Fake(paged=paged, fmt=fmt)
        f.blocks.stride_s += 1
        f.blocks.layer_bytes *= 2
        assert f.attn() == kv.KV_EINVAL
    assert kv.lib().kv_tree_attn_workspace(None, 1, 1) == 0 and kv.lib().kv_tree_attn_workspace(ok.plan.handle, -1, 1) == 0
    assert kv.kv_tree_attn_workspace(ok.plan, 64, 32768) > 0


def test_binding_refuses_tensors_that_do_not_fit():
    plan = kv.kv_layout_plan(1, 2, 4, 64, [32], kv.KV_F16, 512, 4096, kv.KV_PER_SEQ)
    k = torch.zeros((1, 2, 32, 64), dtype=torch.float16)
    view = kv.bhsd_view([k], [k], [20], torch.zeros(1, dtype=torch.int32))
    i = torch.zeros(4, dtype=torch.int32)
    rows = torch.zeros((4, 2, 64), dtype=torch.float16)
    r = kv.Rope(torch.zeros((8, 16, 2)))
    for call in (lambda: kv.kv_cache_write(plan, view, None, 0, rows.float(), rows.float(), i, i), lambda: kv.kv_cache_write(plan, view, None, 0, rows[:, :1], rows[:, :1], i, i),
                 lambda: kv.kv_cache_write(plan, view, None, 0, rows, rows, i[:3], i), lambda: kv.kv_cache_write(plan, view, None, 0, rows, rows, i, i, r),
                 lambda: kv.kv_cache_write(plan, view, None, 0, rows.bfloat16(), rows.bfloat16(), i, i), lambda: kv.kv_cache_read(plan, view, None, 0, i, i, rows, rows[..., :32]),
                 lambda: kv.kv_rope(r, i[:3], rows, rows), lambda: kv.kv_rope(r, i, rows.double(), rows.double()), lambda: kv.kv_rope(r, i, rows, rows[:, :1]),
                 lambda: kv.tree_batch([0, 4], i[:1]), lambda: kv.tree_batch([0, 4], i[:2], torch.zeros((3, 1), dtype=torch.int64))):
        with pytest.raises(kv.KVError) as e:
            call()
        assert e.value.code == kv.KV_EINVAL
    tree = kv.tree_batch([0, 4], i[:2])
    q, ws = torch.zeros((4, 4, 64), dtype=torch.float16), torch.zeros(16, dtype=torch.uint8)
    for call in (lambda: kv.kv_tree_attn(plan, view, None, 0, tree, q[:3], q[:3], kv.KV_OUT_SAME, 0, ws), lambda: kv.kv_tree_attn(plan, view, None, 0, tree, q, q, kv.KV_OUT_F32, 0, ws),
                 lambda: kv.kv_tree_attn(plan, view, None, 0, tree, q[:, :2], q[:, :2], kv.KV_OUT_SAME, 0, ws),
                 lambda: kv.kv_tree_attn(plan, view, None, 0, kv.tree_batch([0, 2, 4], i[:3]), q, q, kv.KV_OUT_SAME, 0, ws)):
        with pytest.raises(kv.KVError) as e:
            call()
        assert e.value.code == kv.KV_EINVAL


def test_importing_the_binding_needs_no_torch():
    """What the binding did before: torch is imported when the library is loaded, not with the module."""
    code = "import sys; sys.path.insert(0, %r); from paper_2604_26557_amd import binding; print('torch' in sys.modules)" % ROOT
    assert subprocess.check_output([sys.executable, "-c", code], text=True).strip() == "False"


@pytest.mark.parametrize("fmt", [0, 1, 2])
def test_attention_refuses_groups_and_contexts_past_its_arithmetic(fmt):
    """4095 query heads per KV head and 2^30 tokens are the most."""
    def fake(Hq, n):
        f = Fake(H=1, Hq=Hq, paged=True, fmt=fmt, max_blocks_per_seq=1 << 27)
        f.lens[0] = n
        return f.attn()
    assert fake(4095, 50) == kv.KV_OK and fake(4096, 50) == kv.KV_EINVAL
    assert fake(4, 1 << 30) == kv.KV_OK and fake(4, (1 << 30) + 1) == kv.KV_ERANGE
