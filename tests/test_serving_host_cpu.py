"""The serving step's host side where it is easily got wrong: ends of schedules, sizes, kinds of tensors."""
import ctypes as C
import math
import os
import random
import subprocess

import numpy as np
import pytest
import torch

from conftest import ROOT
from paper_2604_26557_amd import binding as kv
from test_serving_cpu import P, Fake
from test_tree_cut_cpu import cut  # noqa: F401
from treeshapes import SHAPES, without_a_context


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


@pytest.fixture(scope="module")
def units(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("units") / "tree_units_harness")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I",
                           os.path.join(ROOT, "paper_2604_26557_amd", "csrc"), os.path.join(ROOT, "tests", "tree_units_harness.cpp"), "-o", exe])

    def run(cases):
        """cases: (D, H, G, n_splits, ws_splits, lens, drafted)"""
        text = "".join(f"{D} {H} {G} {n} {ws} {len(lens)} {' '.join(map(str, lens))} {' '.join(map(str, drafted))}\n" for D, H, G, n, ws, lens, drafted in cases)
        out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout.splitlines()
        assert len(out) == len(cases)
        return [tuple(map(int, line.split())) for line in out]
    return run


def test_workgroups_past_the_last_split_have_no_tokens(units):
    """Every token of a sequence is gone over once per head and row block, also where the numbers of splits that do not exist times their tokens pass 32 bits."""
    rnd = random.Random(3)
    cases = [(128, 1, 40, 1, 1, [n, 5], [4, 3]) for n in (1, 1000, 1 << 28, 306783379, 306783380, 1 << 29, (1 << 30) - 1, 1 << 30)]
    cases += [(128, 1, 40, 0, 0, [1 << 30] * 3, [2, 1, 200])]
    for _ in range(300):
        B = rnd.randint(2, 64)
        cases.append((rnd.choice([64, 128, 256]), rnd.choice([1, 2, 3, 5, 8]), rnd.choice([1, 4, 20, 40]), rnd.choice([0, 0, 1, 3]), rnd.choice([0, 1, 4, 128]),
                      [rnd.choice([0, 40, 5000, rnd.randrange(1 << 30), 1 << 30]) for _ in range(B)], [rnd.choice([1, 2, 9, 256]) for _ in range(B)]))
    past = 0
    for (D, H, G, n, ws, lens, drafted), (groups, idle, tokens, nb, split_tokens) in zip(cases, units(cases)):
        blocks = [-(-t * G // (16 * nb)) for t in drafted]
        assert tokens == H * sum((a + t) * k for a, t, k in zip(lens, drafted, blocks))
        assert groups - idle == H * sum(-(-(a + t) // split_tokens) * k for a, t, k in zip(lens, drafted, blocks))
        past += idle > 0 and 7 * split_tokens >= 1 << 31
    assert past > 50   # such launches are among them


@pytest.mark.parametrize("D,H,G", [(128, 8, 4), (64, 16, 7), (64, 4, 7), (256, 2, 3), (128, 1, 40), (64, 1, 33), (128, 1, 1), (64, 2, 100), (128, 32, 1)])
def test_a_workspace_serves_fewer_tokens_as_well(cut, D, H, G):
    """Sized for n_tok drafted tokens and max_len of context, it holds what is chosen for fewer of either: the size does not fall as they grow, and the cut is the one that
    unlimited room gives.  A call with fewer tokens may want more splits of them."""
    plan = kv.kv_layout_plan(1, H, H * G, D, [16], kv.KV_F16, 512, 4096, kv.KV_PER_SEQ)
    tokens = list(range(1, 140)) + [200, 256]
    for max_len in (0, 40, 700, 2000, 32768):
        size = [kv.kv_tree_attn_workspace(plan, n, max_len) for n in tokens]
        assert size == sorted(size)
    assert kv.kv_tree_attn_workspace(plan, 64, 700) <= kv.kv_tree_attn_workspace(plan, 64, 2000) <= kv.kv_tree_attn_workspace(plan, 64, 32768)
    rnd = random.Random(D + H + G)
    limited, free = [], []
    for _ in range(300):
        n_max, max_len = rnd.choice([16, 17, 48, 64, 65, 256]), rnd.choice([40, 700, 1100, 2080, 4000, 32768, 131072])
        n, length = rnd.randint(1, n_max), rnd.randint(max_len // 2, max_len)
        case = (D, H, G, rnd.choice([16, 8, 4]), rnd.random() < 0.5, 0)
        room = kv.kv_tree_attn_workspace(plan, n_max, max_len) // (n * H * G * (D + 2) * 4)
        limited.append(case + (room, [length], [n]))
        free.append(case + (1000, [length], [n]))
    for case, a, b in zip(limited, cut(limited), cut(free)):
        assert a == b, case


def refused(call):
    with pytest.raises(kv.KVError) as e:
        call()
    return e.value.code == kv.KV_EINVAL


def test_binding_refuses_numbers_of_another_type_or_order():
    """Indices are read as int32 side by side, masks as 64-bit words, results written as what they are asked to be: tensors of another kind would be read past
    their end, or as other tokens' numbers.  torch's default is int64."""
    plan = kv.kv_layout_plan(1, 2, 4, 64, [32], kv.KV_F16, 512, 4096, kv.KV_PER_SEQ)
    k = torch.zeros((1, 2, 32, 64), dtype=torch.float16)
    view = kv.bhsd_view([k], [k], [20], torch.zeros(1, dtype=torch.int32))
    i = torch.arange(4, dtype=torch.int32)
    rows = torch.zeros((4, 2, 64), dtype=torch.float16)
    r = kv.Rope(torch.zeros((8, 16, 2)))
    for bad in (i.long(), i.short(), i.float(), torch.arange(8, dtype=torch.int32)[::2], torch.zeros(1, dtype=torch.int32).expand(4), torch.zeros((4, 2), dtype=torch.int32)[:, 0]):
        assert refused(lambda: kv.kv_rope(r, bad, rows, rows))
        assert refused(lambda: kv.kv_cache_write(plan, view, None, 0, rows, rows, bad, i))
        assert refused(lambda: kv.kv_cache_write(plan, view, None, 0, rows, rows, i, bad))
        assert refused(lambda: kv.kv_cache_write(plan, view, None, 0, rows, rows, i, i, r, bad))
        assert refused(lambda: kv.kv_cache_read(plan, view, None, 0, bad, i, rows, rows))
        assert refused(lambda: kv.kv_cache_read(plan, view, None, 0, i, bad, rows, rows))
        assert refused(lambda: kv.tree_batch([0, 1, 2, 4], bad))
    for bad in (torch.int32, torch.float64, torch.bool, torch.uint8):
        assert refused(lambda: kv.tree_batch([0, 4], i[:2], torch.zeros((4, 1), dtype=bad)))
    assert refused(lambda: kv.tree_batch([0, 4], i[:2], torch.zeros((4, 2), dtype=torch.int64)[:, :1]))
    kv.tree_batch([0, 4], i[:2], torch.zeros((4, 1), dtype=torch.int64))
    tree = kv.tree_batch([0, 4], i[:2])
    q, ws = torch.zeros((4, 4, 64), dtype=torch.float16), torch.zeros(16, dtype=torch.uint8)
    for out, kind in ((torch.bfloat16, kv.KV_OUT_SAME), (torch.int16, kv.KV_OUT_SAME), (torch.float32, kv.KV_OUT_SAME), (torch.int32, kv.KV_OUT_F32), (torch.float16, kv.KV_OUT_F32),
                      (torch.float64, kv.KV_OUT_F32)):
        assert refused(lambda: kv.kv_tree_attn(plan, view, None, 0, tree, q, q.to(out), kind, 0, ws))


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("fmt", [0, 1, 2])
@pytest.mark.parametrize("which", ["seq_off_host", "seq_off_dev"])
def test_views_whose_rows_start_later_are_refused(paged, fmt, which):
    """The calls do not know such rows, in either layout."""
    off = (C.c_int64 * 2)(0, 0)
    ok = Fake(paged=paged, fmt=fmt)
    assert ok.attn() == ok.rows_call("kv_cache_write") == ok.rows_call("kv_cache_read") == kv.KV_OK
    setattr(ok.view, which, C.cast(off, type(getattr(ok.view, which))) if which == "seq_off_host" else P)
    assert ok.attn() == ok.rows_call("kv_cache_write") == ok.rows_call("kv_cache_read") == kv.KV_EINVAL


@pytest.mark.parametrize("D,nb", list(SHAPES))
def test_batches_for_wide_kernels_take_them(cut, D, nb):
    """What the GPU tests of 32 and 64 rows a workgroup go by: in every format and layout, with the workspace that they have."""
    cases = []
    for H, G, lens, drafted, splits in SHAPES[D, nb] + [without_a_context(SHAPES[D, nb][2])[0]]:
        plan = kv.kv_layout_plan(1, H, H * G, D, [16], kv.KV_F16, 512, 4096, kv.KV_PER_SEQ)
        room = kv.kv_tree_attn_workspace(plan, sum(drafted), max(lens) + 256) // (sum(drafted) * H * G * (D + 2) * 4)
        cases += [(D, H, G, bits, paged, n, room, lens, drafted) for n in splits for bits in (16, 8, 4) for paged in (False, True)]
    got = cut(cases)
    assert [c["nb"] for c in got] == [nb] * len(cases)
    assert max(c["ns"] for c in got) > 1 and max(c["row_blocks"] for c in got) > 1 and max(c["split_tokens"] for c in got) >= 576


def test_more_sequences_than_are_counted_one_by_one(cut):
    """From 65 sequences on workgroups are estimated from sums: the cut still covers everything, and equal batches on either side are cut alike."""
    rnd = random.Random(9)
    cases = []
    for _ in range(200):
        B = rnd.choice([64, 65, 66, 100, 300])
        cases.append((rnd.choice([64, 128, 256]), rnd.choice([1, 4, 8]), rnd.choice([1, 4, 7]), rnd.choice([16, 8, 4]), rnd.random() < 0.5, rnd.choice([0, 0, 2]), -1,
                      [rnd.choice([0, 31, 700, 4096, rnd.randrange(1, 40000)]) for _ in range(B)], [rnd.choice([1, 1, 5, 64]) for _ in range(B)]))
    for (D, H, G, bits, paged, n, ws, lens, drafted), c in zip(cases, cut(cases)):
        rows, longest = max(drafted) * G, max(a + t for a, t in zip(lens, drafted))
        assert 16 * c["nb"] * c["row_blocks"] >= rows > 16 * c["nb"] * (c["row_blocks"] - 1)
        assert c["split_tokens"] % 32 == 0 and c["ns"] * c["split_tokens"] >= longest > (c["ns"] - 1) * c["split_tokens"]
    for n, t in ((300, 1), (4096, 4), (2000, 16)):
        a, b = cut([(128, 8, 4, 8, True, 0, -1, [n] * B, [t] * B) for B in (64, 65)])
        assert a["nb"] == b["nb"] and abs(a["ns"] - b["ns"]) <= 1
