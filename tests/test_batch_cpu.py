"""The host side of a batch's step: refusals (checked before anything is launched), and how kv_group_attn shares its work out."""
import ctypes as C
import os
import random
import subprocess

import pytest
import torch

from conftest import ROOT
from paper_2604_26557_amd import binding as kv
from test_serving_cpu import Fake, P


# ------------------------------------------------------------------------------------------ tables
def tables(**kw):
    a = dict(batch=4, block_tokens=16, max_blocks=8, n_pool=20, n_tok=9, reserved=0)
    a.update({n: P * (i + 1) for i, n in enumerate(("seq_lens", "new_lens", "leader", "shared", "held", "n_free", "block_table", "free_ids", "held_out", "n_free_out",
                                                    "block_table_out", "tok_first", "tok_seq", "tok_slot", "status"))})
    a.update(kw)
    return kv.lib().kv_step_tables(C.byref(kv.kv_tables_args_t(**a)), None)


@pytest.mark.parametrize("kw", [dict(batch=0), dict(batch=-1), dict(batch=8193), dict(block_tokens=0), dict(max_blocks=-1), dict(n_pool=-1), dict(n_tok=-1), dict(leader=None),
                                dict(shared=None), dict(held_out=P * 5), dict(n_free_out=P * 6), dict(block_table_out=P * 7), dict(held_out=P * 5, n_free_out=P * 6)] +
                         [{n: None} for n in ("seq_lens", "new_lens", "held", "n_free", "block_table", "free_ids", "held_out", "n_free_out", "block_table_out", "tok_first",
                                              "tok_seq", "tok_slot", "status")])
def test_tables_refusals(kw):
    assert tables(**kw) == kv.KV_EINVAL


def test_tables_too_large():
    assert tables(batch=8192, max_blocks=1 << 18) == kv.KV_ERANGE
    assert kv.lib().kv_step_tables(None, None) == kv.KV_EINVAL


def test_binding_of_tables():
    i = lambda *shape: torch.zeros(shape, dtype=torch.int32)  # noqa: E731
    ok = dict(block_tokens=16, seq_lens=i(3), new_lens=i(3), held=i(3), free_ids=i(9), n_free=i(1), block_table=i(3, 5), tok_first=i(4), tok_seq=i(7), tok_slot=i(7), status=i(2))
    s = kv.step_tables(**ok).struct
    assert (s.batch, s.max_blocks, s.n_pool, s.n_tok) == (3, 5, 9, 7) and s.held_out == s.held and s.block_table_out == s.block_table and s.leader is None
    other = dict(held_out=i(3), n_free_out=i(1), block_table_out=i(3, 5))
    assert kv.step_tables(**ok, **other).struct.held_out == other["held_out"].data_ptr()
    for kw in (dict(new_lens=i(2)), dict(held=i(3).long()), dict(tok_first=i(3)), dict(tok_slot=i(6)), dict(status=i(1)), dict(block_table=i(2, 5)), dict(block_table=i(15)),
               dict(leader=i(2), shared=i(3)), dict(held_out=i(3)), dict(other, block_table_out=i(3, 4)), dict(block_table=i(5, 3).T), dict(free_ids=i(18)[::2])):
        with pytest.raises(kv.KVError) as e:
            kv.step_tables(**{**ok, **kw})
        assert e.value.code == kv.KV_EINVAL, kw


# ------------------------------------------------------------------------------------------ attention
def attend(f, first=(0, 1, 2), groups=((0, 2), (20,)), scores=None, ws=P, ws_bytes=1 << 20, layer=0, null=(), **kw):
    """A call that a check refuses, or that has no tokens."""
    a = dict(q=P, out=P, q_stride_t=256, q_stride_h=64, out_stride_t=256, out_stride_h=64, tok_first_host=(C.c_int32 * 3)(*first), tok_first_dev=P, mask=None, mask_words=0,
             out_dtype=0, n_splits=0, scale=0.0)
    a.update(kw)
    g = s = None
    if groups is not None:
        gf, pf = (C.c_int32 * len(groups[0]))(*groups[0]), (C.c_int32 * max(1, len(groups[1])))(*groups[1])
        x = dict(n_groups=len(groups[1]), reserved=0, first_host=gf, first_dev=P, prefix_host=pf, prefix_dev=P)
        x.update({n: None for n in null})
        g = C.byref(kv.kv_groups_t(**x))
    if scores is not None:
        s = C.byref(kv.kv_scores_t(**scores))
    return kv.lib().kv_group_attn(*f.refs(), layer, C.byref(kv.kv_tree_args_t(**a)), g, s, ws, ws_bytes, None)


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("fmt", [0, 1, 2])
def test_attention_refusals(paged, fmt):
    ok = Fake(paged=paged, fmt=fmt)   # contexts of 50 and 60 tokens
    none = (0, 0, 0)
    assert attend(ok, none) == kv.KV_OK and attend(ok, none, None) == kv.KV_OK and attend(ok, none, scores=dict(softcap=30.0)) == kv.KV_OK
    assert attend(ok, none, ((1, 1, 2), (70, 60))) == kv.KV_OK   # an empty group, and one of a whole context
    for kw in (dict(ws=None), dict(ws=P + 8), dict(tok_first_host=None), dict(tok_first_dev=None), dict(out_dtype=2), dict(n_splits=-1), dict(n_splits=129),
               dict(scale=float("nan")), dict(first=(1, 1, 1)), dict(first=(0, 2, 1)), dict(q=None), dict(out=None), dict(q=P + 8), dict(q_stride_t=4), dict(out_stride_h=-1),
               dict(groups=((0, 2), (51,))), dict(groups=((0, 3), (20,))), dict(groups=((-1, 2), (20,))), dict(groups=((0, 2, 1), (20, 20))), dict(groups=((0, 2), (-1,))),
               dict(groups=((0,) * 66, (0,) * 65)), dict(null=("first_host",)), dict(null=("first_dev",)), dict(null=("prefix_host",)), dict(null=("prefix_dev",)),
               dict(scores=dict(softcap=-1.0)), dict(scores=dict(softcap=float("inf"))), dict(scores=dict(softcap=float("nan"))), dict(scores=dict(slopes=P)),
               dict(scores=dict(softcap=1.0e-45), scale=1.0e30)):
        assert attend(ok, **kw) == kv.KV_EINVAL, kw
    for kw in (dict(layer=1), dict(layer=-1), dict(first=(0, 0, 101)), dict(first=(0, 65, 65), mask=P, mask_words=1), dict(first=(0, 1, 1), mask=P, mask_words=0)):
        assert attend(ok, **kw) == kv.KV_ERANGE, kw
    assert attend(ok, ws_bytes=2 * 2 * 4 * 66 * 4 - 1) == kv.KV_ENOSPC   # two results of each of 2 tokens x 4 heads
    assert attend(Fake(paged=paged, fmt=fmt, D=96), none) == kv.KV_EINVAL
    assert attend(Fake(paged=paged, fmt=fmt, seq_lens_dev=None), none) == kv.KV_EINVAL
    assert kv.lib().kv_group_attn_workspace(None, 1, 1) == 0 and kv.lib().kv_group_attn_workspace(ok.plan.handle, -1, 1) == 0
    assert kv.kv_group_attn_workspace(ok.plan, 64, 32768) > 0


def test_prompts_may_be_longer_than_drafts():
    f = Fake(paged=True, max_blocks_per_seq=1 << 27)
    f.lens[0] = 1 << 29
    assert attend(f, (0, 257, 257), None, mask=P, mask_words=64) == kv.KV_ERANGE
    assert attend(f, (0, (1 << 29) + 1, (1 << 29) + 1), None) == kv.KV_ERANGE
    # 3000 tokens pass the checks of their number: the next one refuses the call
    assert attend(f, (0, 3000, 3000), None, q=None) == kv.KV_EINVAL


def test_binding_of_attention():
    plan = kv.kv_layout_plan(1, 2, 4, 64, [32], kv.KV_F16, 512, 4096, kv.KV_PER_SEQ)
    k = torch.zeros((1, 2, 32, 64), dtype=torch.float16)
    view = kv.bhsd_view([k], [k], [20], torch.zeros(1, dtype=torch.int32))
    i = torch.zeros(8, dtype=torch.int32)
    q, ws = torch.zeros((4, 4, 64), dtype=torch.float16), torch.zeros(16, dtype=torch.uint8)
    tree = kv.tree_batch([0, 4], i[:2])
    for call in (lambda: kv.prefix_groups([0, 1], i[:1], [5], i[:1]), lambda: kv.prefix_groups([0, 1], i, [5, 6], i), lambda: kv.prefix_groups([0, 1], i.long(), [5], i),
                 lambda: kv.scores(slopes=torch.zeros(4).double()), lambda: kv.scores(sees_from=i.long()), lambda: kv.scores(slopes=torch.zeros(8)[::2], positions=i),
                 lambda: kv.kv_group_attn(plan, view, None, 0, tree, q[:3], q[:3], kv.KV_OUT_SAME, 0, ws),
                 lambda: kv.kv_group_attn(plan, view, None, 0, tree, q, q, kv.KV_OUT_F32, 0, ws),
                 lambda: kv.kv_group_attn(plan, view, None, 0, tree, q, q, kv.KV_OUT_SAME, 0, ws, scores=kv.scores(slopes=torch.zeros(3), positions=i)),
                 lambda: kv.kv_group_attn(plan, view, None, 0, tree, q, q, kv.KV_OUT_SAME, 0, ws, scores=kv.scores(sees_to=i[:3]))):
        with pytest.raises(kv.KVError) as e:
            call()
        assert e.value.code == kv.KV_EINVAL


@pytest.fixture(scope="module")
def cut(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("cut") / "group_cut_harness")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I",
                           os.path.join(ROOT, "paper_2604_26557_amd", "csrc"), os.path.join(ROOT, "tests", "group_cut_harness.cpp"), "-o", exe])

    def run(cases):
        """cases: (D, H, G, bits, paged, chain, n_splits, ws_splits, lens, news, group_first, prefix)"""
        text = "".join(f"{D} {H} {G} {bits} {int(paged)} {int(chain)} {n} {ws} {len(lens)} {len(prefix)} {' '.join(map(str, lens + news + gf + prefix))}\n"
                       for D, H, G, bits, paged, chain, n, ws, lens, news, gf, prefix in cases)
        out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout.splitlines()
        assert len(out) == len(cases)
        return [dict(zip(("nb", "prefix_tokens", "split_tokens", "prefix_ns", "ns", "fit", "workgroups", "covered", "units"), map(int, line.split()))) for line in out]
    return run


def test_every_cut_covers_prefixes_and_own_tokens_within_the_workspace(cut):
    rnd = random.Random(6)
    cases = []
    for _ in range(800):
        B = rnd.choice([1, 2, 3, 16, 17, 70])
        n = rnd.choice([0, 1, 2, 4]) if B > 1 else rnd.choice([0, 1])
        gf = sorted(rnd.randint(0, B) for _ in range(n + 1))
        prefix = [rnd.choice([0, 1, 31, 32, 33, 1000, 16384, 1 << 29]) for _ in range(n)]
        lens = [max([p for g, p in enumerate(prefix) if gf[g] <= b < gf[g + 1]], default=0) + rnd.choice([0, 1, 31, 700, 4096, rnd.randrange(1, 100000), 1 << 28]) for b in range(B)]
        chain = rnd.random() < 0.7
        news = [rnd.choice([0, 1, 1, 3, 16, 64, 256] + ([4096, 100000] if chain else [])) for _ in range(B)]
        news[rnd.randrange(B)] = rnd.choice([1, 8, 64])
        cases.append((rnd.choice([64, 128, 256]), rnd.choice([1, 2, 8, 32]), rnd.choice([1, 4, 7, 20, 4095]), rnd.choice([16, 8, 4]), rnd.random() < 0.5, chain,
                      rnd.choice([0, 0, 0, 1, 2, 7, 128]), rnd.choice([-1, -1, 2, 3, 5, 500]), lens, news, gf, prefix))
    for case, c in zip(cases, cut(cases)):
        D = case[0]
        assert c["covered"] == c["units"] and c["nb"] in ((1, 2) if D == 256 else (1, 2, 4)), (case, c)
        assert c["split_tokens"] % 32 == 0 and c["prefix_tokens"] % 32 == 0 and 0 <= c["prefix_ns"] <= c["ns"] <= 128
        assert c["ns"] <= max(2, c["fit"]), (case, c)   # two are what the call asks room for where there is a prefix; one result needs none
        assert c["ns"] <= c["fit"] or c["ns"] == 1
        assert c["workgroups"] > 0


# ------------------------------------------------------------------------------------------ sampling
@pytest.mark.parametrize("kw", [dict(dtype=3), dict(dtype=-1), dict(n_rows=-1), dict(n_vocab=0), dict(stride=-1), dict(logits=None), dict(u=None), dict(tokens=None), dict(logits=P + 2),
                                dict(ws=None), dict(ws=P + 8)])
def test_sample_refusals(kw):
    a = dict(logits=P, stride=100, n_rows=2, n_vocab=100, dtype=kv.KV_F32, u=P, tokens=P)
    ws = kw.pop("ws", P) if "ws" in kw else P
    a.update(kw)
    assert kv.lib().kv_sample(C.byref(kv.kv_sample_args_t(**a)), ws, 1 << 24, None) == kv.KV_EINVAL


def test_sample_sizes():
    a = dict(logits=P, stride=100, n_rows=0, n_vocab=100, dtype=kv.KV_F32, u=P, tokens=P)
    call = lambda **kw: kv.lib().kv_sample(C.byref(kv.kv_sample_args_t(**{**a, **kw})), P, kw.pop("ws_bytes", 1 << 30), None)  # noqa: E731
    assert call() == kv.KV_OK   # no rows: nothing is launched
    assert call(n_rows=2, n_vocab=(1 << 24) + 1) == kv.KV_ERANGE
    assert call(n_rows=1 << 22) == kv.KV_ERANGE   # threads of a launch
    assert kv.lib().kv_sample(None, P, 1 << 20, None) == kv.KV_EINVAL
    assert kv.lib().kv_sample(C.byref(kv.kv_sample_args_t(**{**a, "n_rows": 2})), P, kv.kv_sample_workspace(2, 100) - 1, None) == kv.KV_ENOSPC
    assert kv.kv_sample_workspace(1, 1000) >= 16 and kv.kv_sample_workspace(-1, 10) == 0 and kv.kv_sample_workspace(1, -1) == 0


def test_binding_of_sample():
    x, f, i, ws = torch.zeros((3, 50)), torch.zeros(3), torch.zeros(3, dtype=torch.int32), torch.zeros(16, dtype=torch.uint8)
    for call in (lambda: kv.kv_sample(x.double(), f, i, ws), lambda: kv.kv_sample(x.T, f, i, ws), lambda: kv.kv_sample(x, f[:2], i, ws), lambda: kv.kv_sample(x, f, i.long(), ws),
                 lambda: kv.kv_sample(x, f, i, ws, temperature=f.double()), lambda: kv.kv_sample(x, f, i, ws, top_k=f), lambda: kv.kv_sample(x, f, i, ws, probs=f[:1]),
                 lambda: kv.kv_sample(x, f, i, ws, top_p=torch.zeros(6)[::2])):
        with pytest.raises(kv.KVError) as e:
            call()
        assert e.value.code == kv.KV_EINVAL
