"""How a launch of kv_tree_attn shares its work out (host arithmetic, no GPU)."""
import os
import random
import subprocess

import pytest

from conftest import ROOT


@pytest.fixture(scope="module")
def cut(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("cut") / "tree_cut_harness")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I",
                           os.path.join(ROOT, "paper_2604_26557_amd", "csrc"), os.path.join(ROOT, "tests", "tree_cut_harness.cpp"), "-o", exe])

    def run(cases):
        """cases: (D, H, G, bits, paged, n_splits, ws_splits, lens, drafted)"""
        text = "".join(f"{D} {H} {G} {bits} 256 {int(paged)} {len(lens)} {n} {ws} {' '.join(map(str, lens))} {' '.join(map(str, drafted))}\n"
                       for D, H, G, bits, paged, n, ws, lens, drafted in cases)
        out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout.splitlines()
        assert len(out) == len(cases)
        return [dict(zip(("nb", "row_blocks", "ns", "split_tokens", "most"), map(int, line.split()))) for line in out]
    return run


def test_every_cut_covers_rows_and_tokens_within_the_workspace(cut):
    rnd = random.Random(5)
    cases = []
    for _ in range(800):
        B = rnd.choice([1, 1, 2, 3, 16, 17, 40])
        lens = [rnd.choice([0, 1, 31, 32, 33, 700, 4096, 32768, rnd.randrange(1, 200000), 1 << 30]) for _ in range(B)]
        drafted = [rnd.choice([0, 1, 1, 3, 16, 64, 256]) for _ in range(B)]
        drafted[rnd.randrange(B)] = rnd.choice([1, 8, 64])
        cases.append((rnd.choice([64, 128, 256]), rnd.choice([1, 2, 8, 32]), rnd.choice([1, 4, 7, 20, 4095]), rnd.choice([16, 8, 4]), rnd.random() < 0.5,
                      rnd.choice([0, 0, 0, 1, 2, 7, 128]), rnd.choice([-1, -1, 0, 1, 3, 500]), lens, drafted))
    for case, c in zip(cases, cut(cases)):
        D, H, G, bits, paged, n, ws, lens, drafted = case
        rows = max(drafted) * G
        longest = max(a + t for a, t in zip(lens, drafted) if t)
        assert c["nb"] in (1, 2, 4) and (D != 256 or c["nb"] <= 2), case
        assert 16 * c["nb"] * c["row_blocks"] >= rows > 16 * c["nb"] * (c["row_blocks"] - 1), case
        assert c["split_tokens"] % 32 == 0 and c["ns"] * c["split_tokens"] >= longest > (c["ns"] - 1) * c["split_tokens"], case
        limit = n or c["most"]
        assert 1 <= c["ns"] <= max(1, min(limit, 128, c["most"] if ws == -1 else ws)), case


def test_an_asked_number_of_splits_is_taken(cut):
    """As far as whole steps of 32 tokens allow."""
    for n, c in zip((1, 2, 5, 100), cut([(128, 2, 4, 16, False, n, 128, [32 * 128 * 100], [1]) for n in (1, 2, 5, 100)])):
        assert c["ns"] == n
    assert cut([(128, 2, 4, 16, False, 100, 128, [64], [1])])[0]["ns"] == 3   # 65 tokens


def test_the_chip_is_filled_and_short_calls_are_not_split(cut):
    long, short, wide = cut([(128, 8, 4, 16, False, 0, -1, [32768], [1]), (64, 2, 4, 16, False, 0, -1, [100], [1]), (128, 8, 4, 8, False, 0, -1, [4096] * 64, [16] * 64)])
    assert long["ns"] * 8 >= 128 and long["nb"] == 1
    assert short["ns"] == 1
    assert wide["ns"] <= 2 and wide["nb"] == 4
