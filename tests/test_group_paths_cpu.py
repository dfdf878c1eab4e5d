"""Which kernels of kv_group_attn the batches of the GPU tests take: without a GPU, by the choice that the call makes."""
import os
import subprocess

import pytest

from conftest import ROOT
from widecase import EIGHT_BITS, SHAPES, WIDTHS, path_line, shape_of

PATHS = ("none", "apart", "joined")


@pytest.fixture(scope="module")
def paths(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("paths") / "group_path_harness")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I",
                           os.path.join(ROOT, "paper_2604_26557_amd", "csrc"), os.path.join(ROOT, "tests", "group_path_harness.cpp"), "-o", exe])

    def run(lines):
        out = subprocess.run([exe], input="".join(lines), capture_output=True, text=True, check=True).stdout.splitlines()
        assert len(out) == len(lines)
        rows = [[int(x) for x in line.split()] for line in out]
        return [(PATHS[r[0]], r[1], r[2] if r[0] == 1 else r[1]) for r in rows]
    return run


def test_every_kernel_has_a_batch(paths):
    """Row groups of a workgroup, with prefixes apart, joined and without any, in every format, of plain and of shaped scores; of chains, of windows and of trees."""
    for D in (64, 128, 256):
        most = 2 if D == 256 else 4
        want = {(D, path, nb, nb) for path in PATHS for nb in (2, most)} | {(D, "apart", 1, most)}
        assert want == {k for k in SHAPES if k[0] == D}
    cases = [(key, fmt, pow2, shaped, chain, bounded) for key in SHAPES for fmt in WIDTHS for pow2 in (0, 1) for shaped in (False, True)
             for chain, bounded in ((True, False), (True, True), (False, False)) if chain > bounded or not (fmt == "fp8" and key in EIGHT_BITS)]
    got = paths([path_line(key[0], fmt, "paged", chain, bounded, shaped, shape_of(key, fmt, pow2)) for key, fmt, pow2, shaped, chain, bounded in cases])
    for case, path in zip(cases, got):
        assert path == case[0][1:], (case, path)
