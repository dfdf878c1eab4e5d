"""kv_group_attn at the ends of what its arguments may be."""
import numpy as np
import pytest
import torch

from batchcase import Batch
from paper_2604_26557_amd import binding as kv

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("layout", ["bhsd", "paged"])
@pytest.mark.parametrize("D,cap", [(64, 0.0), (128, 9.0)])
@pytest.mark.parametrize("ends", [(1, -1), (-1, 1)])
def test_positions_as_far_apart_as_they_may_be(ends, D, cap, layout):
    """2^31 between a token and those that it sees, and a token of the same rows some 1000 behind or ahead of it. With slopes of this size the distances are biases of 0.02 to 4."""
    a, b = (e * 2 ** 30 for e in ends)
    for near in (0, 700, 1000):
        positions = [a, a, b, b - ends[1] * near]
        batch = Batch([70], [4], 1, 8, D, torch.bfloat16, "16", layout, seed=D, slopes=[2.0e-9, 1.0e-9, 1.0e-10, 1.0e-11, 1.5e-9, 0.0, -1.0e-9, -1.0e-10], positions=positions, cap=cap)
        for n_splits in (0, 1, 2):
            batch.check(batch.attend(n_splits=n_splits))


def test_many_sequences():
    """Units of some thousand sequences are counted 64 at a time by each workgroup, behind 64 groups of which some are of nobody."""
    B = 3001
    rng = np.random.default_rng(1)
    first = sorted(rng.integers(0, B, 65).tolist())
    b = Batch((rng.integers(0, 20, B) + 20).tolist(), rng.integers(0, 3, B).tolist(), 1, 2, 64, torch.float16, "16", "bhsd", seed=2, first=first, prefix=rng.integers(0, 21, 64).tolist())
    for n_splits in (0, 2):
        b.check(b.attend(n_splits=n_splits))


@pytest.mark.parametrize("fmt", ["16", "fp8"])
def test_a_prompt_of_some_ten_thousand_tokens(fmt):
    """Rows from its first token to its last by the definition."""
    n, D = 70001, 64
    b = Batch([3], [n], 1, 2, D, torch.bfloat16, fmt, seed=3)
    got, k, v, q = b.attend(), b.rows("k", 0)[0], b.rows("v", 0)[0], b.q.double().numpy()
    u = 2.0 ** -24
    for t in (0, 1, 4095, 4096, 33333, 69999, 70000):
        for h in range(2):
            x = k[:t + 4] @ q[t, h] * D ** -0.5
            # D products and their sum, the exponent's roundings; sums of up to a step's products for every 128 tokens, and of wavefronts and splits
            e = np.abs(k[:t + 4]) @ np.abs(q[t, h]) * D ** -0.5 * (D + 8) + 8 * np.abs(x).max() + 8
            p = np.exp(x - x.max())
            p /= p.sum()
            av = np.abs(v[:t + 4])
            tol = u * (2 * ((p * e) @ av + (p @ e) * (p @ av)) + (64 + t / 32) * (p @ av))
            assert (np.abs(got[t, h].double().cpu().numpy() - p @ v[:t + 4]) <= tol).all(), (t, h)


def test_the_longest_context():
    """2^30 tokens in 4 bits: those of a few places outweigh all others, whose scores are zero."""
    n, D = (1 << 30) - 1, 64
    if torch.cuda.mem_get_info()[0] < 90 << 30:
        pytest.skip("80 GiB of cache")
    k, v = (torch.zeros((1, 1, n + 1, D // 2), dtype=torch.uint8, device="cuda") for _ in range(2))
    kz, vz = (torch.full((1, 1, n + 1, D // 32), 127, dtype=torch.uint8, device="cuda") for _ in range(2))
    at = [0, 31, (1 << 29) + 5, (1 << 30) - 40, n]
    for i, j in enumerate(at):
        k[0, 0, j], kz[0, 0, j] = 0x77, 129          # 6 * 4 in every column: a score of 24 * 64 / 8
        v[0, 0, j, i], vz[0, 0, j] = 0x52, 128 + i   # 1 * 2^(1 + i) and 3 * 2^(1 + i) in two columns of each one's own
    plan = kv.kv_layout_plan(1, 1, 1, D, [n + 1], kv.KV_F16, 512, 4096, kv.KV_PER_SEQ)
    lens, first = torch.tensor([n], dtype=torch.int32, device="cuda"), torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    view, blocks = kv.bhsd_view([k.view(torch.int16)], [v.view(torch.int16)], [n], lens), kv.scale_blocks(kv.KV_FORMAT_FP4, [kz], [vz])
    q, out = torch.ones((1, 1, D), dtype=torch.float16, device="cuda"), torch.zeros((1, 1, D), device="cuda")
    ws = torch.empty(kv.kv_group_attn_workspace(plan, 1, n), dtype=torch.uint8, device="cuda")
    want = torch.zeros(D, dtype=torch.float64)
    for i in range(len(at)):
        want[2 * i], want[2 * i + 1] = 2.0 ** (1 + i) / len(at), 3 * 2.0 ** (1 + i) / len(at)
    for n_splits in (0, 1):
        kv.kv_group_attn(plan, view, blocks, 0, kv.tree_batch([0, 1], first), q, out, kv.KV_OUT_F32, n_splits, ws)
        # five equal weights: a quotient and some sums of them
        assert (out[0, 0].double().cpu() - want).abs().max() <= 16 * 2.0 ** -24 * 32
