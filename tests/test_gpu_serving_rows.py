"""Row kernels of a serving step with so many rows that a thread goes over two or four heads: the same bits as with few."""
import numpy as np
import pytest
import torch

from paper_2604_26557_amd import binding as kv
from servecase import FORMATS
from treeshapes import LAYOUTS, WideCache

pytestmark = pytest.mark.gpu

# heads, head_dim, rows: two heads a thread from 1024 wavefronts of one on, four from 2048; last threads with one, two and three heads of theirs
SIZES = [(3, 64, 11500), (5, 64, 27000), (6, 128, 11500), (7, 128, 10000), (4, 256, 8500), (2, 128, 8500)]


def rows(shape, dtype, seed):
    return torch.from_numpy(np.random.default_rng(seed).standard_normal(shape, dtype=np.float32)).to(dtype).cuda()


def pieces(n, step=97):
    return [slice(i, min(i + step, n)) for i in range(0, n, step)]


def test_sizes_take_several_heads_a_thread():
    """As heads_per_thread counts them: 64-lane wavefronts of vectors of eight elements (16 in the rotation)."""
    per = [[4 if h >= 4 and n * h * (D // w) // 64 >= 8192 else 2 if h >= 2 and n * h * (D // w) // 64 >= 2048 else 1 for h, D, n in SIZES] for w in (8, 16)]
    assert all({2, 4} <= set(p) and 1 not in p for p in per)
    assert all(97 * h * (D // 8) // 64 < 2048 for h, D, _ in SIZES)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("style", [kv.KV_ROPE_HALF, kv.KV_ROPE_PAIRS])
@pytest.mark.parametrize("h,D,n", SIZES)
def test_rotation_of_many_rows(dtype, style, h, D, n):
    x = rows((n, h, D), dtype, 1)
    rope = kv.Rope(kv.kv_rope_table(3000, D // 2 if style else D).cuda(), style)
    pos = torch.from_numpy(np.random.default_rng(2).integers(-1, 3001, n).astype(np.int32)).cuda()
    few = torch.empty_like(x)
    for s in pieces(n):
        kv.kv_rope(rope, pos[s].contiguous(), x[s], few[s])
    out = torch.zeros((n, h + 1, D), dtype=dtype, device="cuda")
    kv.kv_rope(rope, pos, x, out[:, :h])
    assert torch.equal(out[:, :h].view(torch.int16), few.view(torch.int16)) and (out[:, h] == 0).all()
    kv.kv_rope(rope, pos, x, x)
    assert torch.equal(x.view(torch.int16), few.view(torch.int16))


@pytest.mark.parametrize("fmt", list(FORMATS))
@pytest.mark.parametrize("style", [None, kv.KV_ROPE_HALF, kv.KV_ROPE_PAIRS])
@pytest.mark.parametrize("h,D,n", SIZES)
def test_many_rows_into_and_out_of_a_cache(fmt, style, h, D, n):
    dtype, layout = (torch.float16, LAYOUTS[0]) if h % 2 else (torch.bfloat16, LAYOUTS[1])
    many, few = (WideCache([n // 2, n - n // 2 + 30], h, D, 1, dtype, fmt, layout, 5, 3) for _ in range(2))
    rng = np.random.default_rng(4)
    seq = torch.from_numpy((np.arange(n) % 2).astype(np.int32)).cuda()
    slot = np.empty(n, dtype=np.int32)
    for b in range(2):
        slot[b::2] = rng.permutation(n // 2 + 5)[:len(slot[b::2])]
    slot[::1001] = -1                      # without a place
    slot = torch.from_numpy(slot).cuda()
    pos = torch.from_numpy(rng.integers(0, 3000, n).astype(np.int32)).cuda()
    rope = None if style is None else kv.Rope(kv.kv_rope_table(3000, D // 2 if style else D).cuda(), style)
    k, v = rows((n, h, D), dtype, 5), rows((n, h, D), dtype, 6)
    kv.kv_cache_write(many.plan, many.view, many.blocks, 0, k, v, seq, slot, rope, pos if rope else None)
    for s in pieces(n):
        kv.kv_cache_write(few.plan, few.view, few.blocks, 0, k[s], v[s], seq[s].contiguous(), slot[s].contiguous(), rope, pos[s].contiguous() if rope else None)
    for name in many.dev:
        assert torch.equal(many.dev[name].view(torch.uint8), few.dev[name].view(torch.uint8)), name
    back = [torch.full((n, h + 1, D), 7, dtype=dtype, device="cuda") for _ in range(4)]
    kv.kv_cache_read(many.plan, many.view, many.blocks, 0, seq, slot, back[0][:, :h], back[1][:, :h])
    for s in pieces(n):
        kv.kv_cache_read(many.plan, many.view, many.blocks, 0, seq[s].contiguous(), slot[s].contiguous(), back[2][s][:, :h], back[3][s][:, :h])
    assert torch.equal(back[0], back[2]) and torch.equal(back[1], back[3])
    assert (back[0][:, h] == 7).all() and (back[0][::1001] == 7).all() and not (back[0][1:1001, :h] == 7).all(-1).any()
