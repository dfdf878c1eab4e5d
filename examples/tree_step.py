"""A few verification steps of tree drafting over an 8-bit cache, as a serving loop would run them, then the cache's way to host memory and back.

    python examples/tree_step.py [--layers 2] [--context 600] [--steps 4] [--format fp8|fp4]

Per step and layer: rotary positions of the queries, K (rotated) and V of all drafted tokens into the cache, attention of every drafted token over the
context and its ancestors.  After the step the accepted path's rows are written once more, to the places that follow the context, and the others are
forgotten: the next step's context is that much longer.  In the end the cache is offloaded and reloaded as what it is, codes and scales, at half (fp4: a
quarter) of the bytes of 16-bit rows.

Queries, keys, values and the drafts are random: what a model and a drafter would compute.  Every step is checked against plain attention in 32 bits.
"""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

from paper_2604_26557_amd import binding as kv

H, G, D = 8, 4, 128          # KV heads, query heads of each, head_dim
DRAFTED = 12


class Cache:
    """Per layer K and V codes [1, H, S, D] (or D / 2 bytes) and scales, those of a token's heads side by side so that they offload as rows of their own."""

    def __init__(self, layers, rows, fmt):
        self.layers, self.rows = layers, rows
        width = D if fmt == kv.KV_FORMAT_FP8 else D // 2
        make = lambda *shape: torch.zeros((layers,) + shape, dtype=torch.uint8, device="cuda")  # noqa: E731
        self.codes = {k: make(1, H, rows, width) for k in "kv"}
        self.scales = {k: make(1, rows, H, D // 32) for k in "kv"}
        self.length = 0
        self.length_dev = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.plan = kv.kv_layout_plan(layers, H, H * G, D, [rows], kv.KV_BF16, 4096, 256, kv.KV_PER_SEQ)
        # what moves: rows of width / 2 16-bit elements per head, and one row of H * D / 64 for a token's scales
        self.moved = [(kv.kv_layout_plan(layers, H, H, width // 2, [rows], kv.KV_BF16, 4096, 256, kv.KV_PER_SEQ), self.codes),
                      (kv.kv_layout_plan(layers, 1, 1, H * D // 64, [rows], kv.KV_BF16, 4096, 256, kv.KV_PER_SEQ), self.scales)]
        self.blocks = kv.scale_blocks(fmt, *([s.transpose(1, 2) for s in self.scales[k]] for k in "kv"))

    def view(self):
        self.length_dev.fill_(self.length)
        return kv.bhsd_view([c.view(torch.int16) for c in self.codes["k"]], [c.view(torch.int16) for c in self.codes["v"]], [self.length], self.length_dev)

    def offload_and_reload(self):
        """Every byte of the cache to host memory, the device copy wiped, and back."""
        moved = 0
        for plan, tensors in self.moved:
            # codes are [1, H, rows, .], a token's scales one head of a row
            bufs = [[t.view(torch.int16) if tensors is self.codes else t.flatten(2).view(torch.int16)[:, None] for t in tensors[k]] for k in "kv"]
            view = kv.bhsd_view(*bufs, [self.rows], torch.tensor([self.rows], dtype=torch.int32, device="cuda"))
            region = torch.empty(int(plan.info.region_bytes_needed), dtype=torch.uint8, pin_memory=True)
            kv.kv_pipeline_run(plan, kv.KV_DIR_OFFLOAD, 0, self.layers, view, region)
            before = [tensors[k].clone() for k in "kv"]
            for k in "kv":
                tensors[k].zero_()
            stats = kv.kv_pipeline_run(plan, kv.KV_DIR_RELOAD, 0, self.layers, view, region)
            assert all(torch.equal(tensors[k], b) for k, b in zip("kv", before)), "reloaded bytes differ"
            moved += stats.bytes_direct
        return moved


def plain_attention(cache, view, layer, q, parents):
    """32-bit attention over the values that the cache holds."""
    n, ctx = len(parents), cache.length
    seq = torch.zeros(ctx + n, dtype=torch.int32, device="cuda")
    slot = torch.arange(ctx + n, dtype=torch.int32, device="cuda")
    k, v = (torch.empty((ctx + n, H, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    kv.kv_cache_read(cache.plan, view, cache.blocks, layer, seq, slot, k, v)
    sees = torch.zeros((n, ctx + n), dtype=torch.bool)
    sees[:, :ctx] = True
    for i, p in enumerate(parents):
        if p >= 0:
            sees[i] |= sees[p]
        sees[i, ctx + i] = True
    k, v = (x.float().repeat_interleave(G, 1).transpose(0, 1) for x in (k, v))
    s = (q.float().transpose(0, 1) @ k.transpose(1, 2).contiguous()) * D ** -0.5
    return (s.masked_fill(~sees.cuda(), float("-inf")).softmax(-1) @ v).transpose(0, 1)


def main(layers=2, context=600, steps=4, fmt="fp8", say=print):
    fmt = {"fp8": kv.KV_FORMAT_FP8, "fp4": kv.KV_FORMAT_FP4}[fmt]
    gen = torch.Generator(device="cuda").manual_seed(1)
    rand = lambda *shape: torch.randn(shape, generator=gen, device="cuda").to(torch.bfloat16)  # noqa: E731
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    rows = (context + steps * DRAFTED + 255) // 256 * 256
    cache = Cache(layers, rows, fmt)
    # trained on 4096 positions, stretched to four times as many
    rope = kv.Rope(kv.kv_rope_table(rows, D, 500000.0, kv.KV_ROPE_WAVELENGTH, 4.0, 4096).cuda())

    # prefill: the context's rows
    places = torch.arange(context, dtype=torch.int32, device="cuda")
    for layer in range(layers):
        kv.kv_cache_write(cache.plan, cache.view(), cache.blocks, layer, rand(context, H, D), rand(context, H, D), i32([0] * context), places, rope, places)
    cache.length = context

    worst = 0.0
    workspace = torch.empty(kv.kv_tree_attn_workspace(cache.plan, DRAFTED, rows), dtype=torch.uint8, device="cuda")
    for step in range(steps):
        view = cache.view()
        parents = [-1, -1, 0, 0, 1, 2, 2, 3, 5, 5, 6, 8][:DRAFTED]
        masks, depths = kv.kv_tree_masks(parents)
        tree = kv.tree_batch([0, DRAFTED], i32([0, DRAFTED]), masks.cuda())
        seq, slots = i32([0] * DRAFTED), i32([cache.length + i for i in range(DRAFTED)])
        pos = depths.cuda() + cache.length
        accepted = [0, 2, 5][: 1 + step % 3]                       # a path from the root
        # the accepted rows move up to the context's end, the others have no place
        keep = i32([cache.length + accepted.index(i) if i in accepted else -1 for i in range(DRAFTED)])
        for layer in range(layers):
            q, k, v = rand(DRAFTED, H * G, D), rand(DRAFTED, H, D), rand(DRAFTED, H, D)
            out = torch.empty_like(q)
            kv.kv_rope(rope, pos, q, q)
            kv.kv_cache_write(cache.plan, view, cache.blocks, layer, k, v, seq, slots, rope, pos)
            kv.kv_tree_attn(cache.plan, view, cache.blocks, layer, tree, q, out, kv.KV_OUT_SAME, 0, workspace)
            want = plain_attention(cache, view, layer, q, parents)
            worst = max(worst, float((out.float() - want).norm() / want.norm()))
            kv.kv_cache_write(cache.plan, view, cache.blocks, layer, k, v, seq, keep, rope, pos)
        cache.length += len(accepted)
        say(f"step {step}: {DRAFTED} drafted, {len(accepted)} accepted, context {cache.length}, attention off by {worst:.1e} of its norm at most")
    moved = cache.offload_and_reload()
    full = layers * 2 * rows * H * D * 2
    say(f"offloaded and reloaded {moved} bytes; 16-bit rows would have been {full}")
    return worst, moved, full


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--context", type=int, default=600)
    ap.add_argument("--steps", type=int, default=4)
    ap.add_argument("--format", choices=["fp8", "fp4"], default="fp8")
    a = ap.parse_args()
    main(a.layers, a.context, a.steps, a.format)
