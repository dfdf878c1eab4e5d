"""Some steps of a batch of requests behind one system prompt, as a serving loop would run them over a paged cache.

    python examples/batch_step.py [--layers 2] [--requests 6] [--prompt 300] [--steps 6] [--format 16|fp8|fp4]

Per step: block tables and slot maps on the GPU from the lengths of the requests (who ends gives blocks back, who begins shares the system prompt's whole blocks with the first
request).  Per layer: K (rotated) and V of all new tokens into the cache, attention of every new token over the shared prompt and its request's own tokens, with capped scores.
In the end: the next token of each request by temperature, top-k and top-p.  A request begins with a prompt of its own, all of whose tokens are new in its first step; the others
have one each.

Queries, keys, values and the logits' weights are random: what a model would compute.  Every step's attention is checked against plain attention in 32 bits.
"""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

from paper_2604_26557_amd import binding as kv

H, G, D, BLOCK = 4, 4, 128, 16   # KV heads, query heads of each, head_dim, tokens of a block
VOCABULARY, CAP = 1000, 30.0


class Cache:
    """Per layer a pool of blocks of K and V: 16-bit rows, or codes and scales."""

    def __init__(self, layers, blocks, batch, room, fmt):
        width = {"16": 2 * D, "fp8": D, "fp4": D // 2}[fmt]
        make = lambda n: [torch.zeros((blocks, H, BLOCK, n), dtype=torch.uint8, device="cuda") for _ in range(layers)]  # noqa: E731
        self.rows = {k: [t.view(torch.int16) for t in make(width)] for k in "kv"}
        self.blocks = None if fmt == "16" else kv.scale_blocks(getattr(kv, "KV_FORMAT_" + fmt.upper()), make(D // 32), make(D // 32))
        self.plan = kv.kv_layout_plan(layers, H, H * G, D, [room * BLOCK] * batch, kv.KV_BF16, 4096, 256, kv.KV_PER_SEQ)


def plain_attention(cache, view, layer, q, lens, news, shared):
    """32-bit attention over the values that the cache holds: the shared prompt's where the first request has them."""
    out, at = [], 0
    for b, (n, t) in enumerate(zip(lens, news)):
        if t <= 0:
            continue
        slot = torch.arange(n + t, dtype=torch.int32, device="cuda")
        seq = torch.where(slot < shared, 0, b).to(torch.int32)
        k, v = (torch.empty((n + t, H, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        kv.kv_cache_read(cache.plan, view, cache.blocks, layer, seq, slot, k, v)
        k, v = (x.float().repeat_interleave(G, 1).transpose(0, 1) for x in (k, v))
        s = CAP * torch.tanh((q[at:at + t].float().transpose(0, 1) @ k.transpose(1, 2).contiguous()) * (D ** -0.5 / CAP))
        later = torch.ones((t, n + t), dtype=torch.bool, device="cuda").triu(n + 1)
        out.append((s.masked_fill(later, float("-inf")).softmax(-1) @ v).transpose(0, 1))
        at += t
    return torch.cat(out)


def main(layers=2, requests=6, prompt=300, steps=6, fmt="fp8", say=print):
    gen, host = torch.Generator(device="cuda").manual_seed(1), torch.Generator().manual_seed(2)
    rand = lambda *shape: torch.randn(shape, generator=gen, device="cuda").to(torch.bfloat16)  # noqa: E731
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    f32 = lambda v: torch.tensor(v, dtype=torch.float32, device="cuda")  # noqa: E731
    pick = lambda lo, hi: int(torch.randint(lo, hi + 1, (1,), generator=host))  # noqa: E731
    B, whole, room = requests, prompt // BLOCK, (prompt + 60 + steps) // BLOCK + 2
    pool = room * B
    cache = Cache(layers, pool, B, room, fmt)
    rope = kv.Rope(kv.kv_rope_table(room * BLOCK, D, 500000.0).cuda())
    weights = torch.randn((H * G * D, VOCABULARY), generator=gen, device="cuda") * 0.1

    # The first request holds the system prompt, and stays; its first step takes it in. The others begin behind it.
    held, n_free, free, table = i32([0] * B), i32([pool]), i32(list(range(pool - 1, -1, -1))), i32([[-1] * room for _ in range(B)])
    first, seq, slot, status = i32([0] * (B + 1)), i32([-1] * (B * 60 + prompt)), i32([-1] * (B * 60 + prompt)), i32([0, 0])
    leader, shared = i32([-1] + [0] * (B - 1)), i32([0] + [whole] * (B - 1))
    lens, news = [0] * B, [prompt] + [0] * (B - 1)
    worst, drawn = 0.0, []
    for step in range(steps):
        lens_dev, news_dev, positions = i32(lens), i32(news), [n + i for n, t in zip(lens, news) for i in range(max(0, t))]
        n_tok = len(positions)
        kv.kv_step_tables(kv.step_tables(BLOCK, lens_dev, news_dev, held, free, n_free, table, first, seq, slot, status, leader, shared))
        assert status.tolist() == [0, 0]
        tok_first = first.tolist()
        # from the second step on all of them are behind the prompt's whole blocks; one that has ended has no new tokens, and nothing of it is read
        groups = kv.prefix_groups([0, B], i32([0, B]), [whole * BLOCK], i32([whole * BLOCK])) if step else None
        cached = [n if t >= 0 else whole * BLOCK for n, t in zip(lens, news)]
        view = kv.paged_view(cache.rows["k"], cache.rows["v"], table, cached, i32(cached))
        tree = kv.tree_batch(tok_first, first)
        workspace = torch.empty(kv.kv_group_attn_workspace(cache.plan, n_tok, max(lens)), dtype=torch.uint8, device="cuda")
        for layer in range(layers):
            q, k, v = rand(n_tok, H * G, D), rand(n_tok, H, D), rand(n_tok, H, D)
            out = torch.empty_like(q)
            kv.kv_rope(rope, i32(positions), q, q)
            kv.kv_cache_write(cache.plan, view, cache.blocks, layer, k, v, seq[:n_tok], slot[:n_tok], rope, i32(positions))
            kv.kv_group_attn(cache.plan, view, cache.blocks, layer, tree, q, out, kv.KV_OUT_SAME, 0, workspace, groups, kv.scores(softcap=CAP))
            want = plain_attention(cache, view, layer, q, lens, news, whole * BLOCK if groups else 0)
            worst = max(worst, float((out.float() - want).norm() / want.norm()))
        # the last new token of each request decides its next one
        last = [tok_first[b + 1] - 1 for b in range(B) if news[b] > 0]
        logits = out[last].flatten(1).float() @ weights
        n = len(last)
        tokens, probs = i32([-1] * n), torch.zeros(n, device="cuda")
        ws = torch.empty(kv.kv_sample_workspace(n, VOCABULARY), dtype=torch.uint8, device="cuda")
        kv.kv_sample(logits, torch.rand(n, generator=gen, device="cuda"), tokens, ws, temperature=f32([0.8] * n), top_k=i32([50] * n), top_p=f32([0.9] * n), probs=probs)
        assert ((tokens >= 0) & (tokens < VOCABULARY) & (probs > 0)).all()
        drawn += tokens.tolist()
        say(f"step {step}: {n_tok} new tokens of {n} requests{', behind a shared prompt' if groups else ''}; {pool - int(n_free)} of {pool} blocks held, "
            f"attention off by {worst:.1e} of its norm at most")
        # what has ended begins anew, one request ends now and then, the others go on
        for b in range(B):
            if news[b] < 0 or (step == 0 and b > 0):
                lens[b], news[b] = whole * BLOCK, pick(1, 50)
            else:
                lens[b], news[b] = lens[b] + news[b], 1
        if step % 3 == 1 and B > 1:
            news[pick(1, B - 1)] = -1
    return worst, drawn, pool - int(n_free)


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--requests", type=int, default=6)
    ap.add_argument("--prompt", type=int, default=300)
    ap.add_argument("--steps", type=int, default=6)
    ap.add_argument("--format", choices=["16", "fp8", "fp4"], default="fp8")
    a = ap.parse_args()
    main(a.layers, a.requests, a.prompt, a.steps, a.format)
