"""Operators of a serving step for a batch of requests: block tables and slot maps from request lengths, attention over prefixes that sequences
share and with capped, biased or bounded scores (single tokens, drafted tokens, prompts), and sampling.

A case is a dict of plain values.  `kind` says what one pass does:
  tables  the block tables of a step grown from a stack of free blocks, what has ended released, and the maps of the new tokens' places
  attn    attention of new tokens over the cache, the prefix of each group of sequences held once (in its first sequence's place)
  sample  the next token of every row of logits
  step    tables, the new rows of K and V written, attention, sampling

Scores x = q . K * scale become cap * tanh(x / cap), less slope[head] * |distance|.  New token t of a sequence sees token j where j >= from[t] and j is of
the context, one that the token's tree or chain has, or j < to[t].
A cache row of 8 or 4 bits is codes (e4m3; e2m1, two to a byte, the lower half first) and a power of two for every 32 of them (its exponent + 127).
Lengths, trees, tables and everything else that fixes the amount of work come from the case; values from the seed.
"""
import math
import random

import torch

own = False
BLOCK = 32
FP4 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def _attn(B, H, G, D, lo, hi, tlo, thi, dtype, layout, fmt, **more):
    """B sequences of lo..hi cached tokens of their own and tlo..thi new ones each, H KV heads with G query heads each; `groups` of them share
    plo..phi cached tokens (0: nobody shares)."""
    c = {"kind": "attn", "B": B, "H": H, "G": G, "D": D, "lo": lo, "hi": hi, "tlo": tlo, "thi": thi, "dtype": dtype, "layout": layout, "fmt": fmt,
         "bt": 16, "out": "same", "tree": False, "groups": 0, "plo": 0, "phi": 0, "cap": 0.0, "slopes": False, "window": 0, "docs": 0, "both": 0, "shape_seed": 5}
    c.update(more)
    return c


def _tables(B, lo, hi, tlo, thi, **more):
    c = {"kind": "tables", "B": B, "lo": lo, "hi": hi, "tlo": tlo, "thi": thi, "bt": 16, "ended": 0.1, "begun": 0.2, "prefix": 512, "shape_seed": 5}
    c.update(more)
    return c


def _sample(B, V, dtype, **more):
    c = {"kind": "sample", "B": B, "V": V, "dtype": dtype, "k": 0, "p": 1.0, "min_p": 0.0, "t": 1.0, "spread": 2.5, "greedy": 0.0}
    c.update(more)
    return c


def listed():
    return [
        # a decode step's bookkeeping: 64 requests, a token each, some ended, some just begun behind a shared prompt
        _tables(64, 1000, 8000, 1, 1, name="tables_decode"),
        # a step that takes in chunks of many prompts, blocks of 32 tokens
        _tables(384, 1, 16000, 1, 768, bt=32, begun=0.6, name="tables_chunks"),
        # decoding, a token at a time, 32 requests behind one system prompt of 8K, 8B shape, paged
        _attn(32, 8, 4, 128, 100, 2000, 1, 1, "f16", "paged", "16", groups=1, plo=8192, phi=8192, name="shared_decode"),
        # drafted trees of 16 requests over a shared 16K document in an 8-bit cache
        _attn(16, 8, 4, 128, 50, 1000, 5, 13, "bf16", "paged", "fp8", tree=True, groups=1, plo=16384, phi=16384, name="shared_trees_fp8"),
        # four prompts of odd lengths, shared by six requests each, 4 bits, seven query heads to a KV head, 32-bit results
        _attn(24, 4, 7, 128, 1, 700, 1, 1, "bf16", "bhsd", "fp4", groups=4, plo=1000, phi=5000, out="f32", name="shared_groups_fp4"),
        # one request at 8K: capped scores and a window of 4K over wide heads, the smallest attention call
        _attn(1, 16, 1, 256, 8192, 8192, 1, 1, "bf16", "bhsd", "16", cap=50.0, window=4096, name="capped_window_decode"),
        # a prompt of 4K from the start, 8B shape, capped scores: the most arithmetic
        _attn(1, 8, 4, 128, 0, 0, 4096, 4096, "bf16", "bhsd", "16", cap=30.0, name="capped_prompt"),
        # chunks of packed documents behind some context: biased by distance, each document's first tokens see each other both ways
        _attn(2, 12, 1, 64, 300, 900, 1501, 2300, "f16", "paged", "16", slopes=True, docs=5, both=64, name="biased_documents"),
        # one request's next token, a vocabulary of 32000, 32-bit logits: latency
        _sample(1, 32000, "f32", k=50, p=0.9, name="sample_one"),
        # a batch's next tokens from 16-bit logits, which tie often: top-p and min-p over a vocabulary of 128256
        _sample(64, 128256, "bf16", p=0.95, min_p=0.02, t=0.8, greedy=0.1, name="sample_batch"),
        # many rows with nothing cut off, flat, a vocabulary of an odd size: long sums
        _sample(256, 50257, "f32", t=1.3, spread=1.0, name="sample_flat"),
        # everything together: a decode step of 48 requests behind two prompts, with a window
        _attn(48, 8, 4, 128, 60, 1500, 1, 1, "bf16", "paged", "16", groups=2, plo=2048, phi=6000, cap=30.0, V=32000, k=40, p=0.95, min_p=0.0, t=0.9,
              spread=2.5, greedy=0.0, ended=0.0, begun=0.0, prefix=0, kind="step", name="step_shared_decode"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attn"] * 6 + ["tables"] * 2 + ["sample"] * 3 + ["step"])
    seed = rng.randrange(1 << 30)
    if kind == "tables":
        hi, thi = _log_int(rng, 16, 16000), _log_int(rng, 1, 768)
        return _tables(_log_int(rng, 1, 384), rng.randint(1, hi), hi, rng.randint(1, thi), thi, bt=rng.choice([8, 16, 16, 32, 64]), ended=rng.choice([0.0, 0.1, 0.3]),
                       begun=rng.choice([0.0, 0.2, 0.7]), prefix=rng.choice([0, 100, 512]), shape_seed=seed)
    cut = {"k": rng.choice([0, 0, 1, 20, 50, 1000]), "p": rng.choice([1.0, 1.0, 0.5, 0.9, 0.95]), "min_p": rng.choice([0.0, 0.0, 0.02, 0.1]),
           "t": rng.choice([0.5, 0.8, 1.0, 1.3]), "spread": rng.choice([1.0, 2.5, 5.0]), "greedy": rng.choice([0.0, 0.0, 0.2])}
    if kind == "sample":
        B, V = _log_int(rng, 1, 256), _log_int(rng, 1000, 160000)
        return _sample(min(B, 2 ** 24 // V), V, rng.choice(["f32", "f16", "bf16"]), **cut)
    D = rng.choice([64, 128, 128, 256])
    H = rng.choice([1, 2, 3, 4, 5, 8, 8, 16])
    G = rng.choice([1, 1, 2, 3, 4, 4, 5, 6, 7, 8])
    B = _log_int(rng, 1, 48)
    groups = rng.choice([0, 1, 1, 2, 4]) if B > 1 else 0
    groups = min(groups, B)
    phi = _log_int(rng, 100, 16384) if groups else 0
    plo = rng.choice([phi, rng.randint(phi // 4, phi)])
    hi = _log_int(rng, 1, 2000) if groups else _log_int(rng, 1, 16384)
    lo = rng.randint(hi // 8, hi)
    what = rng.choice(["single", "drafted", "prompt"]) if kind == "attn" else "single"
    thi = 1 if what == "single" else _log_int(rng, 2, 64) if what == "drafted" else _log_int(rng, 65, 4096)
    tlo = rng.randint(max(1, thi // 2), thi)
    layout = "paged" if kind == "step" else rng.choice(["bhsd", "paged"])
    more = {"groups": groups, "plo": plo, "phi": phi, "tree": what == "drafted" and rng.random() < 0.5, "out": rng.choice(["f32", "same", "same"]), "shape_seed": seed,
            "cap": rng.choice([0.0, 30.0, 50.0]), "slopes": rng.random() < 0.3, "window": rng.choice([0, 0, 0, 500, 4096])}
    if what == "prompt" and not groups and rng.random() < 0.5:
        more.update(docs=rng.randint(1, 6), both=rng.choice([0, 1, 64]))
    if not (groups or more["cap"] or more["slopes"] or more["window"] or what == "prompt"):
        more["cap"] = 30.0
    if layout == "paged":
        more["bt"] = rng.choice([16, 16, 16, 32, 64])
    # no more than the largest listed cases: so many products, and cached values
    while B * thi * (phi + hi + thi) * H * G * D > 2 ** 36 or B * (phi + hi + thi) * H * D > 2 ** 27:
        if B > max(1, groups) and rng.random() < 0.6:
            B = max(groups, 1, B // 2)
        elif thi > 1 and rng.random() < 0.6:
            thi = max(1, thi // 2)
            tlo = min(tlo, thi)
        else:
            hi, lo, phi, plo = (max(1, hi // 2), lo // 2, phi // 2, plo // 2)
    if kind == "step":
        return _attn(B, H, G, D, lo, hi, 1, 1, rng.choice(["f16", "bf16"]), layout, "16", V=_log_int(rng, 1000, 64000), ended=0.0, begun=0.0, prefix=0, **dict(more, kind="step", **cut))
    return _attn(B, H, G, D, lo, hi, tlo, thi, rng.choice(["f16", "bf16"]), layout, rng.choice(["16", "16", "fp8", "fp4"]), **more)


# ------------------------------------------------------------------------------------------ what the case fixes
def _shapes(c):
    """Of a batch that attends: context lengths, numbers of new tokens, each new token's parent, groups' first sequences and shared tokens."""
    r = random.Random(c["shape_seed"])
    n = c["groups"]
    first = [c["B"] * g // n for g in range(n + 1)] if n else []
    shared = [r.randint(c["plo"], c["phi"]) for _ in range(n)]
    of = [next((shared[g] for g in range(n) if first[g] <= b < first[g + 1]), 0) for b in range(c["B"])]
    lens = [of[b] + r.randint(c["lo"], c["hi"]) for b in range(c["B"])]
    news = [r.randint(c["tlo"], c["thi"]) for _ in range(c["B"])]
    # drafters extend recent tokens most of the time; without a tree every token follows the one before it
    parents = [[max(-1, i - 1 - (int(r.expovariate(0.3)) if c["tree"] else 0)) for i in range(k)] for k in news]
    return lens, news, parents, first, shared


def _depths(parents):
    d = []
    for up in parents:
        d.append(d[up] + 1 if up >= 0 else 0)
    return d


def _bounds(c, lens, news, parents):
    """(from, to) of every new token, in the numbering of its sequence's tokens."""
    r = random.Random(c["shape_seed"] + 1)
    lo, up = [], []
    for n, t, p in zip(lens, news, parents):
        starts = sorted(r.sample(range(1, t), min(c["docs"] - 1, t - 1))) if c["docs"] > 1 and t > 1 else []
        start, ends = (r.randint(0, n) if c["docs"] else 0), [n + x for x in starts] + [n + t]
        for i, depth in enumerate(_depths(p)):
            if i in starts:
                start = n + i
            end = next(e for e in ends if e > n + i)
            lo.append(max(start, n + depth - c["window"] + 1) if c["window"] else start)
            up.append(min(max(start, n if not c["docs"] else start) + c["both"], end) if c["both"] else 0)
    return lo, up


def _masks(parents, words):
    """A bit for every new token that each one sees: its ancestors and itself."""
    masks = []
    for p in parents:
        bits = []
        for i, up in enumerate(p):
            bits.append((bits[up] if up >= 0 else 0) | 1 << i)
        for b in bits:
            w = [b >> 64 * k & (1 << 64) - 1 for k in range(words)]
            masks.append([x - (1 << 64) if x >> 63 else x for x in w])
    return torch.tensor(masks, dtype=torch.int64)


def _requests(c):
    """Of a step's tables: lengths, new tokens (-1: ended), leader and shared blocks, held blocks, row length and size of the pool."""
    if c["kind"] == "step":
        lens, news, _, first, shared = _shapes(c)
        B, bt = c["B"], c["bt"]
        leader, common = [-1] * B, [0] * B
        for g, n in enumerate(shared):
            for b in range(first[g] + 1, first[g + 1]):
                leader[b], common[b] = first[g], n // bt
        held = [-(-n // bt) for n in lens]
    else:
        r = random.Random(c["shape_seed"])
        B, bt = c["B"], c["bt"]
        lens, news, leader, common, held = [], [], [], [], []
        for b in range(B):
            n, t = r.randint(c["lo"], c["hi"]), r.randint(c["tlo"], c["thi"])
            x = r.random()
            follows = b > 0 and c["prefix"] >= bt and r.random() < 0.6
            if b == 0:
                n = max(n, c["prefix"])
            common.append(c["prefix"] // bt if follows else 0)
            leader.append(0 if follows else -1)
            if b > 0 and x < c["ended"]:
                t, h = -1, -(-n // bt)
            elif b > 0 and x < c["ended"] + c["begun"]:  # what it shares is there before its first step
                n, h = common[-1] * bt, 0
            else:
                h = -(-n // bt) + (r.random() < 0.1)  # a block more, of drafted tokens that were not accepted
            n = max(n, common[-1] * bt) if h else n
            lens.append(n)
            news.append(t)
            held.append(max(h, common[-1]) if h else 0)
    need = [max(h, -(-(n + t) // bt)) if t >= 0 else h for n, t, h in zip(lens, news, held)]
    room = max(need) + 3
    pool = sum(need) + 5
    return lens, news, leader, common, held, room, pool


# ------------------------------------------------------------------------------------------ inputs
def _dev(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _rows(shape, gen, outlying=False):
    """N(0, 1), a channel in 16 of K three times as wide."""
    x = torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)
    if outlying:
        x[..., 5::16] *= 3
    return x


def _put_tables(s, c, seed):
    """The stack of free blocks and the rows as the step before left them; which block is which comes from the seed."""
    lens, news, leader, common, held, room, pool = _requests(c)
    ids = list(range(pool))
    random.Random(seed).shuffle(ids)
    rows, at = [], 0
    for b, h in enumerate(held):
        shared = rows[leader[b]][:common[b]] if h and leader[b] >= 0 else []
        take = max(0, h - len(shared))
        rows.append(shared + ids[at:at + take] + [-1] * (room - len(shared) - take))
        at += take
    s["free"] = _dev(ids[at:] + [0] * at)
    s["n_free"], s["held"], s["table"] = _dev([pool - at]), _dev(held), _dev(rows)
    s["seq_lens"], s["new_lens"], s["leader"], s["common"] = _dev(lens), _dev(news), _dev(leader), _dev(common)
    s["n_tok"] = sum(max(0, t) for t in news)
    for name, like in (("n_free", s["n_free"]), ("held", s["held"]), ("table", s["table"]), ("tok_first", _dev([0] * (c["B"] + 1))), ("tok_seq", _dev([0] * s["n_tok"])),
                       ("tok_slot", _dev([0] * s["n_tok"])), ("status", _dev([0, 0]))):
        s[name + "_out"] = torch.zeros_like(like)
    return pool


def _put_logits(s, c, gen):
    """Normal, a few far ahead of the rest, one in 50 excluded."""
    B, V = c["B"], c["V"]
    x = torch.randn((B, V), generator=gen, device="cuda") * c["spread"]
    ahead = torch.randint(0, V, (B, 8), generator=gen, device="cuda")
    x.scatter_add_(1, ahead, torch.rand((B, 8), generator=gen, device="cuda") * 2.5 * c["spread"])
    x[torch.rand((B, V), generator=gen, device="cuda") < 0.02] = -torch.inf
    s["logits"] = x.to(DTYPES[c["dtype"]])
    some = torch.rand((B,), generator=gen, device="cuda")
    s["temperature"] = torch.where(some < c["greedy"], 0.0, c["t"] * (0.9 + 0.2 * some))
    s["top_k"] = torch.full((B,), c["k"], dtype=torch.int32, device="cuda")
    s["top_p"], s["min_p"] = (torch.full((B,), c[k], dtype=torch.float32, device="cuda") for k in ("p", "min_p"))
    s["u"] = torch.rand((B,), generator=gen, device="cuda")
    s["tokens"], s["probs"] = torch.zeros((B,), dtype=torch.int32, device="cuda"), torch.zeros((B,), device="cuda")


def _put_cache(s, c, gen, pool):
    """K and V (and their scales) of every token.  A shared prefix lies in its group's first sequence; the others' places of it hold nothing."""
    B, H, D, bt = c["B"], c["H"], c["D"], c["bt"]
    shape = (pool, H, bt) if c["layout"] == "paged" else (B, H, s["total"])
    for kind in ("k", "v"):
        width = D // 2 if c["fmt"] == "fp4" else D
        s[kind] = torch.zeros(shape + (width,), dtype=DTYPES[c["dtype"]] if c["fmt"] == "16" else torch.uint8, device="cuda")
        if c["fmt"] != "16":
            s[kind + "_scale"] = torch.zeros(shape + (D // BLOCK,), dtype=torch.uint8, device="cuda")
        some = max(1, 2 ** 24 // (H * shape[2] * D))
        for i in range(0, shape[0], some):
            part = s[kind][i:i + some]
            x = _rows(part.shape[:-1] + (D,), gen, kind == "k")
            if c["fmt"] == "16":
                part.copy_(x)
                continue
            x = x.unflatten(-1, (-1, BLOCK))
            e = torch.frexp(x.abs().amax(-1))[1] - (8 if c["fmt"] == "fp8" else 2)
            s[kind + "_scale"][i:i + some] = (e + 127).to(torch.uint8)
            y = torch.ldexp(x, -e[..., None]).flatten(-2)
            if c["fmt"] == "fp8":
                part.copy_(y.to(torch.float8_e4m3fn).view(torch.uint8))
            else:
                near = torch.bucketize(y.abs(), torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device="cuda")).to(torch.uint8) | torch.signbit(y).to(torch.uint8) << 3
                part.copy_(near[..., 0::2] | near[..., 1::2] << 4)


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = {"case": c}
    if c["kind"] in ("tables", "step"):
        pool = _put_tables(s, c, seed)
    if c["kind"] in ("attn", "step"):
        B, H, D, bt = c["B"], c["H"], c["D"], c["bt"]
        lens, news, parents, first, shared = _shapes(c)
        s["lens"], s["news"], s["total"] = lens, news, max(a + b for a, b in zip(lens, news))
        s["first"] = [sum(news[:b]) for b in range(B + 1)]
        s["first_dev"], s["lens_dev"], s["news_dev"] = _dev(s["first"]), _dev(lens), _dev(news)
        s["seq"] = _dev([b for b in range(B) for _ in range(news[b])])
        s["groups"] = (first, shared)
        s["prefix"] = _dev([next((shared[g] for g in range(len(shared)) if first[g] <= b < first[g + 1]), 0) for b in range(B)])
        s["leads"] = _dev([next((first[g] for g in range(len(shared)) if first[g] <= b < first[g + 1]), b) for b in range(B)])
        s["mask"] = _masks(parents, (max(news) + 63) // 64).cuda() if c["tree"] else None
        s["pos"] = _dev([lens[b] + d for b in range(B) for d in _depths(parents[b])])
        lo, up = _bounds(c, lens, news, parents)
        s["from"] = _dev(lo) if c["window"] or c["docs"] else None
        s["to"] = _dev(up) if c["both"] else None
        s["slope"] = 2.0 ** (-8.0 * torch.arange(1, H * c["G"] + 1, device="cuda") / (H * c["G"])) if c["slopes"] else None
        if c["layout"] == "paged" and c["kind"] == "attn":
            rows, pool = [], 0
            for b in range(B):  # a prefix's whole blocks are in its first sequence's row alone
                skip = int(s["prefix"][b]) // bt if int(s["leads"][b]) != b else 0
                n = -(-(lens[b] + news[b]) // bt)
                rows.append([-1] * skip + list(range(pool, pool + n - skip)))
                pool += n - skip
            ids = list(range(pool))
            random.Random(c["shape_seed"] + 2).shuffle(ids)
            room = max(map(len, rows))
            s["table_blocks"] = _dev([[ids[i] if i >= 0 else -1 for i in r] + [-1] * (room - len(r)) for r in rows])
        _put_cache(s, c, gen, pool if c["layout"] == "paged" else 0)
        n = s["first"][-1]
        s["q"] = _rows((n, H * c["G"], D), gen).to(DTYPES[c["dtype"]])
        s["out"] = torch.zeros((n, H * c["G"], D), dtype=torch.float32 if c["out"] == "f32" else DTYPES[c["dtype"]], device="cuda")
    if c["kind"] == "step":
        s["k_new"], s["v_new"] = _rows((n, H, D), gen, True).to(DTYPES[c["dtype"]]), _rows((n, H, D), gen).to(DTYPES[c["dtype"]])
        s["table_blocks"] = s["table_out"]
    if c["kind"] in ("sample", "step"):
        _put_logits(s, c, gen)
    if own:
        _handles(s, c)
    return s


def _handles(s, c):
    """The plan, views, workspaces and descriptions that a program which serves from this cache keeps."""
    from paper_2604_26557_amd import binding as kv
    s["kv"] = kv
    if c["kind"] in ("tables", "step"):
        s["tables"] = kv.step_tables(c["bt"], s["seq_lens"], s["new_lens"], s["held"], s["free"], s["n_free"], s["table"], s["tok_first_out"], s["tok_seq_out"], s["tok_slot_out"],
                                     s["status_out"], leader=s["leader"], shared=s["common"], held_out=s["held_out"], n_free_out=s["n_free_out"], block_table_out=s["table_out"])
    if c["kind"] in ("sample", "step"):
        s["sample_ws"] = torch.empty(kv.kv_sample_workspace(c["B"], c["V"]), dtype=torch.uint8, device="cuda")
    if c["kind"] not in ("attn", "step"):
        return
    B, H, D = c["B"], c["H"], c["D"]
    s["plan"] = kv.kv_layout_plan(1, H, H * c["G"], D, [s["total"]] * B, kv.KV_F16 if c["dtype"] == "f16" else kv.KV_BF16, 512, 4096, kv.KV_PER_SEQ)
    k, v = [s["k"].view(torch.int16)], [s["v"].view(torch.int16)]
    s["view"] = kv.paged_view(k, v, s["table_blocks"], s["lens"], s["lens_dev"]) if c["layout"] == "paged" else kv.bhsd_view(k, v, s["lens"], s["lens_dev"])
    s["blocks"] = None
    if c["fmt"] != "16":
        s["blocks"] = kv.scale_blocks(kv.KV_FORMAT_FP8 if c["fmt"] == "fp8" else kv.KV_FORMAT_FP4, [s["k_scale"]], [s["v_scale"]])
    s["tree"] = kv.tree_batch(s["first"], s["first_dev"], s["mask"])
    first, shared = s["groups"]
    s["shared"] = kv.prefix_groups(first, _dev(first), shared, _dev(shared)) if shared else None
    s["scores"] = None
    if c["cap"] or c["slopes"] or s["from"] is not None or s["to"] is not None:
        s["scores"] = kv.scores(softcap=c["cap"], slopes=s["slope"], positions=s["pos"] if c["slopes"] else None, sees_from=s["from"], sees_to=s["to"])
    s["ws"] = torch.empty(kv.kv_group_attn_workspace(s["plan"], s["first"][-1], s["total"]), dtype=torch.uint8, device="cuda")


# ------------------------------------------------------------------------------------------ plain forms
def _plain_tables(s, c):
    bt, lens, news, held, table = c["bt"], s["seq_lens"].long(), s["new_lens"].long(), s["held"].long(), s["table"]
    B, room = table.shape
    ended = news < 0
    need = torch.where(ended, 0, (lens + news.clamp(min=0) + bt - 1) // bt)
    common = torch.where(s["leader"] >= 0, s["common"], 0).long()
    entry = torch.arange(room, device="cuda")
    # what ends goes onto the stack, in order of sequences and entries
    gone = ended[:, None] & (entry >= common[:, None]) & (entry < held[:, None])
    n_free, n_gone = s["n_free"].long(), gone.sum()
    place = torch.where(gone, n_free + gone.flatten().cumsum(0).reshape(B, room) - 1, s["free"].numel())
    free = torch.cat([s["free"], torch.zeros(1, dtype=torch.int32, device="cuda")]).scatter(0, place.flatten(), table.flatten())[:-1]
    s["free"].copy_(free)
    # what is needed comes from its top
    fresh = (entry >= torch.maximum(held, common)[:, None]) & (entry < need[:, None])
    n_fresh, top = fresh.sum(), n_free + n_gone
    short = (n_fresh - top).clamp(min=0)
    over = (need > room).sum()
    fine = (short == 0) & (over == 0)
    at = (top - fresh.flatten().cumsum(0).reshape(B, room)).clamp(0, s["free"].numel() - 1)
    rows = torch.where(ended[:, None], -1, torch.where(fine & fresh, free[at], table))
    follows = (entry >= held[:, None]) & (entry < torch.minimum(common, need)[:, None])
    rows = torch.where(fine & follows, rows[s["leader"].clamp(min=0).long()], rows)
    s["table_out"].copy_(rows)
    s["held_out"].copy_(torch.where(ended, 0, torch.where(fine, torch.maximum(held, need), held)))
    s["n_free_out"].copy_(top - torch.where(fine, n_fresh, 0))
    s["status_out"].copy_(torch.cat([short, over.reshape(1)]))
    end = news.clamp(min=0).cumsum(0)
    s["tok_first_out"][1:] = end
    t = torch.arange(s["n_tok"], device="cuda")
    seq = torch.searchsorted(end, t, right=True)
    s["tok_seq_out"].copy_(seq)
    s["tok_slot_out"].copy_(lens[seq] + t - s["tok_first_out"].long()[seq])
    return [s[k + "_out"] for k in ("table", "held", "n_free", "status", "tok_first", "tok_seq", "tok_slot")] + [s["free"]]


def _values(codes, scale, fmt):
    """Rows in 32 bits."""
    if fmt == "16":
        return codes.float()
    if fmt == "fp8":
        x = codes.view(torch.float8_e4m3fn).float()
    else:
        t = torch.tensor(FP4 + tuple(-v for v in FP4), device=codes.device)
        x = t[torch.stack([codes & 15, codes >> 4], -1).flatten(-2).int()]
    return torch.ldexp(x.unflatten(-1, (-1, BLOCK)), scale.int()[..., None] - 127).flatten(-2)


def _dense(s, c, kind):
    """[B, H, total, D] in 32 bits, the shared tokens from their first sequence."""
    def laid(x):
        if c["layout"] == "paged":
            x = x[s["table_blocks"].clamp(min=0).long()].transpose(1, 2).flatten(2, 3)[:, :, :s["total"]]
        return x
    x = _values(laid(s[kind]), laid(s[kind + "_scale"]) if c["fmt"] != "16" else None, c["fmt"])
    if c["groups"]:
        n = int(max(s["groups"][1]))
        common = torch.arange(n, device="cuda") < s["prefix"][:, None]
        x[:, :, :n] = torch.where(common[:, None, :, None], x[s["leads"].long(), :, :n], x[:, :, :n])
    return x


def _seen(s, c):
    """[B, T, S]: which tokens each new token sees; its row in the batch; positions of queries [B, T] and keys [B, S]."""
    B, T, S = c["B"], max(s["news"]), s["total"]
    seq, n = s["seq"].long(), s["seq"].numel()
    at = torch.arange(n, device="cuda") - s["first_dev"].long()[seq]
    j = torch.arange(S, device="cuda")
    rel = j - s["lens_dev"].long()[:, None]

    def by_row(x, fill):
        return torch.full((B, T), fill, dtype=torch.int64, device="cuda").index_put((seq, at), x.long())
    if s["mask"] is None:
        has = (torch.arange(T, device="cuda")[:, None] >= rel[:, None])
    else:
        flat = ((s["mask"][:, :, None] >> torch.arange(64, device="cuda")) & 1).bool().flatten(1)
        bits = torch.zeros((B, T, flat.shape[1]), dtype=torch.bool, device="cuda").index_put((seq, at), flat)
        has = bits.gather(2, rel.clamp(0, flat.shape[1] - 1)[:, None].expand(B, T, S))
    sees = (rel < 0)[:, None] | has
    if s["to"] is not None:
        sees = sees | (j < by_row(s["to"], 0)[:, :, None])
    if s["from"] is not None:
        sees = sees & (j >= by_row(s["from"], 0)[:, :, None])
    sees = sees & (rel < s["news_dev"].long()[:, None])[:, None]
    where = by_row(s["pos"], 0)
    keys = torch.where(rel < 0, j, where.gather(1, rel.clamp(0, T - 1)))
    return sees, seq, at, where, keys


def _attend(s, c):
    B, H, G, D, T = c["B"], c["H"], c["G"], c["D"], max(s["news"])
    sees, seq, at, where, keys = _seen(s, c)
    rows = torch.zeros((B, T, H * G, D), device="cuda").index_put((seq, at), s["q"].float())
    rows = rows.unflatten(2, (H, G)).permute(0, 2, 3, 1, 4).reshape(B * H, G * T, D)
    x = torch.bmm(rows, _dense(s, c, "k").flatten(0, 1).transpose(1, 2).contiguous()).view(B, H, G, T, -1)
    x *= D ** -0.5
    if c["cap"]:
        x = c["cap"] * torch.tanh(x / c["cap"])
    if c["slopes"]:
        x -= s["slope"].view(1, H, G, 1, 1) * (where[:, :, None] - keys[:, None]).abs().float()[:, None, None]
    x.masked_fill_(~sees[:, None, None], -torch.inf)
    top = x.amax(-1, keepdim=True)
    p = (x - torch.where(top == -torch.inf, 0.0, top)).exp()
    total = p.sum(-1, keepdim=True)
    out = torch.bmm(p.view(B * H, G * T, -1), _dense(s, c, "v").flatten(0, 1)).view(B, H, G, T, D) / torch.where(total == 0, 1.0, total)
    out = out.permute(0, 3, 1, 2, 4).reshape(B, T, H * G, D)[seq, at]
    return out if c["out"] == "f32" else out.to(DTYPES[c["dtype"]])


def _plain_sample(s, c):
    x, order = s["logits"].float().sort(dim=1, descending=True, stable=True)
    B, V = x.shape
    t = s["temperature"].double()[:, None]
    w = ((x.double() - x[:, :1].double()) / torch.where(t == 0, 1.0, t)).exp()
    k = torch.where(s["top_k"] <= 0, V, s["top_k"].clamp(max=V)).long()[:, None]
    k = torch.where(t == 0, 1, k)
    sums = w.cumsum(1)
    enough = (sums < s["top_p"].double()[:, None] * sums.gather(1, k - 1)).sum(1, keepdim=True) + 1
    keep = torch.minimum(k, torch.where(s["top_p"][:, None] >= 1, V, enough))
    keep = torch.minimum(keep, (w >= s["min_p"].double()[:, None]).sum(1, keepdim=True))
    w = torch.where(torch.arange(V, device="cuda") < keep, w, 0.0)
    w = torch.zeros_like(w).scatter(1, order, w)
    sums = w.cumsum(1)
    last = V - 1 - (w > 0).flip(1).int().argmax(1, keepdim=True)
    token = torch.minimum((sums <= s["u"].double()[:, None] * sums[:, -1:]).sum(1, keepdim=True), last)
    return [token[:, 0].int(), (w.gather(1, token) / sums[:, -1:])[:, 0].float()]


def _plain(s, c):
    if c["kind"] == "tables":
        return _plain_tables(s, c)
    if c["kind"] == "sample":
        return _plain_sample(s, c)
    if c["kind"] == "attn":
        return _attend(s, c)
    got = _plain_tables(s, c)
    seq, slot = s["tok_seq_out"].long(), s["tok_slot_out"].long()
    block, row = s["table_out"][seq, slot // c["bt"]].long(), slot % c["bt"]
    s["k"][block, :, row], s["v"][block, :, row] = s["k_new"], s["v_new"]
    return got + [_attend(s, c)] + _plain_sample(s, c)


# ------------------------------------------------------------------------------------------ one pass
def _sampled(s, c):
    s["kv"].kv_sample(s["logits"], s["u"], s["tokens"], s["sample_ws"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"], probs=s["probs"])
    return [s["tokens"], s["probs"]]


def _attended(s, c):
    s["kv"].kv_group_attn(s["plan"], s["view"], s["blocks"], 0, s["tree"], s["q"], s["out"], s["kv"].KV_OUT_F32 if c["out"] == "f32" else s["kv"].KV_OUT_SAME, 0, s["ws"],
                          groups=s["shared"], scores=s["scores"])
    return s["out"]


def run(state):
    s, c = state, state["case"]
    if not own:
        return _plain(s, c)
    if c["kind"] == "attn":
        return _attended(s, c)
    if c["kind"] == "sample":
        return _sampled(s, c)
    s["kv"].kv_step_tables(s["tables"])
    got = [s[k + "_out"] for k in ("table", "held", "n_free", "status", "tok_first", "tok_seq", "tok_slot")] + [s["free"]]
    if c["kind"] == "tables":
        return got
    s["kv"].kv_cache_write(s["plan"], s["view"], s["blocks"], 0, s["k_new"], s["v_new"], s["tok_seq_out"], s["tok_slot_out"])
    return got + [_attended(s, c)] + _sampled(s, c)


def work(case):
    c = case
    got = {"bytes": 0.0, "flops": 0.0}

    def add(n_bytes, flops=0.0):
        got["bytes"] += n_bytes
        got["flops"] += flops
    if c["kind"] in ("tables", "step"):
        lens, news, _, _, held, room, _ = _requests(c)
        gone = sum(h for h, t in zip(held, news) if t < 0)
        add(28 * c["B"] + 8 * c["B"] * room + 8 * gone + 8 * sum(max(0, t) for t in news))
    if c["kind"] in ("sample", "step"):
        add(c["B"] * (c["V"] * torch.finfo(DTYPES[c["dtype"]]).bits // 8 + 28), 4.0 * c["B"] * c["V"])
    if c["kind"] in ("attn", "step"):
        lens, news, parents, first, shared = _shapes(c)
        lo, up = _bounds(c, lens, news, parents)
        H, Hq, D, at, rows, pairs, least = c["H"], c["H"] * c["G"], c["D"], 0, 0, 0.0, list(shared)
        for b in range(c["B"]):
            n, mine = lens[b], lo[at:at + news[b]]
            own_from = next((shared[g] for g in range(len(shared)) if first[g] <= b < first[g + 1]), 0)
            for g in range(len(shared)):
                if first[g] <= b < first[g + 1]:
                    least[g] = min(least[g], min(mine))
            rows += n + news[b] - max(own_from, min(mine))
            for i, depth in enumerate(_depths(parents[b])):
                end = max(n + depth + 1, up[at + i])
                pairs += max(0, end - mine[i])
            at += news[b]
        rows += sum(p - m for p, m in zip(shared, least))
        row = {"16": 2 * D, "fp8": D + D // BLOCK, "fp4": D // 2 + D // BLOCK}[c["fmt"]]
        out = at * Hq * D * (4 if c["out"] == "f32" else 2)
        add(2 * H * row * rows + at * Hq * 2 * D + out + (8 * at * ((max(news) + 63) // 64) if c["tree"] else 0), 4.0 * Hq * D * pairs)
        if c["kind"] == "step":
            add(at * (2 * H * (2 * D + row) + 8))
    return got


# ------------------------------------------------------------------------------------------ the definition in 64 bits
def _exact_tables(s, c):
    lens, news, leader, common, held, room, _ = _requests(c)
    bt, table, free, n = c["bt"], s["table"].tolist(), s["free"].tolist(), int(s["n_free"])
    stack, rest = free[:n], free[n:]
    rows = [list(r) for r in table]
    common = [k if a >= 0 else 0 for k, a in zip(common, leader)]
    now = list(held)
    for b, t in enumerate(news):
        if t < 0:
            stack += rows[b][common[b]:held[b]]
            rows[b], now[b] = [-1] * room, 0
    free = stack + rest[len(stack) - n:]
    need = [-(-(a + t) // bt) if t >= 0 else 0 for a, t in zip(lens, news)]
    missing = max(0, sum(max(0, x - max(h, k)) for x, h, k in zip(need, held, common)) - len(stack))
    over = sum(x > room for x in need)
    if not missing and not over:
        for b, x in enumerate(need):
            for i in range(max(held[b], common[b]), x):
                rows[b][i] = stack.pop()
            now[b] = max(now[b], x) if news[b] >= 0 else 0
        for b, x in enumerate(need):
            for i in range(held[b], min(common[b], x)):
                rows[b][i] = rows[leader[b]][i]
    first, seq, slot = [0], [], []
    for b, t in enumerate(news):
        first.append(first[-1] + max(0, t))
        seq += [b] * max(0, t)
        slot += range(lens[b], lens[b] + max(0, t))
    put = lambda v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    return [put(x) for x in (rows, now, [len(stack)], [missing, over], first, seq, slot, free)]


def _two_to(e):
    """2^e of whole numbers, put together from its bits."""
    return (e.long() + 1023 << 52).view(torch.float64)


def _exact_rows(s, c, b, kind, n, table):
    """[H, n, D]: the first n cached rows in sequence b's place."""
    def rows(x):
        if c["layout"] == "paged":
            return torch.cat([x[max(i, 0)] for i in table[b][:-(-n // c["bt"])]], 1)[:, :n]
        return x[b, :, :n]
    if n == 0:
        return torch.zeros((c["H"], 0, c["D"]), dtype=torch.float64, device="cuda")
    x = rows(s[kind])
    if c["fmt"] == "16":
        return x.double()
    if c["fmt"] == "fp8":
        m, e = x & 7, x >> 3 & 15
        v = torch.where(e == 0, m.double() * 2.0 ** -9, (8 + m).double() * _two_to(e.long() - 10))
        v = torch.where(x >= 128, -v, v)
    else:
        x = torch.stack([x % 16, x // 16], -1).flatten(-2)
        v = torch.tensor(FP4, dtype=torch.float64, device="cuda")[(x % 8).long()] * torch.where(x >= 8, -1.0, 1.0).double()
    return v * _two_to(rows(s[kind + "_scale"]).long() - 127).repeat_interleave(BLOCK, -1)


def _exact_attn(s, c, table):
    lens, news, parents, first, shared = _shapes(c)
    lo, up = _bounds(c, lens, news, parents)
    H, G, D = c["H"], c["G"], c["D"]
    out = torch.zeros((sum(news), H * G, D), dtype=torch.float64, device="cuda")
    at = 0
    for b in range(c["B"]):
        n, t = lens[b], news[b]
        k, v = (_exact_rows(s, c, b, kind, n + t, table) for kind in ("k", "v"))
        for g in range(len(shared)):
            if first[g] <= b < first[g + 1]:
                k, v = (torch.cat([_exact_rows(s, c, first[g], kind, shared[g], table), x[:, shared[g]:]], 1) for kind, x in (("k", k), ("v", v)))
        sees = torch.zeros((t, n + t), dtype=torch.bool)
        sees[:, :n] = True
        for i, p in enumerate(parents[b]):
            if c["tree"]:
                if p >= 0:
                    sees[i, n:] = sees[p, n:]
                sees[i, n + i] = True
            else:
                sees[i, n:n + i + 1] = True
        for i in range(t):
            if c["both"]:
                sees[i, :min(up[at + i], n + t)] = True
            sees[i, :max(0, lo[at + i])] = False
        sees = sees.cuda()
        pos = torch.cat([torch.arange(n), n + torch.tensor(_depths(parents[b]))]).cuda().double()
        for h in range(H * G):
            x = s["q"][at:at + t, h].double() @ k[h // G].T / math.sqrt(D)
            if c["cap"]:
                x = torch.tanh(x / c["cap"]) * c["cap"]
            if c["slopes"]:
                x = x - s["slope"][h].double() * (pos[n:, None] - pos).abs()
            out[at:at + t, h] = torch.nan_to_num(torch.softmax(x.masked_fill(~sees, -math.inf), -1), 0.0) @ v[h // G]
        at += t
    return out


def _exact_sample(s, c):
    tokens, probs = [], []
    for b in range(c["B"]):
        x = s["logits"][b].double()
        t, k, p, m, u = (float(s[n][b]) for n in ("temperature", "top_k", "top_p", "min_p", "u"))
        if t == 0:
            token, prob = int((x == x.max()).nonzero()[0]), 1.0
        else:
            w = ((x - x.max()) / t).exp()
            order = torch.argsort(-x, stable=True)
            order = order[:int(k)] if k > 0 else order
            if p < 1:
                sums = w[order].cumsum(0)
                order = order[:int((sums < p * sums[-1]).sum()) + 1]
            order = order[w[order] >= m].sort().values
            sums = w[order].cumsum(0)
            i = min(int((sums <= u * sums[-1]).sum()), int((w[order] > 0).nonzero()[-1]))
            token, prob = int(order[i]), float(w[order[i]] / sums[-1])
        tokens.append(token)
        probs.append(prob)
    return [torch.tensor(tokens, dtype=torch.int32), torch.tensor(probs, dtype=torch.float64)]


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    if c["kind"] == "tables":
        return _exact_tables(s, c)
    if c["kind"] == "sample":
        return _exact_sample(s, c)
    if c["kind"] == "attn":
        return _exact_attn(s, c, s["table_blocks"].tolist() if c["layout"] == "paged" else None)
    got = _exact_tables(s, c)
    table = got[0].tolist()
    for i, (b, j) in enumerate(zip(got[5].tolist(), got[6].tolist())):
        at = table[b][j // c["bt"]]
        s["k"][at, :, j % c["bt"]], s["v"][at, :, j % c["bt"]] = s["k_new"][i], s["v_new"][i]
    return got + [_exact_attn(s, c, table)] + _exact_sample(s, c)
