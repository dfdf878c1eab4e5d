"""The operators of a serving step over a cache that may be held in 8 or 4 bits: rotary positions, rows written to and read
back from a block-scaled cache, and attention for a tree of drafted tokens (or one token) over it.

A case is a dict of plain values.  `kind` says what one pass does:
  rope    rotary positions of the query rows of a step or a prefill, or of the gradient that comes back through them
  cache   new K and V rows into a cache of blocks (K rotated on its way), then those rows read back as 16-bit values
  read    all rows of a cache read back as 16-bit values
  attn    attention of drafted tokens over the cache: each sees the whole context and its ancestors among the drafted
  step    a verification step: rope of q, write of k and v, attention over the cache, the written rows read back

A cache row of 8 or 4 bits is codes (e4m3; e2m1, two to a byte, the lower half first) and a power of two for every 32 of
them (its exponent + 127 in a byte), the smallest with which no code saturates.
Lengths, trees, block tables and everything else that fixes the amount of work come from the case; values from the seed.
"""
import math
import random

import torch

own = False
BLOCK = 32
FP4 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _case(kind, B, H, G, D, lo, hi, tlo, thi, dtype, layout, fmt, **more):
    """B sequences of lo..hi cached tokens and tlo..thi new ones each, H KV heads with G query heads each."""
    c = {"kind": kind, "B": B, "H": H, "G": G, "D": D, "lo": lo, "hi": hi, "tlo": tlo, "thi": thi, "dtype": dtype, "layout": layout,
         "fmt": fmt, "bt": 16, "out": "same", "tree": True, "rot": D, "style": "half", "transposed": False, "shape_seed": 3}
    c.update(more)
    return c


def listed():
    return [
        # the smallest call: a short chat with four drafted tokens, latency and launches only
        _case("attn", 1, 2, 2, 64, 256, 256, 4, 4, "f16", "bhsd", "16", name="attn_tiny"),
        # one interactive sequence at 4K context, 8B shape, a tree of 16
        _case("attn", 1, 8, 4, 128, 4096, 4096, 16, 16, "f16", "bhsd", "16", name="attn_4k_tree16"),
        # one long sequence, 8B shape at 32K, the largest trees in use: as much arithmetic as memory traffic
        _case("attn", 1, 8, 4, 128, 32768, 32768, 64, 64, "bf16", "bhsd", "fp8", name="attn_32k_tree64_fp8"),
        # a ragged batch over a paged cache, 8B shape, trees of odd sizes
        _case("attn", 8, 8, 4, 128, 1024, 8192, 5, 29, "f16", "paged", "16", name="attn_ragged_paged"),
        # plain decoding, a token at a time: many ragged sequences over a paged 4-bit cache, an odd number of heads per KV head
        _case("attn", 48, 4, 7, 128, 200, 4000, 1, 1, "bf16", "paged", "fp4", tree=False, name="attn_single_serving_fp4"),
        # wide heads without grouping, batch 4 at 8K: the most bytes, a short chain of drafted tokens, 32-bit results
        _case("attn", 4, 16, 1, 256, 8192, 8192, 6, 6, "bf16", "bhsd", "fp8", tree=False, out="f32", name="attn_wide_chain_fp8"),
        # the queries of a decode step of 8 sequences
        _case("rope", 8, 8, 4, 128, 1024, 8192, 1, 1, "f16", "bhsd", "16", name="rope_step"),
        # the gradient of a prefill's queries; half of each head is rotated, pairs side by side
        _case("rope", 2, 8, 4, 128, 0, 0, 4000, 4096, "bf16", "bhsd", "16", rot=64, style="pairs", transposed=True, name="rope_prefill_gradient"),
        # drafted rows of a ragged batch into a paged 8-bit cache
        _case("cache", 8, 8, 4, 128, 1024, 8192, 5, 29, "f16", "paged", "fp8", name="cache_tree_rows_fp8"),
        # a prefill of 8K tokens into a 4-bit cache
        _case("cache", 1, 8, 4, 128, 0, 0, 8192, 8192, "bf16", "bhsd", "fp4", name="cache_prefill_fp4"),
        # a ragged batch's whole cache back to 16 bits, as ahead of a prefill on top of it
        _case("read", 8, 8, 4, 128, 1024, 8192, 1, 1, "f16", "paged", "fp8", name="read_ragged_fp8"),
        # everything together: a batch's verification step over an 8-bit paged cache
        _case("step", 8, 8, 4, 128, 1024, 8192, 5, 29, "bf16", "paged", "fp8", name="step_ragged_fp8"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attn"] * 6 + ["rope", "cache", "cache", "read", "step", "step"])
    D = rng.choice([64, 128, 128, 256])
    H = rng.choice([1, 2, 3, 4, 5, 8, 8, 16])
    G = rng.choice([1, 1, 2, 3, 4, 4, 5, 6, 7, 8])
    B = _log_int(rng, 1, 48)
    hi = _log_int(rng, 48, 32768)
    lo = hi if rng.random() < 0.3 else rng.randint(hi // 8, hi)
    thi = 1 if rng.random() < 0.25 else _log_int(rng, 2, 64)
    tlo = thi if rng.random() < 0.3 else rng.randint(1, thi)
    dtype, layout = rng.choice(["f16", "bf16"]), rng.choice(["bhsd", "paged"])
    fmt = rng.choice(["16", "fp8", "fp4"] if kind in ("attn", "step") else ["fp8", "fp4"])
    more = {"shape_seed": rng.randrange(1 << 30), "out": rng.choice(["f32", "same", "same"]), "tree": rng.random() < 0.7,
            "rot": rng.choice([D, D, D // 2]), "style": rng.choice(["half", "pairs"]), "transposed": kind == "rope" and rng.random() < 0.5}
    if layout == "paged":
        more["bt"] = rng.choice([16, 16, 16, 32, 64])
    if kind in ("rope", "cache"):  # new rows only: a step's, or a prefill's
        thi = _log_int(rng, 1, 8192)
        tlo = thi if rng.random() < 0.5 else rng.randint(1, thi)
        lo = hi = rng.choice([0, 0, 17, 1000])
        while B * thi * H * D * (G if kind == "rope" else 1) > 2 ** 24:
            B, thi = (B // 2, thi) if B > 1 else (1, thi // 2)
        tlo = min(tlo, thi)
    # no more than the largest listed case: so many cached values, and as many products
    most = 2 ** 25 if kind == "read" else 2 ** 26 if fmt == "16" else 2 ** 27
    while B * hi * H * D > most or B * hi * thi * H * G * D > 2 ** 33:
        if hi > 512 and (B == 1 or rng.random() < 0.5):
            hi = max(48, hi // 2)
            lo = max(1, min(lo // 2, hi))
        elif B > 1:
            B = B // 2
        else:
            thi = max(1, thi // 2)
            tlo = min(tlo, thi)
    return _case(kind, B, H, G, D, lo, hi, tlo, thi, dtype, layout, fmt, **more)


# ------------------------------------------------------------------------------------------ inputs
def _shapes(c):
    """(context lengths, numbers of new tokens, each new token's parent among its sequence's, -1 for none)."""
    r = random.Random(c["shape_seed"])
    lens = [r.randint(c["lo"], c["hi"]) for _ in range(c["B"])]
    news = [r.randint(c["tlo"], c["thi"]) for _ in range(c["B"])]
    # drafters extend recent tokens most of the time; without a tree every token follows the one before it
    parents = [[max(-1, i - 1 - (int(r.expovariate(0.3)) if c["tree"] else 0)) for i in range(n)] for n in news]
    return lens, news, parents


def _masks(parents, words):
    """A bit for every drafted token that each one sees: its ancestors and itself; and how deep each one is."""
    masks, depths = [], []
    for p in parents:
        bits = []
        for i, up in enumerate(p):
            bits.append((bits[up] if up >= 0 else 0) | 1 << i)
            depths.append(depths[len(depths) - i + up] + 1 if up >= 0 else 0)
        for b in bits:
            w = [b >> 64 * k & (1 << 64) - 1 for k in range(words)]
            masks.append([x - (1 << 64) if x >> 63 else x for x in w])
    return torch.tensor(masks, dtype=torch.int64), torch.tensor(depths, dtype=torch.int32)


def _table(c, n_pos, device):
    """Cosines and sines by position and frequency [n_pos, rot / 2, 2].  Waves longer than the context that a model was
    trained on are stretched by 8, shorter than a quarter of it kept, in between a mixture."""
    half = c["rot"] // 2
    f = 500000.0 ** (-torch.arange(half, dtype=torch.float64, device=device) / half)
    keep = ((8192 * f / (2 * math.pi) - 1) / 3).clamp(0, 1)
    f = f * (keep + (1 - keep) / 8)
    a = torch.arange(n_pos, dtype=torch.float64, device=device)[:, None] * f
    return torch.stack([a.cos(), a.sin()], -1).float().contiguous()


def _dtype(c):
    return torch.float16 if c["dtype"] == "f16" else torch.bfloat16


def _rows(shape, gen, outlying):
    """N(0, 1), a channel in 16 of K three times as wide."""
    x = torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)
    if outlying:
        x[..., 5::16] *= 3
    return x


def _code_bytes(c):
    return {"16": 2 * c["D"], "fp8": c["D"], "fp4": c["D"] // 2}[c["fmt"]]


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dt, (B, H, D) = _dtype(c), (c["B"], c["H"], c["D"])
    lens, news, parents = _shapes(c)
    n, Hq = sum(news), H * c["G"]
    s = {"case": c, "lens": lens, "news": news, "total": max(a + b for a, b in zip(lens, news))}
    dev = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    s["lens_dev"], s["news_dev"] = dev(lens), dev(news)
    s["first"] = [sum(news[:b]) for b in range(B + 1)]
    s["first_dev"] = dev(s["first"])
    s["tok_seq"] = dev([b for b in range(B) for _ in range(news[b])])
    s["tok_slot"] = dev([lens[b] + i for b in range(B) for i in range(news[b])])
    if c["kind"] in ("attn", "step"):
        mask, depths = _masks(parents, (max(news) + 63) // 64)
        s["mask"] = mask.cuda() if c["tree"] else None
        s["pos"] = torch.tensor([x for b in range(B) for x in [lens[b]] * news[b]], dtype=torch.int32, device="cuda") + depths.cuda()
    else:
        s["pos"] = s["tok_slot"]
    if c["kind"] != "attn":
        s["table"] = _table(c, s["total"], "cuda")
    if c["kind"] == "read":  # the whole cache, a sequence after the other
        s["tok_seq"] = dev([b for b in range(B) for _ in range(lens[b])])
        s["tok_slot"] = dev([i for b in range(B) for i in range(lens[b])])
    if c["kind"] != "rope":
        _cache(s, c, gen)
    if c["kind"] in ("rope", "attn", "step"):
        s["q"] = _rows((n, Hq, D), gen, False).to(dt)
    if c["kind"] in ("cache", "step"):
        s["k_new"], s["v_new"] = _rows((n, H, D), gen, True).to(dt), _rows((n, H, D), gen, False).to(dt)
    rows = s["tok_seq"].numel()
    if c["kind"] in ("cache", "read", "step"):
        s["k_back"], s["v_back"] = (torch.zeros((rows, H, D), dtype=dt, device="cuda") for _ in range(2))
    if c["kind"] in ("attn", "step"):
        s["out"] = torch.zeros((n, Hq, D), dtype=torch.float32 if c["out"] == "f32" else dt, device="cuda")
    if c["kind"] in ("rope", "step"):
        s["q_out"] = torch.zeros((n, Hq, D), dtype=dt, device="cuda")
    if own:
        _handles(s, c)
    return s


def _cache(s, c, gen):
    """K and V (and their scales) of every context and, where nothing writes them, of the drafted tokens, in the cache's layout."""
    B, H, D, bt = c["B"], c["H"], c["D"], c["bt"]
    if c["layout"] == "paged":
        per = [(a + b + bt - 1) // bt for a, b in zip(s["lens"], s["news"])]
        ids = list(range(sum(per)))
        random.Random(c["shape_seed"] + 1).shuffle(ids)
        table, at = torch.full((B, max(per)), -1, dtype=torch.int32), 0
        for b, k in enumerate(per):
            table[b, :k] = torch.tensor(ids[at:at + k], dtype=torch.int32)
            at += k
        s["table_blocks"] = table.cuda()
        shape = (len(ids), H, bt)
    else:
        shape = (B, H, s["total"])
    for kind in ("k", "v"):
        dtype = _dtype(c) if c["fmt"] == "16" else torch.uint8
        s[kind] = torch.empty(shape + (D if c["fmt"] != "fp4" else D // 2,), dtype=dtype, device="cuda")
        if c["fmt"] != "16":
            s[kind + "_scale"] = torch.empty(shape + (D // BLOCK,), dtype=torch.uint8, device="cuda")
        some = max(1, 2 ** 23 // (H * shape[2] * D))
        for i in range(0, shape[0], some):
            x = _rows((min(some, shape[0] - i),) + shape[1:] + (D,), gen, kind == "k").to(_dtype(c))
            if c["fmt"] == "16":
                s[kind][i:i + some] = x
            else:
                s[kind][i:i + some], s[kind + "_scale"][i:i + some] = _quantise(x.float(), c["fmt"], c["dtype"])


def _handles(s, c):
    """The plan, views and workspace that a program which serves from this cache keeps."""
    from paper_2604_26557_amd import binding as kv
    s["kv"] = kv
    B, H, D = c["B"], c["H"], c["D"]
    s["plan"] = kv.kv_layout_plan(1, H, H * c["G"], D, [s["total"]] * B, kv.KV_F16 if c["dtype"] == "f16" else kv.KV_BF16, 512, 4096, kv.KV_PER_SEQ)
    if "table" in s:
        s["rope"] = kv.Rope(s["table"], kv.KV_ROPE_HALF if c["style"] == "half" else kv.KV_ROPE_PAIRS)
    if c["kind"] == "rope":
        return
    k, v = [s["k"].view(torch.int16)], [s["v"].view(torch.int16)]
    if c["layout"] == "paged":
        s["view"] = kv.paged_view(k, v, s["table_blocks"], s["lens"], s["lens_dev"])
    else:
        s["view"] = kv.bhsd_view(k, v, s["lens"], s["lens_dev"])
    s["blocks"] = None
    if c["fmt"] != "16":
        s["blocks"] = kv.scale_blocks(kv.KV_FORMAT_FP8 if c["fmt"] == "fp8" else kv.KV_FORMAT_FP4, [s["k_scale"]], [s["v_scale"]])
    if c["kind"] in ("attn", "step"):
        s["tree"] = kv.tree_batch(s["first"], s["first_dev"], s["mask"])
        s["ws"] = torch.empty(kv.kv_tree_attn_workspace(s["plan"], s["first"][-1], s["total"]), dtype=torch.uint8, device="cuda")


# ------------------------------------------------------------------------------------------ plain forms
def _rotate(x, c, table, pos):
    """Pairs (d, d + rot / 2), or (2 d, 2 d + 1), turned by the angle of their position and frequency."""
    x, r, cs = x.float(), c["rot"], table[pos.long()][:, None]
    cos, sin = cs[..., 0], -cs[..., 1] if c["transposed"] else cs[..., 1]
    if c["style"] == "half":
        a, b = x[..., :r // 2], x[..., r // 2:r]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([turned, x[..., r:]], -1).to(_dtype(c))


def _power(e):
    """2^e from e + 127, as a byte's value."""
    return torch.where(e == 0, 2.0 ** -127, (e.int() << 23).view(torch.float32))


def _quantise(x, fmt, dtype):
    """Codes and scales of rows [..., D] in 32 bits.  A block with a value that is not finite stands for NaN throughout; what would round
    beyond the 16-bit type saturates."""
    top, shift = (0.875, 9) if fmt == "fp8" else (0.75, 3)  # the largest code, 448 or 6, as top * 2^shift
    if dtype == "f16":
        limit = 61440.0 if fmt == "fp8" else 49152.0
        x = torch.where(x.isfinite(), x.clamp(-limit, limit), x)
    x = x.unflatten(-1, (-1, BLOCK))
    big = x.abs().amax(-1)
    fine = x.isfinite().all(-1)
    m, e = torch.frexp(torch.where(fine, big, 1.0))
    e = torch.where(big == 0, -127, e - shift + (m > top)).clamp(-127, 127) + 127
    y = x * _power(254 - e)[..., None]
    y = torch.where(fine[..., None], y, 0.0).flatten(-2)
    scale = torch.where(fine, e, 255).to(torch.uint8)
    if fmt == "fp8":
        return y.to(torch.float8_e4m3fn).view(torch.uint8), scale
    a = y.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    code = torch.bucketize((a / step).round() * step, torch.tensor(FP4, device=x.device)).to(torch.uint8) | torch.signbit(y).to(torch.uint8) << 3
    return code[..., 0::2] | code[..., 1::2] << 4, scale


def _values(codes, scale, fmt):
    """Rows in 32 bits."""
    if fmt == "16":
        return codes.float()
    if fmt == "fp8":
        x = codes.view(torch.float8_e4m3fn).float()
    else:
        t = torch.tensor(FP4 + tuple(-v for v in FP4), device=codes.device)
        x = t[torch.stack([codes & 15, codes >> 4], -1).flatten(-2).int()]
    return (x.unflatten(-1, (-1, BLOCK)) * torch.where(scale == 255, torch.nan, _power(scale))[..., None]).flatten(-2)


def _place(s, c):
    """Index of each row in [first dimension, H, row] of the cache."""
    seq, slot = s["tok_seq"].long(), s["tok_slot"].long()
    if c["layout"] == "paged":
        return s["table_blocks"][seq, slot // c["bt"]].long(), slot % c["bt"]
    return seq, slot


def _write(s, c):
    at, row = _place(s, c)
    for kind, x in (("k", _rotate(s["k_new"], c, s["table"], s["pos"])), ("v", s["v_new"])):
        if c["fmt"] == "16":
            s[kind][at, :, row] = x
        else:
            s[kind][at, :, row], s[kind + "_scale"][at, :, row] = _quantise(x.float(), c["fmt"], c["dtype"])


def _read(s, c):
    at, row = _place(s, c)
    return [_values(s[kind][at, :, row], s[kind + "_scale"][at, :, row] if c["fmt"] != "16" else None, c["fmt"]).to(_dtype(c)) for kind in ("k", "v")]


def _dense(s, c, kind):
    """[B, H, total, D] in 32 bits."""
    def laid(x):
        if c["layout"] == "paged":
            x = x[s["table_blocks"].clamp(min=0).long()].transpose(1, 2).flatten(2, 3)[:, :, :s["total"]]
        return x
    return _values(laid(s[kind]), laid(s[kind + "_scale"]) if c["fmt"] != "16" else None, c["fmt"])


def _visible(s, c):
    """[B, T, total]: which rows of the cache each new token sees."""
    B, T, S = c["B"], max(s["news"]), s["total"]
    first, n = s["tok_seq"].long(), s["tok_seq"].numel()
    index = torch.arange(n, device="cuda") - s["first_dev"].long()[first]
    j = torch.arange(S, device="cuda")
    rel = j - s["lens_dev"].long()[:, None]  # [B, S]
    if s["mask"] is None:
        bits = torch.arange(T, device="cuda")[:, None] >= torch.arange(T, device="cuda")
        bits = bits.expand(B, T, T)
    else:
        words = s["mask"].shape[1]
        flat = ((s["mask"][:, :, None] >> torch.arange(64, device="cuda")) & 1).bool().flatten(1)
        bits = torch.zeros((B, T, 64 * words), dtype=torch.bool, device="cuda")
        bits[first, index] = flat
    drafted = bits.gather(2, rel.clamp(0, bits.shape[2] - 1)[:, None].expand(B, T, S))
    inside = (rel >= 0) & (rel < s["news_dev"].long()[:, None])
    return (rel < 0)[:, None] | (inside[:, None] & drafted), first, index


def _attend(s, c, q):
    B, H, G, D, T = c["B"], c["H"], c["G"], c["D"], max(s["news"])
    visible, seq, index = _visible(s, c)
    rows = torch.zeros((B, T, H * G, D), device="cuda")
    rows[seq, index] = q.float()
    rows = rows.unflatten(2, (H, G)).transpose(1, 2).flatten(2, 3)  # [B, H, T * G, D]
    scores = torch.matmul(rows, _dense(s, c, "k").transpose(2, 3).contiguous()) * D ** -0.5
    scores = scores.masked_fill(~visible.repeat_interleave(G, 1)[:, None], -torch.inf)
    top = scores.amax(-1, keepdim=True)
    p = (scores - torch.where(top == -torch.inf, 0.0, top)).exp()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, _dense(s, c, "v")) / torch.where(total == 0, 1.0, total)
    out = out.unflatten(2, (T, G)).transpose(1, 2).flatten(2, 3)[seq, index]
    return out if c["out"] == "f32" else out.to(_dtype(c))


def _plain(s, c):
    if c["kind"] == "rope":
        return _rotate(s["q"], c, s["table"], s["pos"])
    if c["kind"] == "read":
        return _read(s, c)
    if c["kind"] == "cache":
        _write(s, c)
        return _read(s, c)
    if c["kind"] == "attn":
        return _attend(s, c, s["q"])
    q = _rotate(s["q"], c, s["table"], s["pos"])
    _write(s, c)
    return [_attend(s, c, q)] + _read(s, c)


# ------------------------------------------------------------------------------------------ one pass
def run(state):
    s, c = state, state["case"]
    if not own:
        return _plain(s, c)
    kv, kind = s["kv"], c["kind"]
    if kind in ("rope", "step"):
        kv.kv_rope(s["rope"], s["pos"], s["q"], s["q_out"], transposed=c["transposed"])
    if kind == "rope":
        return s["q_out"]
    if kind in ("cache", "step"):
        kv.kv_cache_write(s["plan"], s["view"], s["blocks"], 0, s["k_new"], s["v_new"], s["tok_seq"], s["tok_slot"], s["rope"], s["pos"])
    if kind in ("attn", "step"):
        kv.kv_tree_attn(s["plan"], s["view"], s["blocks"], 0, s["tree"], s["q_out"] if kind == "step" else s["q"], s["out"],
                        kv.KV_OUT_F32 if c["out"] == "f32" else kv.KV_OUT_SAME, 0, s["ws"])
    if kind == "attn":
        return s["out"]
    kv.kv_cache_read(s["plan"], s["view"], s["blocks"], 0, s["tok_seq"], s["tok_slot"], s["k_back"], s["v_back"])
    return [s["out"], s["k_back"], s["v_back"]] if kind == "step" else [s["k_back"], s["v_back"]]


def work(case):
    c = case
    lens, news, _ = _shapes(c)
    H, Hq, D, n = c["H"], c["H"] * c["G"], c["D"], sum(news)
    row = _code_bytes(c) + (0 if c["fmt"] == "16" else D // BLOCK)  # a head's cached row of K or V
    angles = 4 * c["rot"] + 4  # cosines, sines and position of a token
    rope = {"bytes": n * (2 * Hq * 2 * D + angles), "flops": 3.0 * n * Hq * c["rot"]}
    write = n * (2 * H * (2 * D + row) + 8 + angles)
    back = 2 * H * (2 * D + row) + 8
    out = n * Hq * D * (4 if c["out"] == "f32" else 2)
    attn = {"bytes": 2 * H * row * (sum(lens) + n) + n * Hq * 2 * D + out + (8 * n * ((max(news) + 63) // 64) if c["tree"] else 0),
            "flops": 4.0 * Hq * D * sum(t * (a + (t + 1) // 2) for a, t in zip(lens, news))}
    if c["kind"] == "rope":
        return rope
    if c["kind"] == "cache":
        return {"bytes": write + n * back, "flops": 3.0 * n * H * c["rot"]}
    if c["kind"] == "read":
        return {"bytes": sum(lens) * back, "flops": 0}
    if c["kind"] == "attn":
        return attn
    return {"bytes": rope["bytes"] + write + attn["bytes"] + n * back, "flops": rope["flops"] + 3.0 * n * H * c["rot"] + attn["flops"]}


# ------------------------------------------------------------------------------------------ the definition in 64 bits
def _exact_rope(x, c, table, pos):
    """Each pair as a complex number times that of its angle."""
    x, r = x.double().clone(), c["rot"]
    turn = torch.view_as_complex(table.double())[pos.long()][:, None]
    turn = turn.conj() if c["transposed"] else turn
    i = torch.arange(r // 2, device=x.device)
    re, im = (i, i + r // 2) if c["style"] == "half" else (2 * i, 2 * i + 1)
    z = torch.complex(x[..., re], x[..., im]) * turn
    x[..., re], x[..., im] = z.real, z.imag
    return x


def _two_to(e):
    """2^e of whole numbers, put together from its bits."""
    return (e.long() + 1023 << 52).view(torch.float64)


def _exact_blocks(x, fmt, dtype):
    """The values that rows of finite numbers [..., D] are cached as: the nearest of the format's, ties to the even code."""
    codes = torch.arange(127 if fmt == "fp8" else 8, device=x.device)
    if fmt == "fp8":  # 4 bits of exponent, 3 of mantissa
        grid = torch.where(codes < 8, codes * 2.0 ** -9, (8 + codes % 8).double() * _two_to(codes // 8 - 10))
    else:
        grid = torch.tensor(FP4, dtype=torch.float64, device=x.device)
    if dtype == "f16":
        x = x.clamp(-61440.0, 61440.0) if fmt == "fp8" else x.clamp(-49152.0, 49152.0)
    x = x.unflatten(-1, (-1, BLOCK))
    need = x.abs().amax(-1, keepdim=True) / grid[-1]
    e = torch.log2(need).ceil().clamp(-127, 127)
    e = e + (_two_to(e) < need).double()
    e = torch.where((_two_to(e - 1) >= need) & (e > -127), e - 1, e).clamp(-127, 127)
    y = x.abs() / _two_to(e)
    above = torch.searchsorted(grid, y).clamp(max=len(grid) - 1)
    below = (above - 1).clamp(min=0)
    up, down = grid[above] - y, y - grid[below]
    code = torch.where((up < down) | ((up == down) & (above % 2 == 0)), above, below)
    code = torch.where(grid[above] == y, above, code)
    return (torch.copysign(grid[code], x) * _two_to(e)).flatten(-2)


def _exact_values(s, c, b, kind):
    """[H, rows, D]: sequence b's cached rows."""
    n = s["lens"][b] + s["news"][b]

    def rows(x):
        if c["layout"] == "paged":
            return torch.cat([x[i] for i in s["table_blocks"][b].tolist() if i >= 0], 1)[:, :n]
        return x[b, :, :n]
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


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    lens, news, parents = _shapes(c)
    H, G, D, dt = c["H"], c["G"], c["D"], _dtype(c)
    if c["kind"] == "rope":
        return _exact_rope(s["q"], c, s["table"], s["pos"])
    if c["kind"] == "read":
        return [torch.cat([_exact_values(s, c, b, kind)[:, :lens[b]] for b in range(c["B"])], 1).transpose(0, 1).contiguous() for kind in ("k", "v")]
    q = s.get("q")
    if c["kind"] in ("cache", "step"):  # what is rotated is rounded to 16 bits before it is cached
        new = [_exact_rope(s["k_new"], c, s["table"], s["pos"]).to(dt).double(), s["v_new"].double()]
        new = [x if c["fmt"] == "16" else _exact_blocks(x, c["fmt"], c["dtype"]) for x in new]
        if c["kind"] == "cache":
            return new
        q = _exact_rope(q, c, s["table"], s["pos"]).to(dt)
    out = torch.zeros((sum(news), H * G, D), dtype=torch.float64, device="cuda")
    for b in range(c["B"]):
        at, n = s["first"][b], lens[b]
        k, v = (_exact_values(s, c, b, kind) for kind in ("k", "v"))
        if c["kind"] == "step":
            k, v = (torch.cat([x[:, :n], y[at:at + news[b]].transpose(0, 1)], 1) for x, y in zip((k, v), new))
        sees = torch.zeros((news[b], n + news[b]), dtype=torch.bool)
        sees[:, :n] = True
        for i, up in enumerate(parents[b]):
            if up >= 0:
                sees[i, n:] = sees[up, n:]
            sees[i, n + i] = True
        sees = sees.cuda()
        for h in range(H):
            x = q[at:at + news[b], h * G:(h + 1) * G].double().flatten(0, 1) @ k[h].T / math.sqrt(D)
            x = x.masked_fill(~sees.repeat_interleave(G, 0), -math.inf)
            out[at:at + news[b], h * G:(h + 1) * G] = (torch.softmax(x, -1) @ v[h]).unflatten(0, (news[b], G))
    return [out] + new if c["kind"] == "step" else out
