"""Plain 64-bit forms of the serving step's operators on the CPU, and caches of every format and layout built from the same values."""
import math

import numpy as np
import torch

from paper_2604_26557_amd import binding as kv

FP8_GRID = np.array([m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10) for e in range(16) for m in range(8)][:127])
FP4_GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
FORMATS = {"16": None, "fp8": kv.KV_FORMAT_FP8, "fp4": kv.KV_FORMAT_FP4}
UNIT = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}   # half a unit in the last place, relative: 11 and 8 significant bits


def ref_quantise(x, fmt, f16):
    """Codes (one per element) and scale bytes of float64 rows [..., D], element by element from the definition."""
    grid = FP8_GRID if fmt == "fp8" else FP4_GRID
    most = (1.875 if fmt == "fp8" else 1.5) * 2.0 ** (15 if f16 else 127)   # what lies above rounds to 2^16, 2^128
    x = np.where(np.isfinite(x), np.clip(x, -most, most), x)
    b = x.reshape(x.shape[:-1] + (-1, 32))
    fine = np.isfinite(b).all(-1)
    big = np.where(fine, np.abs(np.where(np.isfinite(b), b, 0)).max(-1), 0)
    e = np.full(big.shape, -127)
    for k in range(-127, 128):   # the smallest that fits
        e = np.where(big > grid[-1] * 2.0 ** (k - 1), k, e) if k > -127 else e
    y = np.where(fine[..., None], b, 0) * 2.0 ** -e[..., None].astype(np.float64)
    a = np.abs(y)
    above = np.minimum(np.searchsorted(grid, a), len(grid) - 1)
    below = np.maximum(above - 1, 0)
    up, down = grid[above] - a, a - grid[below]
    code = np.where((up < down) | ((up == down) & (above % 2 == 0)), above, below)
    code = np.where(grid[above] == a, above, code)
    sign = 128 if fmt == "fp8" else 8
    code = code + np.where(np.signbit(y), sign, 0)
    return code.reshape(x.shape).astype(np.uint8), np.where(fine, e + 127, 255).astype(np.uint8)


def ref_values(code, scale, fmt):
    grid, sign = (FP8_GRID, 128) if fmt == "fp8" else (FP4_GRID, 8)
    if fmt == "fp8":
        grid = np.append(grid, np.nan)
    v = grid[code % sign] * np.where(code >= sign, -1.0, 1.0)
    s = np.where(scale == 255, np.nan, 2.0 ** (scale.astype(np.float64) - 127))
    return v * np.repeat(s, 32, -1)


def pack_codes(code, fmt):
    return code if fmt == "fp8" else (code[..., 0::2] | code[..., 1::2] << 4)


def unpack_codes(codes, fmt):
    return codes if fmt == "fp8" else np.stack([codes & 15, codes >> 4], -1).reshape(codes.shape[:-1] + (-1,))


def ref_rope(x, table, pos, rot, style, transposed=False):
    """float64 rows [n, heads, D]; table [n_pos, rot/2, 2]."""
    x = x.copy()
    i = np.arange(rot // 2)
    a, b = (i, i + rot // 2) if style == kv.KV_ROPE_HALF else (2 * i, 2 * i + 1)
    cs = table.astype(np.float64)[pos][:, None]
    c, s = cs[..., 0], -cs[..., 1] if transposed else cs[..., 1]
    xa, xb = x[..., a].copy(), x[..., b].copy()
    x[..., a], x[..., b] = xa * c - xb * s, xb * c + xa * s
    return x


def random_parents(rng, n, tree=True):
    return [int(rng.integers(-1, i)) if tree else i - 1 for i in range(n)]


def sees(parents):
    m = np.zeros((len(parents), len(parents)), dtype=bool)
    for i, p in enumerate(parents):
        if p >= 0:
            m[i] = m[p]
        m[i, i] = True
    return m


def ref_attention(q, k, v, n_ctx, m, scale):
    """q [T, Hq, D], k, v [H, n_ctx + T, D] in float64, m [T, T]: (out, sum p |v|, largest error of an exponent per 2^-24).  What a row does not
    see is left out of its sums."""
    T, Hq, D = q.shape
    H = k.shape[0]
    out, weight, spread = np.zeros((T, Hq, D)), np.zeros((T, Hq, D)), np.zeros((T, Hq))
    for t in range(T):
        idx = np.concatenate([np.arange(n_ctx), n_ctx + np.flatnonzero(m[t])])
        if len(idx) == 0:
            continue
        for h in range(Hq):
            kk, vv = k[h // (Hq // H)][idx], v[h // (Hq // H)][idx]
            s = (kk @ q[t, h]) * scale
            with np.errstate(all="ignore"):
                p = np.exp(s - s.max())
                p = p / p.sum()
                out[t, h], weight[t, h] = p @ vv, p @ np.abs(vv)
                spread[t, h] = (np.abs(kk) @ np.abs(q[t, h])).max() * scale * (D + 8) + np.abs(s).max() + 8
    return out, weight, spread


class Cache:
    """A cache of random rows in one format and layout, its copies on the device, and its values in float64 [B][H, rows, D]."""

    def __init__(self, lens, H, D, dtype, fmt="16", layout="bhsd", bt=16, seed=0, extra=0, device="cuda", n_q_heads=None, token_major_scales=False,
                 scale=1.0):
        self.fmt, self.layout, self.lens, self.dtype, self.D, self.H, self.bt = fmt, layout, list(lens), dtype, D, H, bt
        rng = np.random.default_rng(seed)
        B, rows = len(lens), max(max(lens) + extra, 1)
        self.rows, self.rng = rows, rng
        if layout == "paged":
            per = [(n + extra + bt - 1) // bt for n in lens]
            ids = rng.permutation(sum(per) + 2)
            table = np.full((B, max(max(per), 1)), -1, dtype=np.int32)
            at = 0
            for b, n in enumerate(per):
                table[b, :n] = ids[at:at + n]
                at += n
            self.table_host = table
            self.table = torch.from_numpy(table).to(device)
            shape = (len(ids), H, bt)
        else:
            shape = (B, H, rows)
        self.dev, self.values, self.code = {}, {}, {}
        for kind in ("k", "v"):
            x = torch.from_numpy(rng.standard_normal(shape + (D,)).astype(np.float32) * scale).to(dtype)
            if fmt == "16":
                self.dev[kind] = x.to(device)
                self.values[kind] = x.double().numpy()
            else:
                code, s = ref_quantise(x.double().numpy(), fmt, dtype == torch.float16)
                self.values[kind] = ref_values(code, s, fmt)
                self.dev[kind] = torch.from_numpy(pack_codes(code, fmt)).to(device)
                st = torch.from_numpy(s).to(device)
                if token_major_scales:   # [B, S, H, D/32] seen as [B, H, S, D/32]
                    st = st.transpose(1, 2).contiguous().transpose(1, 2)
                self.dev[kind + "_scale"] = st
        Hq = n_q_heads or H
        cap = [max(rows, 1)] * B
        self.plan = kv.kv_layout_plan(1, H, Hq, D, cap, kv.KV_F16 if dtype == torch.float16 else kv.KV_BF16, 512, 4096, kv.KV_PER_SEQ)
        self.lens_dev = torch.tensor(self.lens, dtype=torch.int32, device=device)
        self.remake()

    def remake(self):
        k, v = [self.dev["k"].view(torch.int16)], [self.dev["v"].view(torch.int16)]
        if self.layout == "paged":
            self.view = kv.paged_view(k, v, self.table, self.lens, self.lens_dev)
        else:
            self.view = kv.bhsd_view(k, v, self.lens, self.lens_dev)
        self.blocks = None if self.fmt == "16" else kv.scale_blocks(FORMATS[self.fmt], [self.dev["k_scale"]], [self.dev["v_scale"]])

    def place(self, b, slot):
        if self.layout == "paged":
            return int(self.table_host[b, slot // self.bt]), slot % self.bt
        return b, slot

    def seq(self, kind, b, n):
        """[H, n, D] of sequence b."""
        if n == 0:
            return np.zeros((self.H, 0, self.D))
        return np.stack([self.values[kind][self.place(b, j)[0], :, self.place(b, j)[1]] for j in range(n)], 1)

    def set_value(self, kind, b, slot, d, value):
        """One element of every head in a 16-bit cache; in a block-scaled one the whole block becomes NaN."""
        i, r = self.place(b, slot)
        if self.fmt == "16":
            self.dev[kind][i, :, r, d] = value
            self.values[kind][i, :, r, d] = value
        else:
            self.dev[kind + "_scale"][i, :, r, d // 32] = 255
            self.values[kind][i, :, r, d // 32 * 32:d // 32 * 32 + 32] = math.nan

    def attend(self, q, parents, out_dtype=None, n_splits=0, mask="tree", ws=None, scale=0.0, out=None, stream=None):
        """q [n, Hq, D] on the device; parents per sequence."""
        first = np.concatenate([[0], np.cumsum([len(p) for p in parents])]).astype(int).tolist()
        m = None
        if mask == "tree":
            words = max(1, (max(len(p) for p in parents) + 63) // 64)
            m = torch.cat([kv.kv_tree_masks(p, words)[0] for p in parents]).to(q.device)
        elif mask is not None:
            m = mask
        tree = kv.tree_batch(first, torch.tensor(first, dtype=torch.int32, device=q.device), m)
        od = kv.KV_OUT_F32 if out_dtype is None else out_dtype
        if out is None:
            out = torch.full(q.shape, 7.0, dtype=torch.float32 if od == kv.KV_OUT_F32 else self.dtype, device=q.device)
        if ws is None:
            ws = torch.empty(kv.kv_tree_attn_workspace(self.plan, first[-1], max(self.lens) + 256), dtype=torch.uint8, device=q.device)
        kv.kv_tree_attn(self.plan, self.view, self.blocks, 0, tree, q, out, od, n_splits, ws, scale, stream)
        return out

    def expected(self, q, parents, chain=False, masks=None, scale=None):
        outs, at = [], 0
        q = q.double().cpu().numpy()
        for b, p in enumerate(parents):
            n = self.lens[b]
            m = masks[b] if masks is not None else np.tril(np.ones((len(p), len(p)), dtype=bool)) if chain else sees(p)
            outs.append(ref_attention(q[at:at + len(p)], self.seq("k", b, n + len(p)), self.seq("v", b, n + len(p)), n, m, scale or self.D ** -0.5))
            at += len(p)
        return [np.concatenate([o[i] for o in outs]) for i in range(3)]


def attention_bound(out, weight, spread, rows, dtype, f32):
    """How far a result may be: 32-bit scores shift exponents by up to `spread` units of 2^-24 (the sum of D products, and the exponent's own
    rounding), which changes weights by that factor twice (numerator and sum); each sum over the rows adds a unit per doubling at least and per
    row at most, here 64 of them.  With 16-bit results probabilities are rounded once, numerator and sum alike, and so is the result;
    in fp16 what lies below 2^-36 of the largest is lost."""
    u = 2.0 ** -24
    tol = weight * (2 * spread[..., None] * u + 64 * u)
    if not f32:
        h = UNIT[dtype]
        tol = tol + 2 * h * weight + h * np.abs(out) + 2.0 ** -24   # fp16 results may be subnormal
    return tol + rows * 2.0 ** -35 * np.where(np.isfinite(weight), weight, 0).max(initial=1.0) + 1e-30
