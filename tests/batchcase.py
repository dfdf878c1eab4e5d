"""Plain forms of a batch's step on the CPU: tables, attention over shared prefixes and of shaped scores in 64 bits, sampling in 64 bits."""
import numpy as np
import torch

from paper_2604_26557_amd import binding as kv
from servecase import UNIT, Cache, sees


# ------------------------------------------------------------------------------------------ tables
def ref_tables(bt, lens, news, held, free, n_free, rows, leader=None, shared=None, n_tok=0):
    """(rows, held, free ids, n_free, status, tok_first, tok_seq, tok_slot) after a step, from the definition."""
    B, room = len(lens), len(rows[0])
    follows = [leader is not None and 0 <= leader[b] < B and leader[b] != b for b in range(B)]
    common = [min(shared[b], room) if follows[b] else 0 for b in range(B)]
    old, rows, now = rows, [list(r) for r in rows], list(held)
    stack, rest = list(free[:n_free]), list(free[n_free:])
    for b in range(B):
        if news[b] < 0:
            stack += old[b][common[b]:held[b]]
            rows[b], now[b] = [-1] * room, 0
    need = [-(-(n + t) // bt) if t >= 0 else 0 for n, t in zip(lens, news)]
    missing = max(0, sum(max(0, need[b] - max(held[b], common[b])) for b in range(B)) - len(stack))
    over = sum(x > room for x in need)
    pushed = list(stack)
    if not missing and not over:
        for b in range(B):
            if news[b] < 0:
                continue
            for i in range(max(held[b], common[b]), need[b]):
                rows[b][i] = stack.pop()
            now[b] = max(held[b], need[b])
        filled = [list(r) for r in rows]
        for b in range(B):
            a = leader[b] if follows[b] else -1
            for i in range(held[b], min(common[b], need[b])):
                rows[b][i] = -1 if news[a] < 0 or held[a] <= i < common[a] else filled[a][i]
    first, seq, slot = [0], [], []
    for b in range(B):
        t = max(0, news[b])
        first.append(first[-1] + t)
        seq += [b] * t
        slot += range(lens[b], lens[b] + t)
    pad = max(0, n_tok - len(seq))
    return rows, now, pushed + rest[len(pushed) - n_free:], len(stack), [missing, over], first, (seq + [-1] * pad)[:n_tok], (slot + [-1] * pad)[:n_tok]


# ------------------------------------------------------------------------------------------ attention
class Batch:
    """Sequences over a Cache, some in groups that share a prefix, with what shapes their scores."""

    def __init__(self, lens, news, H, G, D, dtype, fmt="16", layout="bhsd", bt=16, seed=0, first=(), prefix=(), trees=None, cap=0.0, slopes=None, sees_from=None, sees_to=None,
                 positions=None, scale_k=1.0):
        self.c = Cache(lens, H, D, dtype, fmt, layout, bt=bt, seed=seed, extra=max(news), n_q_heads=H * G, scale=scale_k)
        self.lens, self.news, self.H, self.G, self.D, self.dtype = list(lens), list(news), H, G, D, dtype
        self.first, self.prefix, self.trees = list(first), list(prefix), trees
        self.cap, self.slopes, self.sees_from, self.sees_to = cap, slopes, sees_from, sees_to
        self.tok_first = np.concatenate([[0], np.cumsum(news)]).astype(int).tolist()
        n = self.tok_first[-1]
        rng = np.random.default_rng(seed + 100)
        self.q = torch.from_numpy(rng.standard_normal((n, H * G, D)).astype(np.float32)).to(dtype)
        if positions is None:
            positions = []
            for b, t in enumerate(news):
                depth = kv.kv_tree_masks(trees[b])[1].tolist() if trees else range(t)
                positions += [lens[b] + d for d in depth]
        self.positions = positions

    def shared(self, b):
        """(first sequence, tokens) of sequence b's group."""
        for g, n in enumerate(self.prefix):
            if self.first[g] <= b < self.first[g + 1]:
                return self.first[g], n
        return b, 0

    def rows(self, kind, b):
        a, n = self.shared(b)
        x = self.c.seq(kind, b, self.lens[b] + self.news[b])
        return np.concatenate([self.c.seq(kind, a, n), x[:, n:]], 1) if n else x

    def dev(self, v):
        return torch.tensor(v, dtype=torch.int32, device="cuda") if v is not None else None

    def handles(self):
        i32 = self.dev
        mask = None
        if self.trees:
            words = max(1, (max(self.news) + 63) // 64)
            mask = torch.cat([kv.kv_tree_masks(p, words)[0] for p in self.trees]).cuda()
        tree = kv.tree_batch(self.tok_first, i32(self.tok_first), mask)
        groups = kv.prefix_groups(self.first, i32(self.first), self.prefix, i32(self.prefix)) if self.prefix else None
        scores = None
        if self.cap or self.slopes is not None or self.sees_from is not None or self.sees_to is not None:
            slopes = torch.tensor(self.slopes, dtype=torch.float32, device="cuda") if self.slopes is not None else None
            scores = kv.scores(self.cap, slopes, i32(self.positions) if slopes is not None else None, i32(self.sees_from), i32(self.sees_to))
        return tree, groups, scores

    def attend(self, out_dtype=kv.KV_OUT_F32, n_splits=0, ws=None, scale=0.0, out=None, q=None):
        tree, groups, scores = self.handles()
        q = self.q.cuda() if q is None else q
        if out is None:
            out = torch.full(q.shape, 7.0, dtype=torch.float32 if out_dtype == kv.KV_OUT_F32 else self.dtype, device="cuda")
        if ws is None:
            ws = torch.empty(kv.kv_group_attn_workspace(self.c.plan, self.tok_first[-1], max(self.lens)), dtype=torch.uint8, device="cuda")
        kv.kv_group_attn(self.c.plan, self.c.view, self.c.blocks, 0, tree, q, out, out_dtype, n_splits, ws, groups, scores, scale)
        return out

    def seen(self, b):
        n, t, at = self.lens[b], self.news[b], self.tok_first[b]
        m = np.zeros((t, n + t), dtype=bool)
        m[:, :n] = True
        m[:, n:] = sees(self.trees[b]) if self.trees else np.tril(np.ones((t, t), dtype=bool))
        for i in range(t):
            if self.sees_to is not None:
                m[i, :max(0, self.sees_to[at + i])] = True
            if self.sees_from is not None:
                m[i, :max(0, self.sees_from[at + i])] = False
        return m

    def expected(self, scale=None, f32=True):
        """(out, bound, sum p |v|): the definition in float64 of what the cache holds, and how far 32-bit arithmetic may be from it, token by token.  A score is a sum of D products (D + 8 roundings
        of it), its cap is off by 6 units of 2^-24, with 16-bit
        results and caps up to 64 by 8 units times the cap (2 cap / (1 + e): a quarter of 2 units of the exponential, one of the sum, 2 of the reciprocal), a bias by 8 of the distance's (4 operations, and 64 tokens more from which a group of rows counts), the exponent's argument by 4 of the
        largest and its own; what that changes of a weight changes numerator and sum.  Sums of rows over 64 wavefronts and splits add 64 units."""
        scale = scale or self.D ** -0.5
        q, u = self.q.double().numpy(), 2.0 ** -24
        out, tol, weight = np.zeros(q.shape), np.zeros(q.shape), np.zeros(q.shape)
        for b, t in enumerate(self.news):
            if t == 0:
                continue
            k, v, m, at = self.rows("k", b), self.rows("v", b), self.seen(b), self.tok_first[b]
            key_pos = np.concatenate([np.arange(self.lens[b]), self.positions[at:at + t]])
            for i in range(t):
                idx = np.flatnonzero(m[i])
                if len(idx) == 0:
                    continue
                for h in range(self.H * self.G):
                    kk, vv, x0 = k[h // self.G][idx], v[h // self.G][idx], q[at + i, h]
                    x = (kk @ x0) * scale
                    e = (np.abs(kk) @ np.abs(x0)) * abs(scale) * (self.D + 8)
                    if self.cap:
                        x = self.cap * np.tanh(x / self.cap)
                        e = e + (8 * self.cap if not f32 and self.cap <= 64 else 6 * np.abs(x))
                    if self.slopes is not None:
                        dist = np.abs(self.positions[at + i] - key_pos[idx])
                        x = x - self.slopes[h] * dist
                        e = e + 8 * abs(self.slopes[h]) * (dist + 64)
                    e = e + 4 * np.abs(x) + 4 * np.abs(x).min() + 8
                    with np.errstate(all="ignore"):
                        p = np.exp(x - x.max())
                        p = p / p.sum()
                        out[at + i, h], weight[at + i, h] = p @ vv, p @ np.abs(vv)
                        tol[at + i, h] = u * (2 * ((p * e) @ np.abs(vv) + (p @ e) * (p @ np.abs(vv))) + 64 * (p @ np.abs(vv))) + len(idx) * 2.0 ** -35 * np.abs(vv).max(initial=1.0)
        return out, tol + 1e-30, weight

    def check(self, got, f32=True, scale=None):
        out, tol, weight = self.expected(scale, f32)
        g = got.double().cpu().numpy()
        if not f32:   # what the parts of a probability lose, in numerator and sum, and one rounding
            tol = tol + 2 * (2.0 ** -22 if self.dtype == torch.float16 else 2.0 ** -16) * weight
            tol = tol * (1 + UNIT[self.dtype]) + UNIT[self.dtype] * np.abs(out) + 2.0 ** -25
        assert np.isfinite(g).all()
        err = np.abs(g - out)
        assert (err <= tol).all(), (float(err.max()), float((err / tol).max()), np.unravel_index((err / tol).argmax(), err.shape))


# ------------------------------------------------------------------------------------------ sampling
def ref_sample(x, t=1.0, k=0, p=1.0, m=0.0, u=0.0):
    """(token, probability) of one row of float64 logits; k, p, m, u as 32 bits hold them."""
    if np.isnan(x).any() or np.isposinf(x).any() or not np.isfinite(x).any():
        return -1, 0.0
    if not t > 0:
        return int(np.flatnonzero(x == x.max())[0]), 1.0
    with np.errstate(all="ignore"):
        w = np.where(np.isneginf(x), 0.0, np.exp((x - x.max()) / t))
    order = np.lexsort((np.arange(len(x)), -x))
    if 0 < k < len(x):
        order = order[:k]
    if p < 1:
        sums = np.cumsum(w[order])
        order = order[:int((sums < max(p, 0.0) * sums[-1]).sum()) + 1]
    order = np.sort(order[w[order] >= min(m, 1.0)])
    sums = np.cumsum(w[order])
    i = min(int((sums <= min(max(u, 0.0), 1.0) * sums[-1]).sum()), int(np.flatnonzero(w[order] > 0)[-1]))
    return int(order[i]), float(w[order[i]] / sums[-1])
