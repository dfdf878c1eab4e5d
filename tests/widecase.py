"""Batches whose calls of kv_group_attn take the kernels of 32 and 64 query rows a workgroup, and the one with prefixes of many rows beside sequences of few: which, test_group_paths_cpu.py checks
without a GPU.  The definition in 64 bits for all rows of a head at once."""
import numpy as np
import torch

from batchcase import Batch
from paper_2604_26557_amd import binding as kv
from servecase import UNIT, random_parents


def make(H, G, n_splits, B, t, own, P=0, Q=0, step=5):
    """B sequences of up to t new tokens, the third of none if t > 1, and up to `own` of their own; behind a prefix of P tokens all but the last one, or behind one of P and one of Q the halves of all but the first."""
    news = [max(0 if t > 1 else 1, t - i * step % (t // 2 + 2)) for i in range(B)]
    if t > 1:
        news[2] = 0
    m = B // 2
    if not P:
        lens, first, prefix = [i * 37 % own for i in range(B)], [], []
    elif Q:
        lens, first, prefix = [5] + [P + i * 7 % own for i in range(1, m)] + [Q + i * 11 % own for i in range(m, B)], [1, m, B], [P, Q]
    else:
        lens, first, prefix = [P + i * 7 % own for i in range(B - 1)] + [17], [0, B - 1], [P]
    return dict(H=H, G=G, n_splits=n_splits, lens=lens, news=news, first=first, prefix=prefix)


# (head_dim, path, row groups of a workgroup, of a prefix' workgroup): heads that are no power of two; heads that are, whose slopes stay with their lanes
SHAPES = {
    (64, "none", 2, 2): (make(7, 7, 0, 33, 5, 10), make(8, 16, 2, 33, 3, 10)),
    (64, "none", 4, 4): (make(5, 6, 1, 66, 9, 10), make(8, 16, 2, 20, 9, 10)),
    (64, "apart", 1, 4): (make(7, 7, 5, 66, 1, 10, 100, 41), make(5, 16, 5, 66, 1, 45, 100, 41)),
    (64, "apart", 2, 2): (make(5, 3, 5, 9, 17, 10, 100, 41), make(3, 8, 5, 13, 9, 10, 100, 77)),
    (64, "apart", 4, 4): (make(12, 3, 5, 9, 17, 45, 100, 41), make(2, 16, 5, 13, 17, 45, 100, 41)),
    (64, "joined", 2, 2): (make(5, 7, 0, 9, 30, 10, 100, 77), make(7, 8, 0, 9, 17, 10, 100, 77)),
    (64, "joined", 4, 4): (make(8, 7, 0, 20, 17, 10, 100, 77), make(7, 8, 0, 13, 30, 10, 100, 77)),
    (128, "none", 2, 2): (make(8, 6, 5, 33, 5, 10), make(5, 16, 1, 13, 9, 10)),
    (128, "none", 4, 4): (make(16, 7, 0, 20, 9, 10), make(12, 16, 0, 13, 9, 10)),
    (128, "apart", 1, 4): (make(16, 5, 5, 33, 1, 10, 100, 77), make(3, 16, 5, 66, 1, 90, 100, 41)),
    (128, "apart", 2, 2): (make(2, 7, 5, 13, 9, 10, 100, 150), make(2, 16, 5, 13, 5, 90, 100, 77)),
    (128, "apart", 4, 4): (make(6, 3, 5, 9, 30, 90, 100, 77), make(7, 8, 5, 9, 17, 10, 100, 41)),
    (128, "joined", 2, 2): (make(3, 5, 0, 33, 17, 10, 100, 41), make(12, 16, 0, 9, 9, 10, 100, 41)),
    (128, "joined", 4, 4): (make(8, 6, 0, 20, 17, 45, 100, 41), make(3, 8, 0, 33, 30, 10, 100, 41)),
    (256, "none", 2, 2): (make(8, 6, 1, 33, 5, 10), make(8, 16, 0, 9, 9, 10)),
    (256, "apart", 1, 2): (make(5, 7, 5, 33, 3, 10, 100, 77), make(16, 16, 5, 13, 1, 10, 100, 41)),
    (256, "apart", 2, 2): (make(8, 6, 5, 9, 5, 45, 100, 77), make(3, 4, 5, 9, 30, 90, 203, 41)),
    (256, "joined", 2, 2): (make(3, 5, 0, 33, 17, 10, 203, 150), make(5, 8, 0, 13, 17, 10, 100)),
}
# head_dim 256 in 8 bits: an LDS of its own size
EIGHT_BITS = {(256, "apart", 1, 2): (make(1, 14, 0, 65, 1, 500, 1500),) * 2}
WIDTHS = {"16": 16, "fp8": 8, "fp4": 4}


def shape_of(key, fmt, pow2):
    return (EIGHT_BITS if fmt == "fp8" and key in EIGHT_BITS else SHAPES)[key][pow2]


def path_line(D, fmt, layout, chain, bounded, shaped, s):
    """A line of group_path_harness.cpp's input."""
    v = s["lens"] + s["news"] + (s["first"] or [0]) + s["prefix"]
    return (f"{D} {s['H']} {s['G']} {WIDTHS[fmt]} {int(layout == 'paged')} {int(chain)} {int(bounded)} {int(shaped)} {s['n_splits']} {len(s['lens'])} {len(s['prefix'])} "
            + " ".join(map(str, v)) + "\n")


def slopes_of(n):
    return [float(np.float32(2.0 ** (-8 * (i + 1) / n))) for i in range(n)]


class Wide(Batch):
    def __init__(self, D, s, dtype, fmt, layout, seed=0, tree=False, bt=16):
        self.splits, self.kept = s["n_splits"], {}
        rng = np.random.default_rng(seed + 1)
        super().__init__(s["lens"], s["news"], s["H"], s["G"], D, dtype, fmt, layout, bt=bt, seed=seed, first=s["first"], prefix=s["prefix"],
                         trees=[random_parents(rng, n) for n in s["news"]] if tree else None)

    def shape(self, cap=0.0, slopes=False, window=0):
        """What is asked of the scores, from now on."""
        at = [n + i for n, t in zip(self.lens, self.news) for i in range(t)]
        self.cap, self.slopes = cap, slopes_of(self.H * self.G) if slopes else None
        self.sees_from = [max(0, j - window + 1) for j in at] if window else None
        return self

    def run(self, out_dtype=kv.KV_OUT_F32):
        return self.attend(out_dtype, self.splits)

    def rows(self, kind, b):
        if (kind, b) not in self.kept:
            self.kept[kind, b] = super().rows(kind, b)
        return self.kept[kind, b]

    def expected(self, scale=None, f32=True):
        """(out, bound, sum p |v|), as Batch.expected but for what follows.  The error e of an exponent's argument, in units of 2^-24: D products and their sum (D + 8 times the sum of their magnitudes); a
        cap's 6 units of its result, or 8 of the cap by sigmoids; a bias' 8 of its own and of 64 tokens'; the roundings of the argument and of its reference, 4 of each at most, and 8 of the exponential's.
        A weight is off by e of itself, which counts in numerator and sum; parts of probabilities lose 2^-22 of them (fp16) or, with bf16 results, 2^-16; sums over wavefronts, splits and a step's
        products 64 units and one for every 32 tokens more; what of fp16 lies below 2^-36 of the largest, twice that for each token."""
        scale = scale or self.D ** -0.5
        u = 2.0 ** -24
        q = self.q.double().numpy()
        out, tol, weight = np.zeros(q.shape), np.zeros(q.shape), np.zeros(q.shape)
        lost = 2.0 ** -22 if self.dtype == torch.float16 else 0.0 if f32 else 2.0 ** -16
        for b, t in enumerate(self.news):
            if t == 0:
                continue
            k, v, m, at = self.rows("k", b), self.rows("v", b), self.seen(b), self.tok_first[b]
            key_pos = np.concatenate([np.arange(self.lens[b]), self.positions[at:at + t]])
            m = np.repeat(m, self.G, 0)
            dist = np.repeat(np.abs(np.asarray(self.positions[at:at + t])[:, None] - key_pos[None]), self.G, 0)
            for h in range(self.H):
                x0 = q[at:at + t, h * self.G:(h + 1) * self.G].reshape(t * self.G, self.D)
                x = x0 @ k[h].T * scale
                e = np.abs(x0) @ np.abs(k[h]).T * abs(scale) * (self.D + 8)
                if self.cap:
                    x = self.cap * np.tanh(x / self.cap)
                    e = e + (8 * self.cap if not f32 and self.cap <= 64 else 6 * np.abs(x))
                if self.slopes is not None:
                    slope = np.tile(np.abs(self.slopes[h * self.G:(h + 1) * self.G]), t)[:, None]
                    x = x - np.tile(self.slopes[h * self.G:(h + 1) * self.G], t)[:, None] * dist
                    e = e + 8 * slope * (dist + 64)
                none = ~m.any(1)
                top = np.where(none, 0, np.where(m, x, -np.inf).max(1, initial=-np.inf))[:, None]
                e = e + 4 * np.abs(x) + 4 * np.abs(top) + 8
                p = np.where(m, np.exp(np.minimum(x - top, 0)), 0)
                p = p / np.where(none, 1, p.sum(1))[:, None]
                av, to = np.abs(v[h]), (slice(at, at + t), slice(h * self.G, (h + 1) * self.G))
                w = p @ av
                back = lambda y: y.reshape(t, self.G, self.D)  # noqa: E731
                out[to], weight[to] = back(p @ v[h]), back(w)
                tol[to] = back(u * (2 * ((p * e) @ av + (p * e).sum(1)[:, None] * w) + (64 + m.shape[1] / 32) * w) + 2 * lost * w + m.sum(1)[:, None] * 2.0 ** -35 * av.max(initial=1.0))
        return out, tol + 1e-30, weight

    def check(self, got, f32=True, scale=None, rows=None):
        """rows: of the tokens, those that are looked at."""
        out, tol, _ = self.expected(scale, f32)
        if not f32:   # one rounding
            tol = tol * (1 + UNIT[self.dtype]) + UNIT[self.dtype] * np.abs(out) + 2.0 ** -25
        g = got.double().cpu().numpy()
        if rows is not None:
            g, out, tol = g[rows], out[rows], tol[rows]
        assert np.isfinite(g).all()
        err = np.abs(g - out)
        assert (err <= tol).all(), (float(err.max()), float((err / tol).max()), np.unravel_index((err / tol).argmax(), err.shape))
