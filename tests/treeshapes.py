"""Batches whose attention kv_tree_attn does with 32 or 64 query rows a workgroup, and their plain 64-bit form."""
import numpy as np
import torch

from paper_2604_26557_amd import binding as kv
from servecase import Cache

# (head_dim, row groups of 16): (KV heads, query heads of each, contexts, drafted tokens, numbers of splits to ask for).  On 256 compute units the cut takes that many row groups for each, in every
# format and layout and whatever the results' type.  Last row blocks of 1 to 64 rows, sequences without context or drafted tokens, several steps of each wavefront.
SHAPES = {
    (64, 2): [(3, 5, [167, 715, 291, 375, 37, 958, 490], [56, 7, 64, 39, 44, 0, 64], (0, 1)), (4, 5, [495] * 7, [29] * 7, (0, 1)),
              (4, 7, [584, 90, 44, 292, 40, 1035, 1327], [0, 24, 28, 30, 25, 26, 1], (2,))],
    (64, 4): [(4, 7, [819, 271, 908, 8, 349, 958], [0, 57, 0, 92, 84, 53], (0, 1)), (4, 7, [436] * 6, [50] * 6, (0, 1)),
              (3, 3, [676, 502, 796, 798, 472, 270, 351, 1043], [42, 82, 87, 70, 98, 0, 64, 26], (2,))],
    (128, 2): [(3, 3, [1205, 281, 36, 139, 539, 509], [0, 100, 89, 98, 66, 100], (0, 1)), (4, 3, [1989] * 6, [12] * 6, (0,)),
               (3, 7, [670, 957, 319, 497, 305, 946], [19, 0, 30, 30, 25, 18], (2,))],
    (128, 4): [(4, 7, [144, 168, 464, 913, 206, 102, 553], [100, 20, 0, 66, 91, 64, 0], (0, 1)), (2, 7, [427] * 6, [100] * 6, (0, 1)),
               (2, 7, [61, 1002, 661, 632, 415, 899, 0], [100, 0, 0, 17, 100, 100, 57], (2,))],
    (256, 2): [(3, 4, [302, 789, 613, 632, 48, 4, 386], [99, 0, 0, 21, 100, 100, 100], (0, 1)), (2, 4, [410] * 7, [73] * 7, (0, 1)),
               (3, 2, [777, 50, 240, 895, 1072, 414, 55, 1, 920], [0, 0, 100, 100, 0, 100, 100, 64, 0], (2,))],
}


def without_a_context(shape):
    """The batch, the context of one sequence taken away (the shortest with 10 drafted tokens or more), and that sequence."""
    H, G, lens, drafted, splits = shape
    b = lens.index(min(n for n, t in zip(lens, drafted) if t >= 10))
    return (H, G, lens[:b] + [0] + lens[b + 1:], drafted, splits), b


# name, block tokens (0: strided), rows of a head apart
LAYOUTS = [("bhsd", 0, False), ("paged", 16, False), ("paged", 48, False), ("paged", 5, False), ("bhsd", 0, True)]


def decode(codes, scale, fmt):
    """Values of codes and scale bytes in 64 bits: e4m3 and e2m1 by their definitions."""
    if fmt == "fp8":
        e, m = (codes >> 3 & 15).double(), (codes & 7).double()
        x = torch.where(e == 0, m * 2.0 ** -9, (8 + m) * torch.exp2(e - 10)) * torch.where(codes >= 128, -1.0, 1.0)
    else:
        codes = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
        x = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64)[(codes & 7).long()] * torch.where(codes >= 8, -1.0, 1.0)
    return x * torch.exp2(scale.double() - 127).repeat_interleave(32, -1)


class WideCache(Cache):
    """Random codes and scales (or 16-bit rows) in any layout; `values` are float64 on the device, in the cache's own order."""

    def __init__(self, lens, H, D, G, dtype, fmt, layout, extra, seed):
        name, bt, apart = layout
        self.fmt, self.layout, self.lens, self.dtype, self.D, self.H, self.bt = fmt, name, list(lens), dtype, D, H, bt
        gen = torch.Generator().manual_seed(seed)
        B, self.rows = len(lens), max(lens) + extra
        shape = (B, H, self.rows)
        if bt:
            per = [-(-(n + extra) // bt) for n in lens]
            ids = torch.randperm(sum(per) + 2, generator=gen).tolist()
            self.table_host = np.full((B, max(per)), -1, dtype=np.int32)
            at = 0
            for b, n in enumerate(per):
                self.table_host[b, :n] = ids[at:at + n]
                at += n
            self.table = torch.from_numpy(self.table_host).cuda()
            shape = (len(ids), H, bt)
        self.dev, self.values = {}, {}
        for kind in "kv":
            if fmt == "16":
                rows = torch.randn(shape + (D,), generator=gen).to(dtype)
                self.values[kind] = rows.double().cuda()
            else:
                if fmt == "fp8":
                    rows = torch.randn(shape + (D,), generator=gen).mul_(60).clamp_(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
                    scale = torch.randint(119, 123, shape + (D // 32,), generator=gen, dtype=torch.uint8)
                else:
                    rows = torch.randint(0, 256, shape + (D // 2,), generator=gen, dtype=torch.uint8)
                    scale = torch.randint(123, 127, shape + (D // 32,), generator=gen, dtype=torch.uint8)
                self.values[kind] = decode(rows, scale, fmt).cuda()
                self.dev[kind + "_scale"] = scale.cuda()
            if apart:   # every other row of a buffer of them
                rows = torch.stack([rows, torch.full_like(rows, 0x7f)], 3).cuda()[:, :, :, 0]
            self.dev[kind] = rows.cuda()
        self.plan = kv.kv_layout_plan(1, H, H * G, D, [self.rows] * B, kv.KV_F16 if dtype == torch.float16 else kv.KV_BF16, 512, 4096, kv.KV_PER_SEQ)
        self.lens_dev = torch.tensor(self.lens, dtype=torch.int32, device="cuda")
        self.remake()

    def seq64(self, kind, b, n):
        """[H, n, D] of sequence b."""
        x = self.values[kind]
        if not self.bt:
            return x[b, :, :n]
        ids = torch.from_numpy(self.table_host[b, :-(-n // self.bt)]).long().cuda()
        return x[ids].transpose(0, 1).flatten(1, 2)[:, :n]

    def expected64(self, q, masks):
        """(out, sum p |v|, largest error of an exponent per 2^-24), as servecase's ref_attention has them; masks: [T, T] of each sequence."""
        outs, at, G = [], 0, q.shape[1] // self.H
        scale = self.D ** -0.5
        for b, m in enumerate(masks):
            T, n = len(m), self.lens[b]
            if T == 0:
                continue
            k, v = self.seq64("k", b, n + T), self.seq64("v", b, n + T)
            sees = torch.ones((T, n + T), dtype=torch.bool)
            sees[:, n:] = torch.from_numpy(np.ascontiguousarray(m))
            sees = sees.cuda().repeat_interleave(G, 0)
            res = [torch.zeros((T, self.H, G, x), dtype=torch.float64, device="cuda") for x in (self.D, self.D, 1)]
            for h in range(self.H):
                rows = q[at:at + T, h * G:(h + 1) * G].double().flatten(0, 1)
                s = torch.mm(rows, k[h].T.contiguous()) * scale
                top = s.masked_fill(~sees, -torch.inf).amax(1, keepdim=True)
                some = top != -torch.inf
                p = torch.where(sees & some, (s - torch.where(some, top, 0.0)).exp(), 0.0)
                p = p / p.sum(1, keepdim=True).clamp(min=1e-300)
                size = torch.mm(rows.abs(), k[h].abs().T.contiguous()).masked_fill(~sees, 0.0).amax(1, keepdim=True) * scale
                spread = size * (self.D + 8) + s.abs().masked_fill(~sees, 0.0).amax(1, keepdim=True) + 8
                for to, x in zip(res, (torch.mm(p, v[h].contiguous()), torch.mm(p, v[h].abs().contiguous()), spread)):
                    to[:, h] = x.unflatten(0, (T, G))
            outs.append([x.flatten(1, 2) for x in res])
            at += T
        out, weight, spread = (torch.cat([o[i] for o in outs]).cpu().numpy() for i in range(3))
        return out, weight, spread[..., 0]


def words_of(masks):
    """[n_tok, words] as kv_tree_attn takes them."""
    words = max(1, -(-max(len(m) for m in masks) // 64))
    out = np.zeros((sum(len(m) for m in masks), words), dtype=np.uint64)
    at = 0
    for m in masks:
        for i, j in zip(*np.nonzero(m)):
            out[at + i, j // 64] |= np.uint64(1) << np.uint64(j % 64)
        at += len(m)
    return torch.from_numpy(out.view(np.int64)).cuda()
