"""A batch's step against plain forms: block tables and slot maps, sampling, and the operators together."""
import random

import numpy as np
import pytest
import torch

from batchcase import Batch, ref_sample, ref_tables
from paper_2604_26557_amd import binding as kv

pytestmark = pytest.mark.gpu


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


# ------------------------------------------------------------------------------------------ tables
def requests(rnd, B, bt, longest, most_new, ended=0.2, begun=0.2, prefix=0):
    """Requests as earlier steps left them: blocks that are held are different ones."""
    lens, news, held, leader, shared, rows = [], [], [], [], [], []
    for b in range(B):
        follows = b > 0 and prefix > 0 and rnd.random() < 0.5
        leader.append(rnd.choice([0, 0, 0, b, B + 3]) if follows else rnd.choice([-1, -5]))
        shared.append(prefix)
        own = prefix if leader[b] == 0 and follows else 0
        n = max(rnd.randint(0, longest), prefix * bt if b == 0 else 0)
        if b > 0 and rnd.random() < begun:
            n, h = own * bt, 0
        else:
            n = max(n, own * bt)
            h = max(-(-n // bt) + rnd.choice([0, 0, 1]), own)
        lens.append(n)
        held.append(h)
        news.append(-1 if b > 0 and rnd.random() < ended else rnd.randint(0, most_new))
    room = max(max(held), max(-(-(n + max(t, 0)) // bt) for n, t in zip(lens, news))) + rnd.choice([0, 2])
    room = max(room, 1)
    at = 0
    for b in range(B):
        own = prefix if leader[b] == 0 and b > 0 and held[b] else 0
        row = (rows[0][:own] if own else []) + list(range(at, at + held[b] - own))
        at += held[b] - own
        rows.append(row + [-1] * (room - len(row)))
    return lens, news, held, leader, shared, rows, at


def run_tables(case, bt, free, n_free, n_tok, in_place, lead=True, stream=None):
    lens, news, held, leader, shared, rows = case
    B = len(lens)
    t = dict(held=i32(held), n_free=i32([n_free]), block_table=i32(rows))
    free_dev, first, seq, slot, status = i32(free), i32([7] * (B + 1)), i32([7] * n_tok), i32([7] * n_tok), i32([7, 7])
    outs = t if in_place else {k: torch.full_like(v, 99) for k, v in t.items()}
    more = {} if in_place else {k + "_out": v for k, v in outs.items()}
    if lead:
        more.update(leader=i32(leader), shared=i32(shared))
    before = {k: v.clone() for k, v in t.items()}
    kv.kv_step_tables(kv.step_tables(bt, i32(lens), i32(news), t["held"], free_dev, t["n_free"], t["block_table"], first, seq, slot, status, **more), stream)
    torch.cuda.synchronize()
    if not in_place:
        assert all(torch.equal(t[k], before[k]) for k in t)
    return [outs["block_table"].tolist(), outs["held"].tolist(), free_dev.tolist(), int(outs["n_free"]), status.tolist(), first.tolist(), seq.tolist(), slot.tolist()]


NAMES = ("rows", "held", "free", "n_free", "status", "tok_first", "tok_seq", "tok_slot")


def same_tables(got, want):
    for n, x, y in zip(NAMES, got, want):
        assert x == y, n


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("B,bt,longest,most_new,prefix", [(1, 16, 100, 1, 0), (1, 1, 3, 0, 0), (5, 16, 300, 40, 3), (64, 16, 4000, 1, 32), (63, 7, 90, 9, 2), (200, 32, 9000, 700, 5),
                                                          (1000, 16, 64, 5, 1), (1025, 8, 40, 3, 2), (8192, 16, 100, 2, 0), (3, 4, 9000, 5, 0)])
def test_tables(in_place, B, bt, longest, most_new, prefix):
    for seed in range(3):
        rnd = random.Random(1000 * B + seed)
        *case, at = requests(rnd, B, bt, longest, most_new, prefix=prefix)
        spare = sum(-(-(n + max(t, 0)) // bt) for n, t in zip(case[0], case[1])) + 3
        ids = list(range(at, at + spare))
        rnd.shuffle(ids)
        free, total = ids + [-7] * at, sum(max(0, t) for t in case[1])
        for n_tok, lead in ((total, True), (total + 77, prefix == 0), (max(0, total - 5), True)):
            lead = lead or prefix > 0
            want = ref_tables(bt, *case[:2], case[2], free, spare, case[5], *(case[3:5] if lead else ()), n_tok=n_tok)
            assert want[4] == [0, 0]
            same_tables(run_tables(case, bt, free, spare, n_tok, in_place, lead), want)


@pytest.mark.parametrize("in_place", [False, True])
def test_tables_take_what_has_just_ended(in_place):
    """Free blocks run out: what ends in a call is handed out in it, from the last one on; one block fewer and nobody gets any."""
    lens, news, held = [40, 33, 64, 10], [-1, 16, -1, 40], [3, 3, 5, 1]
    rows = [[1, 2, 3, -1, -1], [4, 5, 6, -1, -1], [7, 8, 9, 10, 11], [12, -1, -1, -1, -1]]
    for n_free, fits in ((0, True), (1, True)):
        free = [20] * n_free + [-1] * (16 - n_free)
        case = (lens, news, held, None, None, rows)
        want = ref_tables(16, lens, news, held, free, n_free, rows, n_tok=60)
        same_tables(run_tables(case, 16, free, n_free, 60, in_place, False), want)
        assert want[0][1][:4] == [4, 5, 6, 11] and want[0][3][:4] == [12, 10, 9, 8] and want[0][0] == [-1] * 5
    # 9 wanted, 8 there
    news = [-1, 60, -1, 40]
    rows9 = [r + [-1] for r in rows]
    case = (lens, news, held, None, None, rows9)
    news_more = [-1, 60, -1, 85]
    want = ref_tables(16, lens, news_more, held, [-1] * 16, 0, rows9, n_tok=3)
    assert want[4][0] == 0
    tight = [40, 33, 64, 10], [-1, 60, -1, 86], held, None, None, rows9
    want = ref_tables(16, *tight[:3], [-1] * 16, 0, rows9, n_tok=3)
    assert want[4] == [0, 0]
    for extra in (100, 101):
        case = ([40, 33, 64, 10], [-1, extra - 40, -1, 86], held, None, None, [r + [-1] * 6 for r in rows9])
        want = ref_tables(16, *case[:3], [-1] * 16, 0, case[5], n_tok=3)
        same_tables(run_tables(case, 16, [-1] * 16, 0, 3, in_place, False), want)


@pytest.mark.parametrize("in_place", [False, True])
def test_tables_when_blocks_are_missing_or_rows_too_short(in_place):
    """Nothing is handed out, what ended is released, and the maps are written all the same."""
    lens, news, held, rows = [16, 30, 5], [1, 200, -1], [1, 2, 1], [[3, -1, -1], [4, 5, -1], [6, -1, -1]]
    case = (lens, news, held, None, None, rows)
    want = ref_tables(16, lens, news, held, [9, 8, -1, -1], 2, rows, n_tok=201)
    assert want[4][1] == 1 and want[1] == [1, 2, 0] and want[2] == [9, 8, 6, -1] and want[3] == 3
    same_tables(run_tables(case, 16, [9, 8, -1, -1], 2, 201, in_place, False), want)
    rows = [r + [-1] * 20 for r in rows]
    case = (lens, news, held, None, None, rows)
    want = ref_tables(16, lens, news, held, [9, 8, -1, -1], 2, rows, n_tok=201)
    assert want[4] == [1 + 13 - 3, 0] and want[0][0][1] == -1
    same_tables(run_tables(case, 16, [9, 8, -1, -1], 2, 201, in_place, False), want)


@pytest.mark.parametrize("in_place", [False, True])
def test_tables_of_numbers_out_of_range(in_place):
    """Lengths, counts and held blocks that no program means: nothing is read or written outside, and what is right stays right."""
    B, room, big = 6, 4, 2 ** 31 - 1
    guard = 64
    held, n_free = i32([big, -9, 2, 1, 0, 3]), i32([big])
    buf = torch.full((guard + B * room + guard,), 77, dtype=torch.int32, device="cuda")
    table = buf[guard:guard + B * room].view(B, room)
    table.fill_(-1)
    free = i32([5, 6, 7])
    outs = {} if in_place else dict(held_out=torch.zeros_like(held), n_free_out=torch.zeros_like(n_free), block_table_out=table.clone())
    first, seq, slot, status = i32([0] * 7), i32([3] * 10), i32([3] * 10), i32([3, 3])
    t = kv.step_tables(16, i32([big, -5, 10, 20, 0, 7]), i32([big, 1, -big, 2, big, 0]), held, free, n_free, table, first, seq, slot, status, leader=i32([big, -1, 0, 3, 9, 2]),
                       shared=i32([big, 2, big, 1, -4, 1]), **outs)
    kv.kv_step_tables(t)
    torch.cuda.synchronize()
    assert status.tolist()[1] == 2 and (buf[:guard] == 77).all() and (buf[guard + B * room:] == 77).all()
    assert first.tolist()[-1] == big and seq.tolist() == [0] * 10
    # one sequence of no length in a table without entries
    none = i32([]).view(1, 0)
    status.fill_(3)
    kv.kv_step_tables(kv.step_tables(16, i32([0]), i32([0]), i32([0]), i32([]), i32([0]), none, i32([5, 5]), i32([]), i32([]), status))
    assert status.tolist() == [0, 0]


def test_tables_leaders():
    """A leader that begins with its followers, one that ends, and one that follows somebody itself."""
    lens, news = [48, 48, 48, 48, 48], [1, 1, 1, -1, 1]
    held, leader, shared = [0, 0, 0, 4, 0], [-1, 0, 1, -1, 3], [0, 3, 2, 0, 2]
    rows = [[-1] * 4, [-1] * 4, [-1] * 4, [40, 41, 42, 43], [-1] * 4]
    for in_place in (False, True):
        case = (lens, news, held, leader, shared, rows)
        free = list(range(10, 30)) + [0] * 10
        want = ref_tables(16, lens, news, held, free, 20, rows, leader, shared, n_tok=4)
        got = run_tables(case, 16, free, 20, 4, in_place)
        same_tables(got, want)
        assert got[0][1][:3] == got[0][0][:3] and got[0][2][:2] == [-1, -1] and got[0][4][:2] == [-1, -1] and got[0][0][0] == 43


# ------------------------------------------------------------------------------------------ sampling
def sample(x, u, **kw):
    """x: [B, V] on the device; the others lists or numbers."""
    B = x.shape[0]
    dev = lambda v, t: torch.tensor([v] * B if not isinstance(v, (list, np.ndarray)) else list(v), dtype=t, device="cuda")  # noqa: E731
    a = dict(temperature=dev(kw["t"], torch.float32) if "t" in kw else None, top_k=dev(kw["k"], torch.int32) if "k" in kw else None,
             top_p=dev(kw["p"], torch.float32) if "p" in kw else None, min_p=dev(kw["m"], torch.float32) if "m" in kw else None)
    tokens, probs = i32([-9] * B), torch.full((B,), 9.0, device="cuda")
    ws = torch.empty(kv.kv_sample_workspace(*x.shape), dtype=torch.uint8, device="cuda").fill_(171)
    kv.kv_sample(x, dev(u, torch.float32), tokens, ws, probs=probs, **a)
    return tokens.tolist(), probs.double().tolist()


def check_sample(x, u, **kw):
    tokens, probs = sample(x, u, **kw)
    rows = x.double().cpu().numpy()
    of = lambda n, b: float(np.float32(kw[n][b] if isinstance(kw[n], (list, np.ndarray)) else kw[n]))  # noqa: E731
    for b in range(x.shape[0]):
        more = {n: of(n, b) for n in ("t", "p", "m") if n in kw}
        token, prob = ref_sample(rows[b], k=int(of("k", b)) if "k" in kw else 0, u=float(np.float32(u[b])), **more)
        assert tokens[b] == token, (b, more, u[b], tokens[b], token)
        # 53-bit arithmetic, weights in the sum off by half a unit of at most 2^-38 each, and a rounding to 24 bits
        assert abs(probs[b] - prob) <= 2.0 ** -23 * prob + x.shape[1] * 2.0 ** -39, (b, probs[b], prob)


CUTS = [dict(), dict(t=0.7), dict(k=1), dict(k=5), dict(k=50, t=1.4), dict(p=0.9), dict(p=0.3, t=0.5), dict(m=0.05), dict(k=40, p=0.8), dict(k=100, p=0.95, m=0.02, t=1.2), dict(t=0.0),
        dict(p=0.0), dict(p=1.0, k=0, m=0.0), dict(k=10 ** 6, p=0.999), dict(m=1.0), dict(t=30.0, p=0.5), dict(t=0.01, k=3)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("V", [1, 2, 63, 64, 65, 257, 1000, 4097, 32003])
def test_sample(dtype, V):
    gen = torch.Generator().manual_seed(V)
    B = 6
    x = (torch.randn((B, V), generator=gen) * 2.5).to(dtype)
    x[1] = x[1] * 8          # a few carry all
    x[2] = x[2] * 0.1        # flat
    x[3, ::2] = float("-inf") if V > 1 else x[3, ::2]
    x[4] = torch.round(x[4].float()).to(dtype)   # ties by the hundred
    x = x.cuda()
    for i, kw in enumerate(CUTS):
        u = np.random.default_rng(i).random(B)
        check_sample(x, u, **kw)
    check_sample(x, [0.0, 1.0 - 2.0 ** -24, 0.5, 1.0, 0.25, 0.9999], t=[0.5, 1.0, 0.0, 2.0, 1.0, 0.1], k=[0, 3, 5, 7, -1, 2], p=[1.0, 0.5, 0.9, 1.0, 0.2, 0.99], m=[0.1, 0.0, 0.0, 0.5, 0.0, 0.01])


def test_sample_large_vocabularies():
    gen = torch.Generator().manual_seed(5)
    for V, dtype in ((151937, torch.bfloat16), (300001, torch.float32), ((1 << 20) + 3, torch.float16)):
        x = (torch.randn((3, V), generator=gen) * 2).to(dtype).cuda()
        for kw in (dict(), dict(p=0.95), dict(k=1000, p=0.9), dict(k=V - 1), dict(m=0.001, t=2.0)):
            check_sample(x, [0.1, 0.6, 0.99], **kw)


def test_sample_of_equal_logits():
    """Everything ties: the first ones by index are kept."""
    for V in (10, 5000):
        x = torch.full((4, V), -3.5, dtype=torch.float16, device="cuda")
        check_sample(x, [0.0, 0.5, 0.75, 0.999])
        check_sample(x, [0.0, 0.5, 0.75, 0.999], k=7)
        check_sample(x, [0.0, 0.5, 0.75, 0.999], p=0.5, k=8)
        assert max(sample(x, [0.0, 0.5, 0.75, 0.999], k=7)[0]) == 6
    # +0 and -0 are equal
    x = torch.zeros((1, 64), device="cuda")
    x[0, ::2] = -0.0
    assert sample(x, [0.99], k=3)[0] == [2] and sample(x, [0.5], t=0.0)[0] == [0]


def test_sample_rows_without_an_answer():
    x = torch.randn((7, 300), device="cuda")
    x[0] = float("-inf")
    x[1, 5] = float("nan")
    x[2, 299] = float("inf")
    x[3] = float("nan")
    x[5, 1:] = float("-inf")
    x[6] = -3.0e38
    tokens, probs = sample(x, [0.5] * 7, k=20, p=0.9)
    assert tokens[:4] == [-1] * 4 and probs[:4] == [0.0] * 4
    assert tokens[5] == 0 and probs[5] == 1.0
    check_sample(x[4:], [0.5] * 3, k=20, p=0.9)
    check_sample(x[4:], [0.5] * 3)
    assert sample(x, [0.5] * 7, t=0.0)[0][:4] == [-1] * 4


def test_sample_odd_parameters():
    """Temperatures that leave no range, numbers that are none, random numbers outside [0, 1)."""
    x = torch.randn((1, 999), generator=torch.Generator().manual_seed(1)).cuda()
    best, nan, inf = int(x.argmax()), float("nan"), float("inf")
    for t in (0.0, -1.0, nan, 1.0e-45, 1.0e-30):
        assert sample(x, [0.7], t=t)[0] == [best], t
    check_sample(x, [0.7], t=3.0e38)   # all weigh the same
    check_sample(x, [0.7], t=3.0e38, k=11)
    assert sample(x, [0.7], t=inf, k=11)[0] == sample(x, [0.7], t=3.0e38, k=11)[0]
    assert sample(x, [nan])[0] == sample(x, [0.0])[0] == sample(x, [-1.0])[0]
    assert sample(x, [7.0])[0] == sample(x, [1.0])[0] == [998]
    assert sample(x, [0.3], p=nan)[0] == sample(x, [0.3])[0]
    assert sample(x, [0.3], m=5.0)[0] == [best]


def test_sample_strides_and_alignment():
    """Rows that start anywhere, one row for all, a part of a wider row."""
    for dtype in (torch.float32, torch.bfloat16):
        wide = torch.randn((5, 1003), generator=torch.Generator().manual_seed(2)).to(dtype).cuda()
        for part in (wide[:, 1:902], wide[:, 3:], wide[::2, :77]):
            check_sample(part, [0.1, 0.4, 0.6, 0.8, 0.95][:part.shape[0]], k=30, p=0.9)
        same = wide[:1].expand(5, 1003)
        check_sample(same, [0.1, 0.4, 0.6, 0.8, 0.95], p=0.9)


def test_sample_more_rows_than_workgroups_run_at_once():
    x = (torch.randn((3000, 200), generator=torch.Generator().manual_seed(3)) * 2).cuda()
    check_sample(x, np.random.default_rng(3).random(3000), p=0.8, k=50)


def test_sample_twice_and_in_a_graph():
    x = (torch.randn((4, 50000), generator=torch.Generator().manual_seed(4)) * 2).to(torch.bfloat16).cuda()
    u, tokens, probs = torch.rand(4, device="cuda"), i32([0] * 4), torch.zeros(4, device="cuda")
    top_p, ws = torch.full((4,), 0.95, device="cuda"), torch.empty(kv.kv_sample_workspace(4, 50000), dtype=torch.uint8, device="cuda")
    call = lambda: kv.kv_sample(x, u, tokens, ws, top_p=top_p, probs=probs)  # noqa: E731
    call()
    first = tokens.clone(), probs.clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        call()
    s.synchronize()
    assert torch.equal(first[0], tokens) and torch.equal(first[1], probs)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for seed in range(4):
        gen = torch.Generator().manual_seed(seed)
        x.copy_((torch.randn((4, 50000), generator=gen) * 3).to(torch.bfloat16))
        u.copy_(torch.rand(4, generator=gen))
        tokens.fill_(-5)
        g.replay()
        torch.cuda.synchronize()
        got = tokens.clone(), probs.clone()
        call()
        torch.cuda.synchronize()
        assert torch.equal(got[0], tokens) and torch.equal(got[1], probs) and (tokens >= 0).all()


# ------------------------------------------------------------------------------------------ together
@pytest.mark.parametrize("fmt", ["16", "fp8"])
def test_a_batch_decodes_behind_a_shared_prompt(fmt):
    """Tables, cache rows, attention and sampling of some steps, as a graph that is replayed and eagerly, give the same; and attention is that of the definition."""
    H, G, D, bt, B, P, steps, V = 2, 4, 64, 16, 5, 70, 5, 500
    lens = [P + n for n in (0, 3, 25, 9, 40)]
    base = Batch(lens, [1] * B, H, G, D, torch.bfloat16, fmt, "paged", bt, seed=7, first=[0, B], prefix=[P], cap=20.0)
    c = base.c
    pool = c.dev["k"].shape[0]
    # rows of a table whose followers hold the leader's whole blocks
    whole = P // bt
    host = c.table_host
    held = [-(-n // bt) for n in lens]
    rows = [(host[0][:whole].tolist() + host[b][whole:held[b]].tolist() if b else host[0][:held[0]].tolist()) for b in range(B)]
    used = {i for r in rows for i in r}
    free = [i for i in range(pool) if i not in used]
    room = 12
    dt = torch.bfloat16
    gen = torch.Generator().manual_seed(8)
    data = [[torch.randn((B, h, D), generator=gen).to(dt) for h in (H * G, H, H)] + [torch.randn((B, V), generator=gen) * 2, torch.rand(B, generator=gen)] for _ in range(steps)]

    def loop(graphed):
        cache = {k: v.clone() for k, v in c.dev.items()}
        sets = [dict(held=i32(held), n_free=i32([len(free)]), table=i32([r + [-1] * (room - len(r)) for r in rows])) for _ in range(2)]
        stack, lens_dev, news = i32(free), i32(lens), i32([1] * B)
        first, seq, slot, status = i32([0] * (B + 1)), i32([0] * B), i32([0] * B), i32([0, 0])
        q, k, v, logits, u = (torch.empty_like(t, device="cuda") for t in data[0])
        out, tokens = torch.zeros((B, H * G, D), device="cuda"), i32([0] * B)
        leader, shared = i32([-1] + [0] * (B - 1)), i32([whole] * B)
        tree = kv.tree_batch(list(range(B + 1)), i32(list(range(B + 1))))
        groups, scores = kv.prefix_groups([0, B], i32([0, B]), [P], i32([P])), kv.scores(softcap=20.0)
        ws, sws = torch.empty(kv.kv_group_attn_workspace(c.plan, B, 200), dtype=torch.uint8, device="cuda"), torch.empty(kv.kv_sample_workspace(B, V), dtype=torch.uint8, device="cuda")
        got = []
        for s in range(steps):
            old, new = sets[s % 2], sets[1 - s % 2]
            now = [n + s for n in lens]
            mk = [cache["k"].view(torch.int16)], [cache["v"].view(torch.int16)]
            view = kv.paged_view(*mk, new["table"], now, lens_dev)
            blocks = None if fmt == "16" else kv.scale_blocks(kv.KV_FORMAT_FP8, [cache["k_scale"]], [cache["v_scale"]])
            tables = kv.step_tables(bt, lens_dev, news, old["held"], stack, old["n_free"], old["table"], first, seq, slot, status, leader, shared, new["held"], new["n_free"], new["table"])

            def step():
                kv.kv_step_tables(tables)
                kv.kv_cache_write(c.plan, view, blocks, 0, k, v, seq, slot)
                kv.kv_group_attn(c.plan, view, blocks, 0, tree, q, out, kv.KV_OUT_F32, 0, ws, groups, scores)
                kv.kv_sample(logits, u, tokens, sws, top_p=None)
            for t, x in zip((q, k, v, logits, u), data[s]):
                t.copy_(x)
            lens_dev.copy_(torch.tensor(now, dtype=torch.int32))
            if graphed:
                g = torch.cuda.CUDAGraph()
                with torch.cuda.graph(g):
                    step()
                for _ in range(3):   # a step of the same inputs is the same step: the old tables stay as they were
                    out.fill_(5)
                    g.replay()
                    torch.cuda.synchronize()
            else:
                step()
                torch.cuda.synchronize()
            assert status.tolist() == [0, 0]
            got.append([out.clone(), tokens.clone(), new["table"].clone(), new["held"].clone(), slot.clone()])
        return got, cache

    eager, cache = loop(False)
    graphed, _ = loop(True)
    for a, b in zip(eager, graphed):
        assert all(torch.equal(x, y) for x, y in zip(a, b))
    # the last step by the definition, over the cache as it is now
    n = steps - 1
    last = eager[-1]
    table = last[2].cpu().numpy()
    seq, slot = (i32([b for b in range(B) for _ in range(lens[b] + steps)]), i32([j for b in range(B) for j in range(lens[b] + steps)]))
    total = seq.numel()
    ko, vo = (torch.empty((total, H, D), dtype=dt, device="cuda") for _ in range(2))
    view = kv.paged_view([cache["k"].view(torch.int16)], [cache["v"].view(torch.int16)], last[2], [x + n for x in lens], i32([x + n for x in lens]))
    blocks = None if fmt == "16" else kv.scale_blocks(kv.KV_FORMAT_FP8, [cache["k_scale"]], [cache["v_scale"]])
    kv.kv_cache_read(c.plan, view, blocks, 0, seq, slot, ko, vo)
    assert (table[1:, :whole] == table[0, :whole]).all() and len({i for r, h in zip(table, last[3].tolist()) for i in r[whole:h]}) == sum(h - whole for h in last[3].tolist())
    q = data[-1][0].double().numpy()
    ko, vo = ko.double().cpu().numpy(), vo.double().cpu().numpy()
    at = np.concatenate([[0], np.cumsum([x + steps for x in lens])])
    for b in range(B):
        kb, vb = ko[at[b]:at[b + 1]].copy(), vo[at[b]:at[b + 1]].copy()
        kb[:P], vb[:P] = ko[:P], vo[:P]
        for h in range(H * G):
            x = 20 * np.tanh(kb[:, h // G] @ q[b, h] / 8 / 20)
            p = np.exp(x - x.max())
            want = p @ vb[:, h // G] / p.sum()
            # scores below 20 with (64 + 8 + 16) roundings of at most their terms' sum, some 30; weights off by that twice
            assert np.abs(last[0][b, h].double().cpu().numpy() - want).max() <= 2 * 30 * 90 * 2.0 ** -24 * np.abs(vb).max()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V,B", [(66000, 5), (70001, 40), (65537, 127), (65537, 128)])
def test_sample_rows_shared_by_workgroups(dtype, V, B):
    """Long rows, few enough to be shared, and one more: each way through them, ties by the thousand, rows without an answer, odd starts."""
    gen = torch.Generator().manual_seed(V + B)
    rows = 5 if B <= 40 else 3
    x = torch.randn((rows, V + 3), generator=gen) * 2
    x[1] = torch.round(x[1])          # ties by the thousand, in the bin of any border
    x[2, 5:] = x[2, 5:] * 0.01        # flat, and some above
    if rows > 3:
        x[3, 7] = float("nan")
        x[4, V // 2:] = float("-inf")
    x = x.to(dtype).cuda()[torch.arange(B) % rows]
    u = np.random.default_rng(B).random(B)
    some = [0, 1, 2, 3, 4] + list(range(B - 3, B)) if B <= 40 else [0, 1, 2, B - 1]
    for start, kw in ((0, dict(t=[0.0] * B)), (0, dict()), (1, dict(p=0.9)), (2, dict(k=40, p=0.8)), (0, dict(k=256)), (3, dict(k=257)), (1, dict(k=2000)), (0, dict(k=2000, m=0.001)), (0, dict(m=0.02)),
                      (1, dict(p=0.999, t=3.0)), (0, dict(k=900, p=0.95)), (0, dict(p=0.9, m=0.1))):
        part = x[:, start:start + V]
        tokens, probs = sample(part, u, **kw)
        host = part[some].double().cpu().numpy()
        for r, b in enumerate(some):
            token, prob = ref_sample(host[r], **{n: float(np.float32(v[b] if isinstance(v, list) else v)) if n != "k" else v for n, v in kw.items()}, u=float(np.float32(u[b])))
            assert tokens[b] == token, (b, kw, tokens[b], token)
            assert abs(probs[b] - prob) <= 2.0 ** -23 * prob + V * 2.0 ** -39, (b, kw, probs[b], prob)


@pytest.mark.parametrize("V", [300, 5000, 40000])
def test_sample_of_more_than_256(V):
    """top_k past what is ranked at once, alone and with min_p: bins that hold more ties than a list, temperatures that leave a bin or all of them, infinities."""
    x = torch.randn((6, V), generator=torch.Generator().manual_seed(V)) * 2
    x[1] = torch.round(x[1])
    x[2] = 1.5
    x[3, V // 3:] = float("-inf")
    x[4] = x[4] * 40
    x[5] = x[5].clamp(max=0.5)
    x = x.cuda()
    for k in (257, 270, V // 2, V - 1):
        for kw in (dict(), dict(t=0.01), dict(t=1.0e-38), dict(t=100.0), dict(m=0.05), dict(t=3.0, m=0.3)):
            check_sample(x, np.random.default_rng(k).random(6), k=k, **kw)


def test_sample_with_the_workspace_of_more_rows():
    """Fewer rows than the workspace is for, of a kind that needs more of it each."""
    V = 66000
    x = (torch.randn((9, V), generator=torch.Generator().manual_seed(9)) * 2).to(torch.bfloat16).cuda()
    ws = torch.empty(kv.kv_sample_workspace(200, V), dtype=torch.uint8, device="cuda").fill_(255)
    u = torch.full((9,), 0.5, device="cuda")
    p = torch.full((9,), 0.9, device="cuda")
    want = sample(x, [0.5] * 9, p=0.9)[0]
    for n in (9, 5, 1):
        tokens = i32([-9] * 9)
        kv.kv_sample(x[:n], u[:n], tokens[:n], ws, top_p=p[:n])
        assert tokens.tolist() == want[:n] + [-9] * (9 - n)


@pytest.mark.parametrize("fmt,requests", [("16", 6), ("fp8", 1), ("fp4", 9)])
def test_example_of_a_batch(fmt, requests):
    """Requests that begin, share, end and begin again."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "batch_step.py")
    spec = importlib.util.spec_from_file_location("batch_step", path)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    worst, drawn, blocks = mod.main(layers=2, requests=requests, prompt=150, steps=7, fmt=fmt, say=lambda *a: None)
    # results are rounded once, to 8 bits; the parts of probabilities lose 2^-16 in numerator and sum, scores up to 30 and their plain form some hundred units of 2^-24
    assert worst <= 2.0 ** -8 + 2.0 ** -12
    assert len(drawn) >= 7 and 150 // 16 < blocks <= requests * ((150 + 60 + 7) // 16 + 2)


@pytest.mark.parametrize("kw", [dict(k=50, p=0.9), dict(p=0.9), dict(k=900), dict(m=0.02), dict()])
def test_sample_two_calls_at_once(kw):
    """On two streams with workspaces of their own, again and again, and as a graph of both: the tokens of each alone."""
    V, runs = 70000, []
    for seed in (1, 2):
        x = (torch.randn((9, V), generator=torch.Generator().manual_seed(seed)) * 2).to(torch.bfloat16).cuda()
        dev = {n: torch.full((9,), v, dtype=torch.int32 if n == "k" else torch.float32, device="cuda") for n, v in kw.items()}
        args = dict(top_k=dev.get("k"), top_p=dev.get("p"), min_p=dev.get("m"))
        u = torch.rand(9, generator=torch.Generator().manual_seed(seed)).cuda()
        ws = torch.empty(kv.kv_sample_workspace(9, V), dtype=torch.uint8, device="cuda").fill_(255)
        runs.append((x, u, i32([-9] * 9), ws, args, torch.cuda.Stream(), sample(x, u.tolist(), **kw)[0]))
    torch.cuda.synchronize()
    for _ in range(20):
        for x, u, tokens, ws, args, stream, _w in runs:
            kv.kv_sample(x, u, tokens, ws, stream=stream, **args)
    torch.cuda.synchronize()
    assert all(tokens.tolist() == want for _, _, tokens, _, _, _, want in runs)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        for x, u, tokens, ws, args, _s, _w in runs:
            kv.kv_sample(x, u, tokens, ws, **args)
    for _ in range(3):
        for run in runs:
            run[2].fill_(-9)
            run[3].fill_(85)
        g.replay()
        torch.cuda.synchronize()
        assert all(tokens.tolist() == want for _, _, tokens, _, _, _, want in runs)


@pytest.mark.parametrize("V", [700, 32768, 32770, 65537])
@pytest.mark.parametrize("start", [0, 1, 7])
def test_sample_few_of_rows_that_fit_registers(V, start):
    """Up to, at and past what a workgroup's threads hold; lists of one, of a wavefront's lanes and more; the largest at both ends."""
    for dtype in (torch.float32, torch.float16):
        x = (torch.randn((4, V + 8), generator=torch.Generator().manual_seed(V)) * 2).to(dtype)
        x[0, start] = x[0, start + V - 1] = 20
        x[1] = torch.round(x[1].float()).to(dtype)
        x = x.cuda()[:, start:start + V]
        for kw in (dict(k=1), dict(k=2, t=0.5), dict(k=40, p=0.8), dict(k=64), dict(k=65, p=0.99), dict(k=256, m=0.1), dict(k=60, p=0.5, m=0.5)):
            check_sample(x, [0.0, 0.3, 0.7, 0.999], **kw)


@pytest.mark.parametrize("V", [900, 33000, 70000])
@pytest.mark.parametrize("spread", [5.0, 12.0, 40.0])
def test_sample_of_which_few_have_most(V, spread):
    """top_p alone, and with min_p, where lists of one, some and hundreds of tokens hold all that is kept."""
    x = torch.randn((6, V), generator=torch.Generator().manual_seed(int(spread))) * spread
    x[1] = torch.round(x[1] / 4) * 4          # the border in ties
    x[2, 100:160] = x[2].max()                # sixty of the largest
    x[3, :300] = x[3].max()                   # and more than a list is taken for
    x = x.to(torch.float16 if spread < 40 else torch.float32).cuda()
    for kw in (dict(p=0.5), dict(p=0.9, t=0.7), dict(p=0.999), dict(p=0.95, m=0.2), dict(p=0.9, m=1.0), dict(p=0.0)):
        check_sample(x, [0.1, 0.999, 0.4, 0.7, 0.5, 0.01], **kw)
