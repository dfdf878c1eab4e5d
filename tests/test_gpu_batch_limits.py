"""A batch's step at the ends of what its calls take."""
import pytest
import torch

from batchcase import ref_tables
from paper_2604_26557_amd import binding as kv
from test_gpu_batch import check_sample

pytestmark = pytest.mark.gpu


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("in_place", [False, True])
def test_maps_of_as_many_rows_as_there_can_be(in_place):
    """2^31 - 1 rows, of which all but the last 1000 have a token: the last workgroup's end is past 31 bits."""
    n = 2 ** 31 - 1
    seq, slot = (torch.full((n,), 7, dtype=torch.int32, device="cuda") for _ in range(2))
    held, n_free, table = i32([0, 0]), i32([0]), i32([[-1], [-1]])
    outs = {} if in_place else dict(held_out=i32([5, 5]), n_free_out=i32([5]), block_table_out=i32([[5], [5]]))
    first, status, lens, news = i32([5, 5, 5]), i32([5, 5]), i32([3, 0]), i32([10, n - 1010])
    kv.kv_step_tables(kv.step_tables(16, lens, news, held, i32([]), n_free, table, first, seq, slot, status, **outs))
    assert first.tolist() == [0, 10, n - 1000] and status.tolist()[1] == 1
    assert seq[:12].tolist() == [0] * 10 + [1, 1] and slot[:12].tolist() == list(range(3, 13)) + [0, 1]
    assert seq[n - 1003:].tolist() == [1] * 3 + [-1] * 1000 and slot[n - 1003:].tolist() == [n - 1013, n - 1012, n - 1011] + [-1] * 1000
    at = torch.arange(10, n - 1000, 4099, device="cuda")
    assert (seq[at] == 1).all() and torch.equal(slot[at].long(), at - 10)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("begin", [0, 16, 30, 64, 80, 96, 112])
def test_a_stack_with_less_room_than_what_ends(in_place, begin):
    """Four blocks are free and fill their array; three more end in the call, of which as many as begin are handed out. What is left past the array is lost, and nothing that lies in it."""
    lens, news, held, rows = [40, 0], [-1, begin], [3, 0], [[11, 12, 13, -1, -1, -1, -1], [-1] * 7]
    want_rows, want_held, stack, n_free, status, *_ = ref_tables(16, lens, news, held, [1, 2, 3, 4], 4, rows)
    assert status == [0, 0]
    free, n_dev, table, held_dev, status = i32([1, 2, 3, 4]), i32([4]), i32(rows), i32(held), i32([5, 5])
    outs = dict(held_out=i32([5, 5]), n_free_out=i32([5]), block_table_out=torch.full_like(table, 5))
    kv.kv_step_tables(kv.step_tables(16, i32(lens), i32(news), held_dev, free, n_dev, table, i32([5, 5, 5]), i32([]), i32([]), status, **({} if in_place else outs)))
    got = (table, held_dev, n_dev) if in_place else (outs["block_table_out"], outs["held_out"], outs["n_free_out"])
    assert status.tolist() == [0, 0] and got[0].tolist() == want_rows and got[1].tolist() == want_held
    assert free.tolist() == stack[:4] and int(got[2]) == min(n_free, 4)
    used = {i for r in want_rows for i in r if i >= 0}
    assert not used & set(free.tolist()[:int(got[2])])


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("n_free", [0, 1, 3])
@pytest.mark.parametrize("more", [-1, 0, 1])
def test_the_last_free_block_and_one_more(in_place, n_free, more):
    """Two requests end with 8 blocks; what the others want is one block less than there is, all of it, or one too many: then nobody gets any."""
    lens, held = [40, 33, 64, 10], [3, 3, 5, 1]
    rows = [r + [-1] * (16 - len(r)) for r in ([1, 2, 3], [4, 5, 6], [7, 8, 9, 10, 11], [12])]
    # the fourth wants 2 blocks, the second what is left of 8 + n_free
    want = 8 + n_free - 2 + more
    news, free = [-1, 16 * (3 + want) - 33, -1, 38], [20 + i for i in range(n_free)] + [-1] * (16 - n_free)
    after = ref_tables(16, lens, news, held, free, n_free, rows, n_tok=4)
    assert after[4] == [max(0, more), 0]
    free_dev, n_dev, table, held_dev, status = i32(free), i32([n_free]), i32(rows), i32(held), i32([5, 5])
    seq, slot, first = i32([5] * 4), i32([5] * 4), i32([5] * 5)
    outs = dict(held_out=i32([5] * 4), n_free_out=i32([5]), block_table_out=torch.full_like(table, 5))
    kv.kv_step_tables(kv.step_tables(16, i32(lens), i32(news), held_dev, free_dev, n_dev, table, first, seq, slot, status, **({} if in_place else outs)))
    got = (table, held_dev, n_dev) if in_place else (outs["block_table_out"], outs["held_out"], outs["n_free_out"])
    assert (got[0].tolist(), got[1].tolist(), free_dev.tolist(), int(got[2]), status.tolist(), first.tolist(), seq.tolist(), slot.tolist()) == tuple(after)
    if more > 0:
        assert got[0][1].tolist() == rows[1] and got[1].tolist() == [0, 3, 0, 1] and int(got[2]) == 8 + n_free
    else:
        assert int(got[2]) == -more


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_samples_of_lists_of_every_length_of_a_wavefront(dtype):
    """The k largest of equal, of few different and of different logits, k up to a lane more than there are, at once: a row for each."""
    k = list(range(1, 66)) * 3
    x = torch.randn((len(k), 333), generator=torch.Generator().manual_seed(3)) * 2
    x[65:130] = torch.round(x[65:130])
    x[130:] = 0.25
    u = torch.rand(len(k), generator=torch.Generator().manual_seed(4)).tolist()
    for kw in (dict(), dict(p=[0.7] * len(k)), dict(m=[0.1] * len(k), t=[0.6] * len(k))):
        check_sample(x.to(dtype).cuda(), u, k=k, **kw)


def test_samples_of_rows_that_each_ask_for_something_else():
    """Of long rows that workgroups share: the largest, few of the largest, many, a border by weight, by both, by min_p, nothing, in one call."""
    V, B = 70003, 40
    x = (torch.randn((B, V), generator=torch.Generator().manual_seed(5)) * 2).to(torch.bfloat16).cuda()
    x[9, 77] = float("nan")
    x[17] = float("-inf")
    kw = dict(t=[0.0, 1.0, 0.7, 1.3, 1.0, 0.9, 2.0, 1.0] * 5, k=[0, 40, 1000, 0, 300, 0, 0, 1] * 5, p=[1.0, 0.9, 1.0, 0.95, 0.8, 1.0, 1.0, 0.5] * 5, m=[0.0, 0.0, 0.01, 0.02, 0.0, 0.03, 0.0, 0.0] * 5)
    check_sample(x, torch.rand(B, generator=torch.Generator().manual_seed(6)).tolist(), **kw)


def test_samples_of_the_largest_vocabulary():
    V = 1 << 24
    x = (torch.randn((1, V), generator=torch.Generator().manual_seed(7)) * 2).to(torch.float16).cuda()
    for kw in (dict(), dict(p=0.9), dict(k=50), dict(m=0.01), dict(t=0.0)):
        check_sample(x, [0.83], **kw)


def test_samples_of_as_many_rows_as_a_launch_may_have():
    n = (1 << 22) - 1
    x = torch.randn((n, 3), generator=torch.Generator().manual_seed(8)).cuda()
    tokens, probs, t = torch.full((n,), -9, dtype=torch.int32, device="cuda"), torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    kv.kv_sample(x, t, tokens, torch.empty(16, dtype=torch.uint8, device="cuda"), temperature=t, probs=probs)
    assert torch.equal(tokens.long(), x.argmax(1)) and (probs == 1).all()
