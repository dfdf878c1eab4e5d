"""A batch's step at the ends of what its calls take."""
import pytest
import torch

from paper_2604_26557_amd import binding as kv

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
