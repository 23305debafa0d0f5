"""Page tables so wide that sums of new tokens could pass 32 bits, up to the last that an int32 counts."""
import numpy as np
import pytest
import torch

import oracle
from tests.tree_util import say

pytestmark = pytest.mark.gpu


def _i32(x):
    return torch.from_numpy(np.ascontiguousarray(x, np.int32)).cuda()


def test_steps_of_a_wide_table():
    """2^27 entries: sequences that grow, shrink and end, one of them over its whole row, against the oracle."""
    import paper_2606_26997_amd as rp
    S, width, pages = 4096, 32768, 100000
    say(f"tables {S} x {width}")
    rng = np.random.default_rng(11)
    table, stack, count = np.full((S, width), -1, np.int32), rng.permutation(pages), pages
    lens = np.zeros(S, int)
    d = [_i32(table), _i32(stack), _i32([count])]
    tables = rp.page_tables(*d)
    grown = rng.integers(0, 256, S)
    whole = np.where(np.arange(S) == 77, width * 16, np.maximum(grown - rng.integers(0, 99, S), 0))
    steps = [(grown, 0), (whole, 0), (np.where(np.arange(S) == 5, width * 16 + 1, whole), 2), (whole + (whole < 99), 0),
             (np.full(S, 600), 1), (np.zeros(S, int), 0)]
    for new, code in steps:
        fresh = int(np.maximum(new - lens, 0).sum())
        status, offs, slots = (torch.full((n,), 77, dtype=torch.int32, device="cuda") for n in (4, S + 1, fresh + 3))
        rp.page_tables_resize(tables, _i32(lens), _i32(new), status, offs, slots)
        want = oracle.page_tables_resize(table, stack, count, lens, new, max_slots=fresh + 3)
        assert want[0][0] == code and status.tolist() == want[0]
        np.testing.assert_array_equal(d[0].cpu().numpy(), want[1])
        np.testing.assert_array_equal(d[1].cpu().numpy(), want[2])
        assert d[2].item() == want[3]
        np.testing.assert_array_equal(offs.cpu().numpy(), want[4])
        np.testing.assert_array_equal(slots.cpu().numpy()[:len(want[5])], want[5])
        assert (slots[len(want[5]):] == -1).all()
        if code == 0:
            table, stack, count, lens = want[1], want[2], want[3], new


@pytest.mark.parametrize("total", [2 ** 31 - 1, 2 ** 31])
def test_as_many_new_tokens_as_an_int32_counts_and_one_more(total):
    """The free pages 0, 1, ... are enough for both. Sequences have one token each, so that they take a page less
    than their new tokens fill; page rank o of all is the stack's from the top."""
    import paper_2606_26997_amd as rp
    S, width, pages = 4096, 33100, 2 ** 27 - 1
    say(f"tables {S} x {width}, {total} tokens")
    new = torch.full((S,), 1 + 524287, dtype=torch.int64, device="cuda")
    new[0] += total - S * 524287
    assert int((new - 1).sum()) == total and int(new.max()) <= 16 * width
    taken = (new + 15) // 16 - 1
    assert int(taken.sum()) <= pages
    table = torch.full((S, width), -5, dtype=torch.int32, device="cuda")
    free, count = torch.arange(pages, dtype=torch.int32, device="cuda"), _i32([pages])
    old, new32 = torch.ones(S, dtype=torch.int32, device="cuda"), new.int()
    status, offs = (torch.full((n,), 77, dtype=torch.int32, device="cuda") for n in (4, S + 1))
    tables = rp.page_tables(table, free, count)
    rp.page_tables_resize(tables, old, new32, status, offs)
    N, done = int(taken.sum()), total < 2 ** 31
    assert status.tolist() == [rp.RP_TABLES_OK if done else rp.RP_TABLES_NO_SLOTS, N, 0, 2 ** 31 - 1]
    if not done:
        assert count.item() == pages and bool((table == -5).all()) and bool((offs == 0).all())
        assert torch.equal(free, torch.arange(pages, dtype=torch.int32, device="cuda"))
        return
    assert count.item() == pages - N
    assert torch.equal(offs[1:].long(), (new - 1).cumsum(0)) and offs[0].item() == 0
    p = torch.arange(width, device="cuda")[None]
    rank = (taken.cumsum(0) - taken)[:, None] + p - 1
    live = (p >= 1) & (p <= taken[:, None])
    assert torch.equal(table, torch.where(live, pages - 1 - rank, -5).int())
    del rank
    rp.page_tables_resize(tables, new32, old, status, offs)
    assert status.tolist() == [rp.RP_TABLES_OK, 0, N, 0] and count.item() == pages
    assert torch.equal(free, torch.arange(pages, dtype=torch.int32, device="cuda"))
    assert torch.equal(table, torch.where(live, -1, -5).int())
