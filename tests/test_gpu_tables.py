"""Page tables on the GPU: tables, stack, count, offsets, slots and status equal the oracle's, entry by entry."""
import numpy as np
import pytest
import torch

import oracle
from tests.tree_util import say

pytestmark = pytest.mark.gpu


def _i32(x):
    return torch.from_numpy(np.ascontiguousarray(x, np.int32)).cuda()


class State:
    """A table and its stack on both sides."""

    def __init__(self, rng, S, width, pages):
        import paper_2606_26997_amd as rp
        self.rp = rp
        self.table, self.stack, self.count = np.full((S, width), -1), rng.permutation(pages), pages
        self.lens = np.zeros(S, int)
        self.d = [_i32(self.table), _i32(self.stack), _i32([pages])]
        self.tables = rp.page_tables(*self.d)

    def resize(self, new, spare=5, slots=True, offs=True, max_slots=None):
        """One call on both sides, compared; returns the status code."""
        S = len(self.lens)
        fresh = int(np.maximum(np.asarray(new, np.int64) - self.lens, 0).sum())
        n = max(0, min(fresh, 1 << 20) + spare if max_slots is None else max_slots)
        out = [torch.full((k,), 77, dtype=torch.int32, device="cuda") for k in (4, S + 1, n)]
        status, table, stack, count, want_offs, want_slots = oracle.page_tables_resize(
            self.table, self.stack, self.count, self.lens, new, max_slots=n if slots else None)
        self.rp.page_tables_resize(self.tables, _i32(self.lens), _i32(new), out[0], out[1] if offs else None,
                                   out[2] if slots else None)
        torch.cuda.synchronize()
        assert out[0].tolist() == status
        np.testing.assert_array_equal(self.d[0].cpu().numpy(), table)
        assert int(self.d[2]) == count
        np.testing.assert_array_equal(self.d[1].cpu().numpy(), stack)
        if offs:
            np.testing.assert_array_equal(out[1].cpu().numpy(), want_offs)
        if slots:
            np.testing.assert_array_equal(out[2].cpu().numpy()[:len(want_slots)], want_slots)
            assert (out[2][len(want_slots):] == -1).all()
        if status[0] == 0:
            self.table, self.stack, self.count, self.lens = table, stack, count, np.asarray(new).copy()
        return status[0]


@pytest.mark.parametrize("S,width", [(1, 1), (1, 300), (7, 5), (64, 40), (257, 9), (1024, 6), (1025, 3), (4096, 4)])
def test_random_steps(S, width):
    """Sequences that grow, shrink, end and begin in the same call, over many calls; calls that find too few
    pages change nothing."""
    say(f"tables {S} x {width}")
    rng = np.random.default_rng(S)
    st = State(rng, S, width, max(2, S * width // 2))
    codes = []
    for i in range(12):
        grow = rng.integers(0, [3, 20, 16 * width + 1][i % 3], S)
        new = np.clip(np.where(rng.random(S) < 0.3, st.lens - grow, st.lens + grow), 0, 16 * width)
        new[rng.random(S) < 0.1] = 0
        codes.append(st.resize(new, slots=i % 4 != 1, offs=i % 4 != 1 or i % 2 == 0))
    assert 0 in codes
    assert st.resize(st.lens) == 0
    assert st.resize(np.zeros(S, int)) == 0 and st.count == len(st.stack)


def test_many_pages_and_slots():
    """Long prompts: far more pages and slots than one workgroup takes at a time; ended again at once."""
    say("tables long prompts")
    rng = np.random.default_rng(3)
    st = State(rng, 300, 256, 300 * 130)
    assert st.resize(rng.integers(0, 2049, 300)) == 0
    new = st.lens.copy()
    new[::2] = 0
    new[1::2] += rng.integers(0, 2000, 150)
    assert st.resize(new) == 0
    assert st.resize(np.zeros(300, int)) == 0


@pytest.mark.parametrize("S,width", [(5, 20), (900, 64)])
def test_refusals_change_nothing(S, width):
    rng = np.random.default_rng(1)
    say(f"tables refusals {S}")
    st = State(rng, S, width, S * 8)
    assert st.resize(rng.integers(1, 64, S)) == 0
    assert st.resize(st.lens + 16 * 8) == 1
    for bad in (-1, 16 * width + 1, 2 ** 31 - 1, -2 ** 31):
        new = st.lens + 1
        new[S // 2] = bad
        assert st.resize(new, max_slots=10000) == 2
    assert st.resize(st.lens + 2, max_slots=2 * S - 1) == 3
    assert st.resize(st.lens + 2, max_slots=0) == 3
    assert st.resize(st.lens + 2, max_slots=2 * S) == 0
    for count in (-1, S * 8 + 1):
        keep = st.count
        st.count = count
        st.d[2].fill_(count)
        assert st.resize(st.lens + 1) == 4
        st.count = keep
        st.d[2].fill_(keep)
    assert st.resize(st.lens + 1) == 0


def test_lengths_that_are_wrong_before_the_call():
    rng = np.random.default_rng(1)
    st = State(rng, 4, 4, 16)
    st.lens = np.array([0, -3, 0, 70])
    assert st.resize(np.array([1, 1, 1, 1]), max_slots=10) == 2


def test_no_sequences_and_no_width():
    import paper_2606_26997_amd as rp
    stack, count, status = _i32([2, 1, 0]), _i32([3]), _i32([9] * 4)
    none, offs, slots = _i32([]), _i32([9]), _i32([9, 9])
    rp.page_tables_resize(rp.page_tables(_i32(np.zeros((0, 4))), stack, count), none, none, status, offs, slots)
    torch.cuda.synchronize()
    assert status.tolist() == [0, 0, 0, 0] and offs.tolist() == [0] and slots.tolist() == [-1, -1]
    lens = _i32([0, 0])
    rp.page_tables_resize(rp.page_tables(_i32(np.zeros((2, 0))), stack, count), lens, lens, status)
    torch.cuda.synchronize()
    assert status.tolist() == [0, 0, 0, 0] and count.item() == 3


def test_replayed_graph_and_another_stream():
    """A captured grow-and-release replayed between eager calls, and the same on a side stream: tables and stack
    return to what they were, and the slots of every replay are the eager ones."""
    import paper_2606_26997_amd as rp
    say("tables graph")
    pt = rp.PageTables(num_seqs=40, max_pages=30, num_pages=900)
    pt.resize(torch.randint(0, 200, (40,), dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert pt.status.tolist()[0] == rp.RP_TABLES_OK
    old, new = pt.lens.clone(), pt.lens + 9
    status, offs, slots = _i32([0] * 4), _i32([0] * 41), _i32([0] * 360)

    def step():
        rp.page_tables_resize(pt.tables, old, new, status, offs, slots)
        rp.page_tables_resize(pt.tables, new, old, status)
    before = [t.clone() for t in (pt.block_table, pt.stack[1])]
    step()
    want = slots.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    assert torch.equal(slots, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for _ in range(3):
        slots.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(slots, want) and status.tolist()[0] == 0
        assert all(torch.equal(x, y) for x, y in zip((pt.block_table, pt.stack[1]), before))
        step()


def test_the_handle_keeps_its_lengths_when_a_call_is_refused():
    import paper_2606_26997_amd as rp
    pt = rp.PageTables(num_seqs=2, max_pages=4, num_pages=3)
    more = rp.PageTables(num_seqs=1, max_pages=4, stack=pt.stack)
    pt.resize(torch.tensor([17, 3], dtype=torch.int32, device="cuda"))
    more.resize(torch.tensor([1], dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert pt.status.tolist() == [0, 3, 0, 20] and more.status.tolist() == [1, 1, 0, 1]
    assert pt.lens.tolist() == [17, 3] and more.lens.tolist() == [0]
    assert pt.block_table[:, :2].tolist() == [[0, 1], [2, -1]]


def test_the_handle_on_streams_given_by_address():
    import paper_2606_26997_amd as rp
    pt = rp.PageTables(num_seqs=2, max_pages=4, num_pages=8)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    lens = [torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([20, 3], [33, 40], [0, 16])]
    torch.cuda.synchronize()
    for x, stream in zip(lens, (0, side.cuda_stream, side)):
        pt.resize(x, stream=stream)
        torch.cuda.synchronize()
        assert pt.status.tolist()[0] == rp.RP_TABLES_OK and torch.equal(pt.lens, x)
    assert pt.stack[1].item() == 7
