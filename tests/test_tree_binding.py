"""What the binding refuses of descriptors that do not fit each other, before the library sees them."""
import pytest
import torch

import paper_2606_26997_amd as rp
from paper_2606_26997_amd import _binding as B
from tests.test_abi import A, _kv, _layout


@pytest.fixture
def any_device(monkeypatch):
    monkeypatch.setattr(B, "_tensors", lambda *specs: None)  # which asks for tensors on a GPU


def _calls(layout, tree):
    """Both calls that take a tree; without a softmax scale the library refuses the second one itself."""
    rp.group_tree_attn_workspace_size(_kv(), layout, tree)
    with pytest.raises(rp.RpError, match="softmax_scale"):
        rp.group_tree_attn(_kv(), layout, tree, A, A, A, 0.0, A, None, None)


@pytest.mark.parametrize("seqs", [1, 2, 7])
def test_offsets_of_too_few_sequences(any_device, seqs):
    layout, masks = _layout(num_seqs=seqs), torch.ones(8, dtype=torch.int64)
    for n in range(seqs + 1):
        tree = rp.draft_tree(torch.zeros(n, dtype=torch.int32), masks, max_drafts=4)
        with pytest.raises(ValueError, match="draft_offs"):
            rp.group_tree_attn_workspace_size(_kv(), layout, tree)
        with pytest.raises(ValueError, match="draft_offs"):
            rp.group_tree_attn(_kv(), layout, tree, A, A, A, 0.0, A, None, None)
    for n in (seqs + 1, seqs + 2, seqs + 100):  # longer: offsets of a larger batch, of which the first are used
        _calls(layout, rp.draft_tree(torch.zeros(n, dtype=torch.int32), masks, max_drafts=4))


def test_offsets_given_by_address_are_the_caller_s(any_device):
    _calls(_layout(), rp.draft_tree(A, torch.ones(8, dtype=torch.int64), max_drafts=4))
    _calls(_layout(), rp.draft_tree(A, A, max_drafts=4, num_drafts=8))
    _calls(_layout(), B.RpDraftTree(8, 4, A, A))


@pytest.mark.parametrize("slots", [0, 4])
def test_slots_without_offsets(any_device, slots):
    """Also where the slots' tensor is empty and so has no address: new tokens count against its size."""
    tables = B.RpPageTables(2, 4, 16, 8, A, A, A)
    with pytest.raises(rp.RpError, match="slot_map needs slot_offs") as e:
        rp.page_tables_resize(tables, A, A, A, None, torch.zeros(slots, dtype=torch.int32))
    assert e.value.status == rp.RP_ERR_INVALID_ARG
