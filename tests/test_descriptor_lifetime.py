"""Descriptors hold addresses; the tensors behind those live as long as the descriptor does."""
import gc
import weakref

import pytest
import torch

import paper_2606_26997_amd as rp
from paper_2606_26997_amd import _binding as B


def _zeros(shape, dtype, device):
    return torch.zeros(shape, dtype=dtype, device=device)


def _described(device):
    """(name, [descriptor], weak references to the tensors that it was made from, their addresses)."""
    i32, bf16, f32, u8 = torch.int32, torch.bfloat16, torch.float32, torch.uint8
    makers = {
        "paged_kv bf16": (rp.paged_kv, [((2, 1, 16, 64), bf16)] * 2, {}),
        "paged_kv fp8": (rp.paged_kv, [((2, 1, 16, 64), u8)] * 2 + [((2, 1), f32)] * 2, {}),
        "group_layout": (rp.group_layout, [((3,), i32), ((1,), i32), ((1, 2), i32), ((3,), i32), ((3, 2), i32)],
                         dict(num_q_heads=2)),
        "prefill_layout": (rp.prefill_layout, [((3,), i32), ((2, 4), i32)], dict(num_q_heads=2, num_tokens=7)),
        "draft_tree": (rp.draft_tree, [((4,), i32), ((6,), torch.int64)], dict(max_drafts=2)),
        "page_tables": (rp.page_tables, [((3, 4), i32), ((8,), i32), ((1,), i32)], {}),
    }
    for name, (make, specs, kw) in makers.items():
        tensors = [_zeros(shape, dtype, device) for shape, dtype in specs]
        refs, addresses, box = [weakref.ref(t) for t in tensors], [t.data_ptr() for t in tensors], [make(*tensors, **kw)]
        del tensors
        yield name, box, refs, addresses


def _check(device):
    for name, box, refs, addresses in _described(device):
        gc.collect()
        assert all(r() is not None for r in refs), name
        assert set(addresses) <= {getattr(box[0], f) for f, _ in box[0]._fields_}, name
        box.clear()
        gc.collect()
        assert all(r() is None for r in refs), name


def test_a_descriptor_keeps_its_tensors(monkeypatch):
    monkeypatch.setattr(B, "_tensors", lambda *specs: None)  # which asks for tensors on a GPU
    _check("cpu")


@pytest.mark.gpu
def test_a_descriptor_keeps_its_tensors_on_the_gpu():
    _check("cuda")


def test_raw_addresses_are_held_by_the_caller():
    kv = rp.paged_kv(4096, 8192, num_pages=1, num_kv_heads=1, head_dim=64)
    assert (kv.k_pages, kv.v_pages) == (4096, 8192)
