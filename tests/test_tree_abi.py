"""Refusals of the tree attention, the slot writes and the page tables, on the CPU: every check comes before a
launch, and fake addresses are never read."""
import ctypes

import pytest
import torch

import paper_2606_26997_amd as rp
from paper_2606_26997_amd import _binding as B
from tests.test_abi import A, _kv, _layout

FP8 = dict(kv_dtype=rp.RP_KV_FP8_E4M3, k_scale=A, v_scale=A)


def _tree(**kw):
    d = dict(num_drafts=8, max_drafts=4, draft_offs=A, masks=A)
    d.update(kw)
    return B.RpDraftTree(d["num_drafts"], d["max_drafts"], d["draft_offs"], d["masks"])


def _ref(x):
    return None if x is None else ctypes.byref(x)


def _size(kv, layout, tree):
    n = ctypes.c_size_t(12345)
    return rp.load().rp_group_tree_attn_workspace_size(_ref(kv), _ref(layout), _ref(tree), ctypes.byref(n)), n.value


def _attn(kv, layout, tree, q=A, k=A, v=A, scale=0.1, out=A, lse=A, ws=A, ws_bytes=1 << 40):
    return rp.load().rp_group_tree_attn(_ref(kv), _ref(layout), _ref(tree), q, k, v, scale, out, lse, ws, ws_bytes,
                                        None)


@pytest.mark.parametrize("kw,status,needle", [
    (dict(num_drafts=-1), rp.RP_ERR_INVALID_ARG, "num_drafts"),
    (dict(max_drafts=0), rp.RP_ERR_INVALID_ARG, "max_drafts"),
    (dict(max_drafts=65), rp.RP_ERR_UNSUPPORTED, "limit 64"),
    (dict(draft_offs=None), rp.RP_ERR_INVALID_ARG, "draft_offs"),
    (dict(masks=None), rp.RP_ERR_INVALID_ARG, "masks"),
    (dict(masks=A + 4), rp.RP_ERR_INVALID_ARG, "masks"),
    (dict(num_drafts=1 << 30), rp.RP_ERR_UNSUPPORTED, "too many drafts"),
])
def test_bad_trees(kw, status, needle):
    for st in (_size(_kv(), _layout(), _tree(**kw))[0], _attn(_kv(), _layout(), _tree(**kw))):
        assert st == status and needle in rp.last_error()


@pytest.mark.parametrize("kw,status", [
    (dict(q=None), rp.RP_ERR_INVALID_ARG), (dict(q=A + 8), rp.RP_ERR_INVALID_ARG), (dict(k=None), rp.RP_ERR_INVALID_ARG),
    (dict(v=A + 2), rp.RP_ERR_INVALID_ARG), (dict(out=None), rp.RP_ERR_INVALID_ARG),
    (dict(lse=A + 2), rp.RP_ERR_INVALID_ARG), (dict(scale=0.0), rp.RP_ERR_INVALID_ARG),
    (dict(scale=-1.0), rp.RP_ERR_INVALID_ARG), (dict(scale=float("nan")), rp.RP_ERR_INVALID_ARG),
    (dict(scale=float("inf")), rp.RP_ERR_INVALID_ARG), (dict(ws=None), rp.RP_ERR_WORKSPACE),
    (dict(ws=A + 64), rp.RP_ERR_WORKSPACE), (dict(ws_bytes=4096), rp.RP_ERR_WORKSPACE),
])
def test_bad_attention_arguments(kw, status):
    layout = _layout(mrp=4000)
    assert _size(_kv(), layout, _tree())[1] > 4096
    assert _attn(_kv(), layout, _tree(), **kw) == status and rp.last_error()


def test_the_pool_and_the_layout_are_checked_as_for_a_decode_step():
    for kv, layout, status in ((_kv(head_dim=96), _layout(), rp.RP_ERR_UNSUPPORTED),
                               (_kv(page_size=32), _layout(), rp.RP_ERR_UNSUPPORTED),
                               (_kv(), _layout(num_q_heads=6), rp.RP_ERR_UNSUPPORTED),
                               (_kv(), _layout(resp_lens=None), rp.RP_ERR_INVALID_ARG),
                               (None, _layout(), rp.RP_ERR_INVALID_ARG), (_kv(), None, rp.RP_ERR_INVALID_ARG)):
        assert _size(kv, layout, _tree())[0] == status
        assert _attn(kv, layout, _tree()) == status
    assert _size(_kv(), _layout(), None)[0] == rp.RP_ERR_INVALID_ARG


def test_nothing_to_do():
    assert _size(_kv(), _layout(), _tree(num_drafts=0, draft_offs=None, masks=None)) == (rp.RP_OK, 0)
    assert _attn(_kv(), _layout(), _tree(num_drafts=0), q=None, out=None, ws=None, ws_bytes=0) == rp.RP_OK
    assert _attn(_kv(), _layout(num_seqs=0), _tree(), q=None, ws=None, ws_bytes=0) == rp.RP_OK


def _write(kv, slots=A, n=4, k=A, v=A, src=None, num_src=4):
    return rp.load().rp_kv_write_slots(_ref(kv), slots, n, k, v, src, num_src, None)


@pytest.mark.parametrize("kv_kw", [{}, FP8])
@pytest.mark.parametrize("kw,status", [
    (dict(slots=None), rp.RP_ERR_INVALID_ARG), (dict(slots=A + 2), rp.RP_ERR_INVALID_ARG),
    (dict(src=A + 1), rp.RP_ERR_INVALID_ARG), (dict(k=None), rp.RP_ERR_INVALID_ARG),
    (dict(v=A + 8), rp.RP_ERR_INVALID_ARG), (dict(n=-1), rp.RP_ERR_INVALID_ARG),
    (dict(num_src=-1), rp.RP_ERR_INVALID_ARG), (dict(n=1 << 30), rp.RP_ERR_UNSUPPORTED),
])
def test_bad_slot_writes(kv_kw, kw, status):
    assert _write(_kv(**kv_kw), **kw) == status and rp.last_error()


def test_slot_write_pools():
    assert _write(None) == rp.RP_ERR_INVALID_ARG
    assert _write(_kv(head_dim=32)) == rp.RP_ERR_UNSUPPORTED
    assert _write(_kv(num_pages=1 << 27)) == rp.RP_ERR_UNSUPPORTED
    assert _write(_kv(), n=0, slots=None, k=None, v=None) == rp.RP_OK
    assert _write(_kv(), num_src=0, k=None, v=None) == rp.RP_OK


def _tables(**kw):
    d = dict(num_seqs=2, max_pages=4, page_size=16, num_pages=8, block_table=A, free_pages=A, free_count=A)
    d.update(kw)
    return B.RpPageTables(*(d[n] for n, _ in B.RpPageTables._fields_))


def _resize(t, old=A, new=A, status=A, offs=A, slots=A, max_slots=4):
    return rp.load().rp_page_tables_resize(_ref(t), old, new, status, offs, slots, max_slots, None)


@pytest.mark.parametrize("t_kw,kw,status", [
    (dict(num_seqs=-1), {}, rp.RP_ERR_INVALID_ARG), (dict(num_seqs=4097), {}, rp.RP_ERR_UNSUPPORTED),
    (dict(max_pages=-1), {}, rp.RP_ERR_INVALID_ARG), (dict(num_pages=0), {}, rp.RP_ERR_INVALID_ARG),
    (dict(num_pages=1 << 27), {}, rp.RP_ERR_UNSUPPORTED), (dict(page_size=32), {}, rp.RP_ERR_UNSUPPORTED),
    (dict(num_seqs=4096, max_pages=1 << 20), {}, rp.RP_ERR_UNSUPPORTED),
    (dict(block_table=None), {}, rp.RP_ERR_INVALID_ARG), (dict(free_pages=None), {}, rp.RP_ERR_INVALID_ARG),
    (dict(free_count=A + 2), {}, rp.RP_ERR_INVALID_ARG), ({}, dict(old=None), rp.RP_ERR_INVALID_ARG),
    ({}, dict(new=A + 1), rp.RP_ERR_INVALID_ARG), ({}, dict(status=None), rp.RP_ERR_INVALID_ARG),
    ({}, dict(offs=None), rp.RP_ERR_INVALID_ARG), ({}, dict(slots=A + 2), rp.RP_ERR_INVALID_ARG),
    ({}, dict(max_slots=-1), rp.RP_ERR_INVALID_ARG),
])
def test_bad_page_tables(t_kw, kw, status):
    assert _resize(_tables(**t_kw), **kw) == status and rp.last_error()


def test_null_page_tables():
    assert _resize(None) == rp.RP_ERR_INVALID_ARG


def test_the_binding_refuses_tensors_of_another_kind():
    kv, layout, tree = _kv(), _layout(), _tree()
    q = torch.zeros(8, 4, 64, dtype=torch.bfloat16)
    k = torch.zeros(8, 2, 64, dtype=torch.bfloat16)
    args = dict(q=A, k_draft=A, v_draft=A, softmax_scale=0.1, out=A, lse=None, workspace=None)
    for name, t, needle in (("q", q.float(), "dtype"), ("q", q[:4], "shape"), ("k_draft", q, "shape"),
                            ("q", torch.zeros(8, 64, 4, dtype=torch.bfloat16).transpose(1, 2), "contiguous"),
                            ("q", q, "current GPU"), ("workspace", torch.zeros(8, 2)[:, 0], "contiguous"),
                            ("workspace", q, "current GPU")):
        with pytest.raises(ValueError, match=needle):
            rp.group_tree_attn(kv, layout, tree, **{**args, name: t})
    with pytest.raises(ValueError, match="dtype"):
        rp.draft_tree(torch.zeros(3, dtype=torch.int64), torch.zeros(8, dtype=torch.int64), max_drafts=4)
    with pytest.raises(ValueError, match="shape"):
        rp.kv_write_slots(kv, torch.zeros(8, dtype=torch.int32).view(2, 4), k, k)
    with pytest.raises(ValueError, match="dtype"):
        rp.kv_write_slots(kv, torch.zeros(8, dtype=torch.int64), k, k)
    with pytest.raises(ValueError, match="shape"):
        rp.page_tables(torch.zeros(4, dtype=torch.int32), A, A)
    with pytest.raises(ValueError, match="dtype"):
        rp.page_tables_resize(_tables(), torch.zeros(2, dtype=torch.int64), A, A)
