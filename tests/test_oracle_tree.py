"""Pins of the tree attention, slot write and page table oracles: library attention on dense arrays, the append
and prefill oracles, and invariants."""
import numpy as np
import pytest
import torch

import oracle
from tests.paged import bf16_bits, bf16_value, dense_keys, paged_from_dense, random_dense
from workloads import make_workload


@pytest.mark.parametrize("Hq,Hkv,d", [(4, 2, 64), (8, 1, 64), (2, 2, 128)])
def test_tree_attention_matches_masked_library_attention(Hq, Hkv, d):
    rng = np.random.default_rng(Hq + d)
    P, L, n = [17, 0], [5, 33, 0], [3, 1, 6]
    pk, pv, rk, rv, g, q0 = random_dense(rng, S=3, G=2, Hq=Hq, Hkv=Hkv, d=d, prefix_lens=P, resp_lens=L)
    wl = paged_from_dense(pk, pv, rk, rv, g, q0, num_kv_heads=Hkv)
    offs = np.concatenate([[0], np.cumsum(n)])
    T = int(offs[-1])
    q, kd, vd = (bf16_bits(rng.standard_normal((T, h, d))) for h in (Hq, Hkv, Hkv))
    masks = rng.integers(1, 64, T).astype(np.uint64)
    out, lse, spread, reach = oracle.tree_for_workload(wl, offs, masks, q, kd, vd)
    for s in range(3):
        K, V = dense_keys(pk, pv, rk, rv, g, s)
        a, b = offs[s], offs[s + 1]
        K = np.concatenate([K, bf16_value(kd[a:b])]).repeat(Hq // Hkv, 1)
        V = np.concatenate([V, bf16_value(vd[a:b])]).repeat(Hq // Hkv, 1)
        see = np.ones((b - a, len(K)), bool)
        see[:, len(K) - (b - a):] = [[int(m) >> u & 1 for u in range(b - a)] for m in masks[a:b]]
        x = [torch.from_numpy(np.ascontiguousarray(np.swapaxes(y, 0, 1))) for y in (bf16_value(q[a:b]), K, V)]
        ref = torch.nn.functional.scaled_dot_product_attention(*x, attn_mask=torch.from_numpy(see),
                                                               scale=float(wl.softmax_scale))
        has = see.any(1)
        np.testing.assert_allclose(out[a:b][has], ref.transpose(0, 1).numpy()[has], rtol=1e-10, atol=1e-12)
        assert np.all(out[a:b][~has] == 0) and np.all(lse[a:b][~has] == -np.inf)
        assert np.all(spread[a:b] >= np.abs(out[a:b]) - 1e-12)


def test_one_draft_that_sees_itself_is_the_decode_step():
    rng = np.random.default_rng(3)
    wl = make_workload(num_q_heads=4, num_kv_heads=2, head_dim=64, seq_to_group=[0, 1, 0], prefix_lens=[20, 3],
                       resp_lens=[0, 16, 30], seed=9, append=True)
    after = oracle.append_for_workload(wl)
    want, want_lse = oracle.attention_for_workload(wl, pool=after)
    out, lse, _, _ = oracle.tree_for_workload(wl, [0, 1, 2, 3], np.ones(3, np.uint64), wl.q, wl.k_new, wl.v_new)
    np.testing.assert_allclose(out, want, rtol=1e-12)
    np.testing.assert_allclose(lse, want_lse, rtol=1e-12)


def _pool(rng, pages, hkv, d):
    codes = rng.integers(0, 0x7F, (2, pages, hkv, 16, d)).astype(np.uint8)
    scale = np.exp(rng.standard_normal((2, pages, hkv))).astype(np.float32) / 300
    return dict(k_pages=codes[0], v_pages=codes[1], k_scale=scale[0], v_scale=scale[1], kv_dtype="fp8", page_size=16)


def test_slot_writes_of_single_rows_are_appends():
    rng = np.random.default_rng(1)
    pool = _pool(rng, 8, 2, 64)
    lens, table = np.array([0, 5, 15, 16, 31]), np.array([[0, 1], [2, 2], [3, 3], [4, 5], [6, 7]])
    new = [bf16_bits(3 * rng.standard_normal((5, 2, 64))) for _ in range(2)]
    slots = [table[s, t // 16] * 16 + t % 16 for s, t in enumerate(lens)]
    got = oracle.kv_write_slots(**pool, slot_map=slots, k_new=new[0], v_new=new[1])
    want = oracle.kv_append(**pool, resp_lens=lens, resp_block_table=table, k_new=new[0], v_new=new[1])
    for x, y in zip(got, want):
        np.testing.assert_array_equal(x, y)


@pytest.mark.parametrize("kv_dtype", ["bf16", "fp8"])
def test_slot_writes_of_whole_prompts_are_the_prefill_write(kv_dtype):
    rng = np.random.default_rng(2)
    pool = _pool(rng, 6, 3, 64)
    if kv_dtype == "bf16":
        z = np.zeros((6, 3, 16, 64), np.uint16)
        pool.update(k_pages=z, v_pages=z, k_scale=None, v_scale=None, kv_dtype="bf16")
    table, offs = np.array([[3, 0, 5], [1, 4, 0]]), np.array([0, 40, 57])
    new = [bf16_bits(rng.standard_normal((57, 3, 64))) for _ in range(2)]
    slots = [table[g, t // 16] * 16 + t % 16 for g in range(2) for t in range(offs[g + 1] - offs[g])]
    order = rng.permutation(57)
    got = oracle.kv_write_slots(**pool, slot_map=slots, k_new=new[0][order], v_new=new[1][order],
                                src_rows=np.argsort(order))
    want = oracle.prefill_kv_write(**pool, prefix_block_table=table, prefix_offs=offs, k=new[0], v=new[1])
    for x, y in zip(got, want):
        np.testing.assert_array_equal(x, y)


def test_resizes_hand_out_every_page_once_and_an_opposite_one_restores():
    rng = np.random.default_rng(4)
    S, width, pages = 9, 6, 40
    table, stack, count = np.full((S, width), -1), rng.permutation(pages), pages
    lens = np.zeros(S, int)
    for _ in range(30):
        new = np.where(rng.random(S) < 0.3, 0, np.minimum(lens + rng.integers(0, 40, S), width * 16))
        status, t2, s2, c2, offs, slots = oracle.page_tables_resize(table, stack, count, lens, new)
        if status[0] == 1:
            assert status[1] > count + status[2]
            np.testing.assert_array_equal(t2, table)
            continue
        assert status[0] == 0
        held = [t2[s, p] for s in range(S) for p in range(-(-new[s] // 16))]
        assert sorted(held + list(s2[:c2])) == list(range(pages))
        assert (np.sort(t2, 1)[:, ::-1] >= 0).sum() == len(held)
        assert len(slots) == offs[-1] == np.maximum(new - lens, 0).sum() and len(set(slots)) == len(slots)
        back = oracle.page_tables_resize(t2, s2, c2, new, lens)
        np.testing.assert_array_equal(back[1], table)
        np.testing.assert_array_equal(back[2][:count], stack[:count])
        assert back[0][0] == 0 and back[3] == count
        table, stack, count, lens = t2, s2, c2, new
    assert oracle.page_tables_resize(table, stack, count, lens, lens + 1000)[0][0] == 2
    assert oracle.page_tables_resize(table, stack, 41, lens, lens)[0][0] == 4
    assert oracle.page_tables_resize(table, stack, count, lens * 0, lens * 0 + 1, max_slots=8)[0][0] == 3
