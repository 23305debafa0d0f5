"""Skipped entries of a slot write are as if they were not in the list, in fp8 pages too."""
import numpy as np
import pytest

import oracle
from tests.paged import bf16_bits, bf16_value
from tests.slot_lists import accepted_in_place, pool, skipping_list


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("seed", [0, 1, 2, 3])
def test_a_list_is_the_list_without_its_skipped_entries(seed, dtype):
    rng = np.random.default_rng(seed)
    slots, src, pages = skipping_list(rng, 200, rows=37)
    p = pool(rng, pages, 2, 64, dtype, base=0.005)
    new = [bf16_bits(rng.standard_normal((37, 2, 64))) for _ in range(2)]
    keep = (slots >= 0) & (slots < pages * 16) & (src >= 0) & (src < 37)
    assert 0 < keep.sum() < len(slots)
    args = dict(**p, kv_dtype=dtype, page_size=16, k_new=new[0], v_new=new[1])
    got = oracle.kv_write_slots(**args, slot_map=slots, src_rows=src)
    want = oracle.kv_write_slots(**args, slot_map=slots[keep], src_rows=src[keep])
    for x, y in zip(got, want):
        if x is not None:
            np.testing.assert_array_equal(x, y)


def test_accepted_drafts_in_place_are_the_gathered_ones():
    rng = np.random.default_rng(5)
    slots, pages = accepted_in_place(rng, 20, 16)
    p = pool(rng, pages, 1, 64, "fp8", base=0.005)
    new = [bf16_bits(rng.standard_normal((len(slots), 1, 64))) for _ in range(2)]
    at = np.flatnonzero(slots >= 0)
    args = dict(**p, kv_dtype="fp8", page_size=16, k_new=new[0], v_new=new[1])
    got = oracle.kv_write_slots(**args, slot_map=slots)
    want = oracle.kv_write_slots(**args, slot_map=slots[at], src_rows=at)
    for x, y in zip(got, want):
        np.testing.assert_array_equal(x, y)


def test_one_scale_for_a_run_with_a_gap():
    """Rows 2 and 4 of a page: one scale from both, rows 0 and 1 requantised once, rows 3 and 5 on as they were."""
    rng = np.random.default_rng(6)
    p = pool(rng, 1, 1, 64, "fp8", base=0.001)
    new = bf16_bits(rng.standard_normal((3, 1, 64)) * np.array([1.0, 1.0, 50.0])[:, None, None])
    got = oracle.kv_write_slots(**p, kv_dtype="fp8", page_size=16, slot_map=[2, 3, 4], k_new=new, v_new=new,
                                src_rows=[0, 3, 2])
    x = np.abs(bf16_value(new[[0, 2]])).max().astype(np.float32)
    assert got[2][0, 0] == x / np.float32(448.0)
    np.testing.assert_array_equal(got[0][0, 0, [3, *range(5, 16)]], p["k_pages"][0, 0, [3, *range(5, 16)]])
    want = oracle.kv_write_slots(**p, kv_dtype="fp8", page_size=16, slot_map=[2], k_new=new, v_new=new, src_rows=[2])
    np.testing.assert_array_equal(got[0][0, 0, :2], want[0][0, 0, :2])
    np.testing.assert_array_equal(got[0][0, 0, 4], want[0][0, 0, 2])
