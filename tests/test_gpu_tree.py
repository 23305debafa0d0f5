"""Tree attention on the GPU against the fp64 oracle: head shapes, types, lengths around pages and units, ragged
trees, masks, padding, streams and graphs."""
import numpy as np
import pytest
import torch

import oracle
from tests.paged import bf16_bits
from tests.tree_util import check_tree, compare_tree, drafts_for, run_tree, say
from workloads import make_workload

pytestmark = pytest.mark.gpu


def _wl(hq, hkv, d, dtype, groups, P, L, seed=1, **kw):
    return make_workload(num_q_heads=hq, num_kv_heads=hkv, head_dim=d, seq_to_group=groups, prefix_lens=P, resp_lens=L,
                         seed=seed, kv_dtype=dtype, **kw)


# Tables of this width have too many pages for one unit per sequence.
WIDE = 2000


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv", [(2, 2), (4, 2), (8, 2), (16, 2), (3, 3)])
def test_heads_types_and_lengths_around_pages(hq, hkv, d, dtype):
    """Lengths 0, 1 and around a page, prefixes likewise, 0 to 13 drafts, in one launch and in two."""
    L = [0, 1, 15, 16, 17, 33, 100, 0, 64, 250]
    groups = [0, 1, 2, 0, 1, 2, 3, 3, 0, 4]
    P = [0, 1, 16, 47, 130, 20]
    counts = [1, 2, 0, 13, 5, 1, 9, 4, 3, 8]
    for width in (None, WIDE):
        wl = _wl(hq, hkv, d, dtype, groups, P, L, seed=hq + d, max_resp_pages=width)
        b, *_ = check_tree(wl, counts, 5, f"tree hq {hq} hkv {hkv} d {d} {dtype} width {width}")
        assert (b.draft_workspace.numel() > 256) == (width is not None)


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv,n", [(1, 1, 64), (4, 2, 16), (4, 1, 17), (8, 1, 64), (2, 1, 33), (8, 8, 48)])
def test_large_trees(hq, hkv, n, d, dtype):
    """Row counts on both sides of 16, 32 and 64, and several row blocks; blocks of drafts full and ragged."""
    counts = [n, n - 1, 1, max(1, n - 16)]
    for width in (None, WIDE):
        wl = _wl(hq, hkv, d, dtype, [0, 0, 1, 0], [70, 5], [40, 0, 300, 129], seed=n, max_resp_pages=width)
        check_tree(wl, counts, n, f"tree n {n} hq {hq} hkv {hkv} d {d} {dtype} width {width}")


@pytest.mark.parametrize("hq,hkv,d,dtype", [(4, 2, 128, "bf16"), (8, 2, 64, "fp8"), (2, 2, 128, "fp8"), (8, 1, 64, "bf16")])
def test_long_caches(hq, hkv, d, dtype):
    """Responses of many units, prefixes of several chunks, empty ones beside them."""
    wl = _wl(hq, hkv, d, dtype, [1, 0, 1, 2, 0], [1500, 4000, 0], [9000, 8191, 0, 5000, 16], seed=2)
    check_tree(wl, [3, 8, 5, 1, 2], 3, f"tree long {hq} {hkv} {d} {dtype}")
    wl = _wl(hq, hkv, d, dtype, [0], [3], [24000], seed=3)
    check_tree(wl, [2], 3, f"tree long single {hq} {hkv} {d} {dtype}")


@pytest.mark.parametrize("width", [None, WIDE])
def test_groups_of_every_size_in_any_order(width):
    """600 sequences: a group with most of them (its rows are found over several rounds of the scan), small ones,
    an empty one, sequences without drafts."""
    rng = np.random.default_rng(8)
    S = 600
    groups = np.where(rng.random(S) < 0.6, 2, rng.integers(0, 9, S))
    groups[groups == 5] = 6
    counts = rng.integers(0, 5, S)
    counts[-1] = 0
    wl = _wl(2, 1, 64, "bf16", groups, rng.integers(0, 90, 9), rng.integers(0, 40, S), seed=5, max_resp_pages=width)
    check_tree(wl, counts, 6, f"tree 600 sequences width {width}", max_drafts=4)


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
def test_more_group_rows_than_row_blocks_in_the_grid(dtype):
    """One group holds all drafts of a call that is sized for many groups."""
    wl = _wl(4, 1, 64, dtype, [3] * 40, [9, 0, 80, 600, 1, 2, 3, 4], np.arange(40) * 7, seed=4, max_resp_pages=WIDE)
    check_tree(wl, [16] * 40, 4, f"tree one group of many {dtype}")


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("hq,hkv,d,most", [(4, 2, 128, 3), (2, 2, 64, 3), (8, 1, 64, 40), (8, 1, 128, 40), (16, 4, 64, 2)])
def test_long_prefixes_of_many_members(hq, hkv, d, most, dtype):
    """Prefixes that pay to be read once for all members: units of their own, of several chunks, for row counts on
    both sides of a workgroup's, with members in any order, some without drafts, another group without a prefix."""
    rng = np.random.default_rng(hq + most)
    counts = rng.integers(0, 3, 60)
    counts[7] = most
    groups = np.where(rng.random(60) < 0.9, 1, 0)
    wl = _wl(hq, hkv, d, dtype, groups, [0, 3000], rng.integers(0, 120, 60), seed=5, max_resp_pages=WIDE)
    check_tree(wl, counts, 6, f"tree long prefix {hq} {hkv} {d} {most} {dtype}", max_drafts=most)
    wl = _wl(hq, hkv, d, dtype, groups, [33, 1601], rng.integers(0, 120, 60), seed=5)
    check_tree(wl, counts, 6, f"tree long prefix {hq} {hkv} {d} {most} {dtype}, short table", max_drafts=most)


def test_many_sequences_of_all_lengths():
    """More units than a launch orders at once by length, with ties, empty ones and one that is far the longest."""
    rng = np.random.default_rng(2)
    L = rng.integers(0, 200, 700)
    L[::7], L[300], L[:5] = 64, 6000, 0
    wl = _wl(2, 2, 64, "bf16", np.arange(700) % 5, [10, 0, 40, 3, 100], L, seed=5)
    check_tree(wl, 1 + np.arange(700) % 2, 6, "tree 700 lengths", max_drafts=2)
    wl = _wl(1, 1, 64, "fp8", np.arange(1100) % 5, [10, 0, 40, 3, 100], rng.integers(0, 90, 1100), seed=5)
    check_tree(wl, np.ones(1100, int), 6, "tree 1100 sequences", max_drafts=1)


FORMS = [(1, 1, 16), (2, 1, 16), (4, 1, 16), (8, 1, 16)]  # of 16, 32, 64 and 128 query rows


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv,n", FORMS)
def test_sequences_of_a_thousand_pages_undivided(hq, hkv, n, d, dtype):
    """More sequences than are ordered or divided: long ones are one unit each."""
    rng = np.random.default_rng(n + hq)
    L, counts = rng.integers(0, 30, 1030), np.where(np.arange(1030) % 9 == 0, 1, 0)
    L[[3, 500, 1029]], counts[[3, 500, 1029]] = [8190, 16399, 9000], [n, n - 1, 2]
    wl = _wl(hq, hkv, d, dtype, [0] * 1029 + [1], [20, 4], L, seed=5)
    check_tree(wl, counts, 6, f"tree undivided {hq} {hkv} {n} {d} {dtype}", max_drafts=n)


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("hq,hkv,n", FORMS)
@pytest.mark.parametrize("S,prefix", [(300, 20), (70, 20), (70, 1500), (600, 40)])
def test_long_sequences_among_short_ones(S, prefix, hq, hkv, n, dtype):
    """A few long sequences, first, last and with an empty tree, are divided; the others are one unit each. Tables
    as wide as the longest and wider, prefixes read once for all or with each sequence."""
    rng = np.random.default_rng(S + n)
    L, counts = rng.integers(0, 60, S), rng.integers(0, 3, S)
    at = [0, 31, S // 2, S - 1]
    L[at], counts[at] = [9001, 30000, 7680 - prefix, 20000], [2, n, 3, 0 if S == 70 else 1]
    groups = np.where(np.arange(S) % 5 == 2, 1, 0)
    heads = 4 if S == 70 else 1
    for width in (None, 4000):
        wl = _wl(heads * hq, heads * hkv, 64, dtype, groups, [prefix, 0], L, seed=5, max_resp_pages=width)
        check_tree(wl, counts, 6, f"tree uneven {S} {prefix} {hq} {n} {dtype} width {width}", max_drafts=n)


@pytest.mark.parametrize("width", [None, WIDE])
@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
def test_masks_of_any_kind(dtype, width):
    """Rows that see nothing, everything, only others, and bits at and above the tree's size; with an empty cache
    too, where a row without bits has no key at all."""
    rng = np.random.default_rng(9)
    counts = [20, 5, 64, 3]
    masks = rng.integers(0, 2 ** 63, sum(counts), dtype=np.uint64) * np.uint64(2) + np.uint64(1)
    masks[[0, 3, 22, 30]] = 0
    masks[[1, 25]] = np.uint64(2 ** 64 - 1)
    masks[23] = np.uint64(2 ** 64 - 32)  # five drafts: only bits above them
    for P, L in (([0, 30], [0, 7, 0, 40]), ([0, 0], [0, 0, 0, 0])):
        wl = _wl(4, 2, 128, dtype, [0, 0, 0, 1], P, L, seed=1, max_resp_pages=width)
        _, _, out, lse = check_tree(wl, counts, 7, f"tree masks {dtype} {width} {P}", masks=masks)
        if not any(L):
            assert np.all(out[[0, 3, 22, 23, 30]] == 0) and np.all(lse[[0, 3, 22, 23, 30]] == -np.inf)


@pytest.mark.parametrize("width", [None, WIDE])
@pytest.mark.parametrize("hq,d,dtype", [(2, 64, "bf16"), (8, 128, "bf16"), (4, 128, "fp8"), (8, 64, "fp8")])
def test_hidden_drafts_may_hold_anything(hq, d, dtype, width):
    """NaN, infinities and the type's extremes in the K and V of drafts that others do not see."""
    wl = _wl(hq, 1, d, dtype, [0, 0, 0], [40], [50, 0, 17], seed=6, max_resp_pages=width)
    counts = [40, 17, 3]
    offs = np.concatenate([[0], np.cumsum(counts)])
    rng = np.random.default_rng(3)
    hidden = [1, 7, 16, 33, 39, 40 + 2, 40 + 16, 57 + 1]
    masks = rng.integers(0, 2 ** 62, 60, dtype=np.uint64)
    for t in hidden:
        s = int(np.searchsorted(offs, t, side="right")) - 1
        masks[offs[s]:offs[s + 1]] &= ~(np.uint64(1) << np.uint64(t - offs[s]))
    dr = drafts_for(wl, counts, 12, masks)
    for i, t in enumerate(hidden):
        dr["k_draft"][t, :, i::3] = [0x7FC0, 0x7F80, 0xFF80, 0xFF7F][i % 4]
        dr["v_draft"][t, :, i::5] = [0x7F80, 0x7FC0, 0xFF80, 0xFFFF][i % 4]
    say(f"tree hidden values hq {hq} d {d} {dtype} width {width}")
    _, out, lse = run_tree(wl, dr, 40)
    ref = oracle.tree_for_workload(wl, **dr)
    live = [t for t in range(60) if t not in hidden]
    assert np.isfinite(out[live]).all()
    compare_tree(out, lse, ref, d, "hidden values")


@pytest.mark.parametrize("width", [None, WIDE])
@pytest.mark.parametrize("d", [64, 128])
def test_infinite_v_reaches_the_rows_that_see_it(d, width):
    wl = _wl(4, 1, d, "bf16", [0], [20], [30], seed=6, max_resp_pages=width)
    masks = np.array([1, 3, 5, 9, 1 << 4], np.uint64)
    dr = drafts_for(wl, [5], 1, masks)
    dr["v_draft"][1, 0, 3], dr["v_draft"][2, 0, 5], dr["v_draft"][3, 0, 8] = 0x7F80, 0xFF80, 0x7FC0
    _, out, lse = run_tree(wl, dr, 5)
    r_out, r_lse, spread, reach = oracle.tree_for_workload(wl, **dr)
    assert np.array_equal(np.isnan(out), np.isnan(r_out)) and np.isnan(out[3, :, 8]).all()
    inf = np.isinf(r_out)
    assert np.array_equal(out[inf], r_out[inf]) and inf.sum() == 8
    out, r_out, spread = (np.where(np.isfinite(r_out), x, 0) for x in (out, r_out, spread))
    compare_tree(out, lse, (r_out, r_lse, spread, reach), d, "infinite v")


def test_large_scores_and_a_dominant_key():
    """Scores of several hundred: the running maximum moves far, one key takes all the weight, and its value comes
    out unrounded but for the output's own rounding."""
    wl = _wl(4, 2, 128, "bf16", [0, 0], [100], [500, 70], seed=6, k_mult=4.0, max_resp_pages=WIDE)
    dr = drafts_for(wl, [6, 9], 2)
    dr["q"] = bf16_bits(16 * np.random.default_rng(1).standard_normal(dr["q"].shape))
    say("tree large scores")
    _, out, lse = run_tree(wl, dr, 9)
    ref = oracle.tree_for_workload(wl, **dr)
    compare_tree(out, lse, ref, 128, "large scores")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv,n", FORMS)
def test_scales_of_fp8_pages(hq, hkv, n, d):
    """Scales of very different sizes and of zero; a lone key's value comes out with no rounding but the output's."""
    wl = _wl(hq, hkv, d, "fp8", np.arange(6), [0] * 6, [1, 1, 1, 300, 40, 16], seed=n + d)
    rng = np.random.default_rng(3)
    wl.v_scale *= np.exp2(rng.uniform(-40, 3, wl.v_scale.shape)).astype(np.float32)
    wl.v_scale[wl.resp_block_table[3][2:5]] = 0
    wl.v_scale[wl.resp_block_table[5][0]] = 0
    wl.k_scale[wl.resp_block_table[3][4:7]] = 0
    counts = [n, 1, 2, n, 3, 1]
    dr = drafts_for(wl, counts, 4)
    lone = dr["draft_offs"][3]
    dr["masks"][:lone] = 0
    dr["masks"][-1] = 0  # sees a page of zeros alone
    say(f"tree scales hq {hq} n {n} d {d}")
    _, out, lse = run_tree(wl, dr, n)
    ref = oracle.tree_for_workload(wl, **dr)
    compare_tree(out, lse, ref, d, "scales")
    # fp32 steps of the division by the scale and by the sum: less than 2^-10 of the rounding.
    assert np.all(np.abs(out[:lone] - ref[0][:lone]) <= 2.0 ** -8 * (1 + 2.0 ** -10) * np.abs(ref[0][:lone]))
    assert np.all(out[-1] == 0)


@pytest.mark.parametrize("width", [None, WIDE])
def test_rows_behind_the_last_sequence_stay(width):
    import paper_2606_26997_amd as rp
    wl = _wl(4, 2, 64, "bf16", [0, 1, 0], [20, 0], [9, 30, 0], seed=2, max_resp_pages=width)
    dr = drafts_for(wl, [3, 0, 2], 4)
    _, out, lse = run_tree(wl, dr, 7)
    pad = {k: np.concatenate([v, v[:4]]) if k != "draft_offs" else v for k, v in dr.items()}
    b, out2, lse2 = run_tree(wl, pad, 7)
    np.testing.assert_array_equal(out2[:5], out)
    np.testing.assert_array_equal(lse2[:5], lse)
    assert np.isnan(out2[5:]).all() and np.isnan(lse2[5:]).all()
    # No lse wanted, raw stream handle.
    b.draft_out.zero_()
    rp.group_tree_attn(b.kv, b.append_layout, b.tree, b.draft_q, b.k_draft, b.v_draft, b.softmax_scale, b.draft_out,
                       None, b.draft_workspace, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(b.draft_out[:5].float().cpu().numpy(), out)
    assert not b.draft_out[5:].any()


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
def test_one_draft_equals_the_decode_step(dtype):
    """One draft that sees itself is the next token of its sequence: the cache with it appended (bf16) and the
    decode attention give the same result up to the roundings of both."""
    import paper_2606_26997_amd as rp
    rng = np.random.default_rng(4)
    wl = _wl(16, 8, 128, dtype, np.arange(24) % 3, [300, 64, 0], rng.integers(0, 900, 24), seed=7, append=True,
             max_resp_pages=WIDE)
    dr = dict(draft_offs=np.arange(25, dtype=np.int32), masks=np.ones(24, np.uint64), q=wl.q, k_draft=wl.k_new,
              v_draft=wl.v_new)
    b, out, lse = run_tree(wl, dr, 1)
    if dtype == "bf16":
        b.step()
        torch.cuda.synchronize()
        assert float((b.out.float() - b.draft_out.float()).abs().max()) <= 2e-2
        assert float((b.lse - b.draft_lse).abs().max()) <= 1e-4
    compare_tree(out, lse, oracle.tree_for_workload(wl, **dr), 128, "one draft")


def test_cache_offsets_beyond_32_bits():
    """Pages whose byte offset in the pool passes 2^32: K and V of 4.5 GiB each, only the pages used are filled."""
    import paper_2606_26997_amd as rp
    say("tree in a pool of 9 GiB")
    small = _wl(4, 2, 128, "bf16", [0, 0], [40], [50, 20], seed=9)
    dr = drafts_for(small, [4, 3], 1)
    _, out, lse = run_tree(small, dr, 4)
    n, used = 576000, small.k_pages.shape[0]
    b = rp.DeviceBatch.from_workload(small)
    pools = [torch.empty(n, 2, 16, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    for pool, old in zip(pools, (b.k_pages, b.v_pages)):
        pool[n - used:] = old
    assert (n - used) * 2 * 16 * 128 * 2 > 1 << 32
    b.k_pages, b.v_pages = pools
    b.prefix_block_table += n - used
    b.resp_block_table += n - used
    b.kv = rp.paged_kv(*pools)
    _, out2, lse2 = run_tree(small, dr, 4, batch=b)
    np.testing.assert_array_equal(out2, out)
    np.testing.assert_array_equal(lse2, lse)


@pytest.mark.parametrize("width", [None, WIDE])
@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
def test_repeats_and_graph_replays_are_equal(dtype, width):
    """The same bits from every call, on another stream, and from a graph replayed between eager calls whose
    sequences and masks change in place."""
    wl = _wl(8, 4, 128, dtype, np.arange(16) // 8, [200, 90], np.arange(16) * 30, seed=3, max_resp_pages=width)
    dr = drafts_for(wl, [1 + i % 9 for i in range(16)], 2)
    say(f"tree graph {dtype} {width}")
    b, _, _ = run_tree(wl, dr, 9)
    first = b.draft_out.clone(), b.draft_lse.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    b.draft_out.zero_()
    side.wait_stream(torch.cuda.current_stream())
    b.tree_attention(side)
    side.synchronize()
    assert torch.equal(b.draft_out, first[0])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        b.tree_attention()
    for i in range(3):
        b.draft_out.fill_(float("nan"))
        b.draft_lse.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(b.draft_out, first[0]) and torch.equal(b.draft_lse, first[1])
        b.resp_lens.sub_(1).clamp_(min=0)
        b.draft_masks.bitwise_or_(1 << i)
        b.tree_attention()
        torch.cuda.synchronize()
        first = b.draft_out.clone(), b.draft_lse.clone()


def test_two_calls_at_once():
    """Two streams, each with its own workspace, on one cache: both results are those of the calls one after the
    other."""
    import paper_2606_26997_amd as rp
    say("tree two streams")
    wl = _wl(8, 4, 64, "bf16", [0, 1, 0, 1], [300, 17], [5000, 2000, 0, 9000], seed=8)
    cases = [(drafts_for(wl, counts, i), max(counts)) for i, counts in enumerate(([4, 1, 9, 16], [30, 2, 1, 0]))]
    want = [run_tree(wl, dr, most)[1:] for dr, most in cases]
    batches = []
    for dr, most in cases:
        b = rp.DeviceBatch.from_workload(wl)
        b.set_drafts(**{**dr, "masks": dr["masks"].view(np.int64)}, max_drafts=most)
        batches.append((b, torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(3):
        for b, stream in batches:
            with torch.cuda.stream(stream):
                b.draft_out.zero_()
                b.tree_attention()
        torch.cuda.synchronize()
        for (b, _), (out, lse) in zip(batches, want):
            assert np.array_equal(b.draft_out.float().cpu().numpy().astype(np.float64), out)
            assert np.array_equal(b.draft_lse.cpu().numpy().astype(np.float64), lse)


def test_the_binding_refuses_more_drafts_than_masks():
    import paper_2606_26997_amd as rp
    offs, masks = (torch.zeros(3, dtype=t, device="cuda") for t in (torch.int32, torch.int64))
    with pytest.raises(ValueError, match="masks has 3"):
        rp.draft_tree(offs, masks, max_drafts=2, num_drafts=4)
    assert rp.draft_tree(offs, masks, max_drafts=2, num_drafts=2).num_drafts == 2
