"""Slot writes on the GPU: bytes and scales equal the oracle's, and those of the append and the prefill write."""
import numpy as np
import pytest
import torch

import oracle
from tests.paged import bf16_bits
from tests.tree_util import say
from workloads import make_prefill_workload, make_workload

pytestmark = pytest.mark.gpu


def _pool(rng, pages, hkv, d, dtype, base=1.0):
    if dtype == "bf16":
        k, v = (rng.integers(0, 0x7F00, (pages, hkv, 16, d)).astype(np.uint16) for _ in range(2))
        return dict(k_pages=k, v_pages=v, k_scale=None, v_scale=None)
    k, v = (rng.integers(0, 0x7F, (pages, hkv, 16, d)).astype(np.uint8) for _ in range(2))
    ks, vs = ((base * np.exp(0.5 * rng.standard_normal((pages, hkv)))).astype(np.float32) for _ in range(2))
    return dict(k_pages=k, v_pages=v, k_scale=ks, v_scale=vs)


def _dev(x):
    if x is None:
        return None
    if x.dtype == np.uint16:
        return torch.from_numpy(x.view(np.int16)).view(torch.bfloat16).cuda()
    return torch.from_numpy(x).cuda()


def _host(t):
    return t.view(torch.int16).cpu().numpy().view(np.uint16) if t.dtype == torch.bfloat16 else t.cpu().numpy()


def _check(pool, dtype, slots, k_new, v_new, src=None, repeat=True):
    import paper_2606_26997_amd as rp
    want = oracle.kv_write_slots(**pool, kv_dtype=dtype, page_size=16, slot_map=slots, k_new=k_new, v_new=v_new,
                                 src_rows=src)
    t = {k: _dev(x) for k, x in pool.items()}
    kv = rp.paged_kv(t["k_pages"], t["v_pages"], t["k_scale"], t["v_scale"])
    args = [torch.from_numpy(np.asarray(slots, np.int32)).cuda(), _dev(k_new), _dev(v_new),
            None if src is None else torch.from_numpy(np.asarray(src, np.int32)).cuda()]
    for _ in range(2 if repeat else 1):  # the second call finds its own result
        rp.kv_write_slots(kv, *args)
        torch.cuda.synchronize()
        for name, y in zip(("k_pages", "v_pages", "k_scale", "v_scale"), want):
            if y is not None:
                np.testing.assert_array_equal(_host(t[name]), y, err_msg=name)
    return kv, t, args


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("hkv,d", [(1, 64), (8, 128), (3, 64), (2, 128)])
def test_runs_of_every_place_and_length(hkv, d, dtype):
    """Every first row and length of a run inside a page, one after the other in the list, so that they begin at
    every place of a wave's share."""
    say(f"slot runs hkv {hkv} d {d} {dtype}")
    rng = np.random.default_rng(hkv * d)
    slots, page = [], 0
    for r in range(16):
        for n in range(1, 17 - r):
            slots += range(page * 16 + r, page * 16 + r + n)
            page += 1
    new = [bf16_bits(rng.standard_normal((len(slots), hkv, d)) * np.exp(rng.standard_normal((len(slots), 1, 1))))
           for _ in range(2)]
    _check(_pool(rng, page, hkv, d, dtype, base=0.01), dtype, slots, *new)


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("T", [1, 2, 16, 17, 63, 64, 65, 1000])
def test_gathered_rows_skips_and_repeats(T, dtype):
    """Rows in any order and several times, slots of -1 and outside the pool, rows outside the source."""
    say(f"slot gather {T} {dtype}")
    rng = np.random.default_rng(T)
    pages = T // 4 + 2
    slots, src, page = [], rng.integers(0, 37, T), 0
    while len(slots) < T:  # one run per page, some of them cut by a skipped entry at either end
        r = int(rng.integers(0, 16))
        n = int(rng.integers(1, 17 - r))
        slots += list(range(page * 16 + r, page * 16 + r + n)) if page < pages else [-1] * n
        if rng.random() < 0.3:
            slots.append([-1, -2 ** 31, pages * 16, 2 ** 31 - 1][int(rng.integers(0, 4))])
        page += 1
    slots = np.array(slots[:T])
    ends = np.flatnonzero(np.diff(slots) != 1)
    src[ends[::3]] = [37, -1, 2 ** 31 - 1][T % 3]
    new = [bf16_bits(rng.standard_normal((37, 2, 64))) for _ in range(2)]
    _check(_pool(rng, pages, 2, 64, dtype, base=0.005), dtype, slots, *new, src=src)


@pytest.mark.parametrize("base", [1.0, 2.0 ** -110, 2.0 ** 90])
@pytest.mark.parametrize("d", [64, 128])
def test_fp8_scales_kept_raised_and_reset(d, base):
    """Maxima at fixed ratios of the page's scale, midpoints between codes among the requantised rows; scales out
    of the range that quotients by the inverse cover; zeros."""
    say(f"slot fp8 scales d {d} base {base:g}")
    rng = np.random.default_rng(d)
    ratios = [0.5, 1.0, 2.0, 1.5, 1.25, 7.0, 1.0078125, 0.0]
    slots, rows = [], []
    for page, (r, ratio) in enumerate((r, x) for r in (0, 1, 7, 13) for x in ratios):
        for i in range(3):
            slots.append(page * 16 + r + i)
            x = np.clip(rng.standard_normal((2, d)), -4, 4) * (ratio > 0)
            x[:, 5] = 448.0 * ratio if i == 1 else 0.0
            rows.append(np.clip(x * base, -3e38, 3e38))
    pool = _pool(rng, 4 * len(ratios), 2, d, "fp8")
    pool["k_scale"][:], pool["v_scale"][:] = base, base
    new = bf16_bits(np.array(rows))
    _check(pool, "fp8", slots, new, new[:, ::-1].copy())


def test_nan_and_infinite_rows():
    """As in the append: a NaN does not enter the maximum and takes the saturated code with its sign."""
    rng = np.random.default_rng(5)
    new = bf16_bits(rng.standard_normal((12, 1, 64)))
    new[1, 0, 3], new[6, 0, 9], new[7, 0, 1] = 0x7FC0, 0xFFC0, 0x7F81
    new[10] = 0x7FC0
    slots = list(range(4, 8)) + list(range(16, 20)) + list(range(40, 44))
    _check(_pool(rng, 3, 1, 64, "fp8", base=0.01), "fp8", slots, new, new.copy())
    _check(_pool(rng, 3, 1, 64, "bf16"), "bf16", slots, new, new.copy())


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
def test_single_rows_equal_the_append(dtype):
    import paper_2606_26997_amd as rp
    wl = make_workload(num_q_heads=8, num_kv_heads=4, head_dim=128, seq_to_group=[0] * 48, prefix_lens=[3],
                       resp_lens=np.arange(48), seed=3, append=True, kv_dtype=dtype)
    a, b = (rp.DeviceBatch.from_workload(wl) for _ in range(2))
    a.kv_append()
    t = torch.arange(48, device="cuda")
    slots = (b.resp_block_table[t, t // 16] * 16 + t % 16).int()
    b.write_slots(slots, b.k_new, b.v_new)
    torch.cuda.synchronize()
    for x, y in ((a.k_pages, b.k_pages), (a.v_pages, b.v_pages), (a.k_scale, b.k_scale), (a.v_scale, b.v_scale)):
        if x is not None:
            np.testing.assert_array_equal(_host(x), _host(y))


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
def test_prompts_equal_the_prefill_write(dtype):
    import paper_2606_26997_amd as rp
    w = make_prefill_workload(num_q_heads=4, num_kv_heads=4, head_dim=64, prefix_lens=[1, 16, 0, 100, 333], seed=2,
                              kv_dtype=dtype)
    a, b = (rp.PrefillBatch.from_workload(w) for _ in range(2))
    a.kv_write()
    slots = [w.prefix_block_table[g, t // 16] * 16 + t % 16 for g, n in enumerate(np.diff(w.prefix_offs)) for t in range(n)]
    rp.kv_write_slots(b.kv, torch.tensor(slots, dtype=torch.int32, device="cuda"), b.k, b.v)
    torch.cuda.synchronize()
    for x, y in ((a.k_pages, b.k_pages), (a.v_pages, b.v_pages), (a.k_scale, b.k_scale), (a.v_scale, b.v_scale)):
        if x is not None:
            np.testing.assert_array_equal(_host(x), _host(y))


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
def test_a_long_list(dtype):
    """Far more entries than a launch holds at once, in pages all over the pool."""
    say(f"slot long list {dtype}")
    rng = np.random.default_rng(6)
    pages = 1500
    order = rng.permutation(pages)
    slots = np.concatenate([p * 16 + np.arange(16)[int(rng.integers(0, 3)):] for p in order])
    new = [bf16_bits(rng.standard_normal((len(slots), 2, 128))) for _ in range(2)]
    _check(_pool(rng, pages, 2, 128, dtype, base=0.01), dtype, slots, *new, repeat=False)


def test_slots_of_pages_beyond_32_bits_and_a_graph():
    """A page whose byte offset passes 2^32, written by a captured call that is replayed after the list changed."""
    import paper_2606_26997_amd as rp
    say("slot write in a pool of 9 GiB")
    n = 576000
    k, v = (torch.zeros(n, 2, 16, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    new = torch.randn(5, 2, 128, device="cuda").bfloat16()
    slots = torch.tensor([(n - 1) * 16 + 3, 7, (n - 2) * 16 + 15, -1, 40], dtype=torch.int32, device="cuda")
    kv = rp.paged_kv(k, v)
    rp.kv_write_slots(kv, slots, new, new)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        rp.kv_write_slots(kv, slots, new, new)
    for i in range(3):
        slots.add_(16 * (slots % 16 == 7))
        k.zero_()
        v.zero_()
        g.replay()
        torch.cuda.synchronize()
        for pool in (k, v):
            for j, x in enumerate(slots.tolist()):
                if x >= 0:
                    assert torch.equal(pool[x // 16, :, x % 16], new[j])
            assert int((pool[n - 2:] != 0).any(3).sum() + (pool[:16] != 0).any(3).sum()) == 8
