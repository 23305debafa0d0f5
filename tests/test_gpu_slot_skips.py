"""Slot writes on the GPU whose lists have skipped entries inside a page's run, and lists so long that a wave takes
up to 16 entries: bytes and scales equal the oracle's. A wave of an fp8 write takes one entry for each 12288 that
list entries x kv-heads x 2 amount to, rounded up, at most 16."""
import numpy as np
import pytest

from tests.paged import bf16_bits
from tests.slot_lists import accepted_in_place, pool, skipping_list
from tests.test_gpu_slots import _check
from tests.tree_util import say

pytestmark = pytest.mark.gpu

# (entries, kv-heads, head size, entries per wave)
SHARES = [(70, 1, 128, 1), (900, 2, 64, 1), (1300, 8, 64, 2), (3800, 4, 128, 3), (5800, 8, 64, 8), (12400, 8, 64, 16)]


def _share(entries, hkv):
    return min(16, -(-2 * entries * hkv // 12288))


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("n,hkv,d,share", SHARES)
def test_skipped_entries_inside_runs(n, hkv, d, share, dtype):
    say(f"slot skips {n} hkv {hkv} d {d} {dtype}")
    rng = np.random.default_rng(n)
    slots, src, pages = skipping_list(rng, n, rows=301)
    assert _share(len(slots), hkv) == share
    new = [bf16_bits(rng.standard_normal((301, hkv, d)) * np.exp(rng.standard_normal((301, 1, 1)))) for _ in range(2)]
    _check(pool(rng, pages, hkv, d, dtype, base=0.005), dtype, slots, *new, src=src)


@pytest.mark.parametrize("n,hkv,d,share", SHARES)
def test_runs_of_every_place_and_length_in_every_share(n, hkv, d, share):
    """No entry skipped; runs of every first row and length in any order, pages in any order, rows gathered."""
    say(f"slot shares {n} hkv {hkv} d {d}")
    rng = np.random.default_rng(n + 1)
    runs, slots = [(r, k) for r in range(16) for k in range(1, 17 - r)], []
    pages = rng.permutation(-(-n // 6) * 2)
    for i, page in enumerate(pages):
        r, k = runs[int(rng.integers(0, len(runs)))]
        slots += range(page * 16 + r, page * 16 + r + k)
        if len(slots) >= n:
            break
    assert _share(len(slots), hkv) == share
    src = rng.integers(0, 301, len(slots))
    new = [bf16_bits(rng.standard_normal((301, hkv, d)) * np.exp(rng.standard_normal((301, 1, 1)))) for _ in range(2)]
    _check(pool(rng, len(pages), hkv, d, "fp8", base=0.005), "fp8", np.array(slots), *new, src=src)


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("drafts", [5, 16, 64])
def test_accepted_drafts_in_place(drafts, dtype):
    """-1 for the drafts that are not accepted, without a list of source rows, padded behind the last."""
    say(f"slots in place {drafts} {dtype}")
    rng = np.random.default_rng(drafts)
    slots, pages = accepted_in_place(rng, 40, drafts)
    slots = np.concatenate([slots, np.full(300, -1)])
    new = [bf16_bits(rng.standard_normal((len(slots), 4, 128))) for _ in range(2)]
    _check(pool(rng, pages, 4, 128, dtype, base=0.005), dtype, slots, *new)
