"""K/V rows written into a paged pool by slot, and block tables grown and shrunk from lengths.

A slot is ``page * ps + row``. fp8 pools: a run is a maximal stretch of list entries, skipped ones left out, whose
slots rise inside a page; with ``amax`` over the run's rows (fp32, NaN left out), a run from row 0 sets
``scale = amax / 448`` (1 if 0), one from row ``r > 0`` keeps the scale if ``amax <= 448 * scale`` and else sets
``scale = amax / 448`` and requantises rows ``0..r-1`` from ``code * old``; rows are ``e4m3(x / scale)``, other
codes stay.
"""
import numpy as np

from .formats import bf16_to_f32, e4m3_encode, e4m3_to_f64

_F448 = np.float32(448.0)


def _encode(x):
    """e4m3 codes; a NaN takes the saturated code with its sign."""
    nan = np.isnan(x)
    codes = e4m3_encode(np.where(nan, np.float32(0), x))
    return np.where(nan, np.where(np.signbit(x), 0xFE, 0x7E), codes).astype(np.uint8)


def _runs(live, ps):
    """Every run of a list of (entry, slot): its entries and its slots."""
    runs = []
    for i, slot in live:
        if runs and runs[-1][1][-1] < slot and runs[-1][1][-1] // ps == slot // ps:
            runs[-1][0].append(i)
            runs[-1][1].append(slot)
        else:
            runs.append(([i], [slot]))
    return runs


def kv_write_slots(*, k_pages, v_pages, k_scale, v_scale, kv_dtype, page_size, slot_map, k_new, v_new,
                   src_rows=None):
    """Copies of the pools (and scales) with the list's rows written."""
    pools = [k_pages.copy(), v_pages.copy()]
    scales = [None if x is None else x.copy() for x in (k_scale, v_scale)]
    num_pages, hkv = k_pages.shape[:2]
    src = np.arange(len(slot_map)) if src_rows is None else np.asarray(src_rows)
    live = [(i, int(x)) for i, x in enumerate(slot_map)
            if 0 <= x < num_pages * page_size and 0 <= src[i] < len(k_new)]
    for entries, slots in _runs(live, page_size):
        page, r = divmod(slots[0], page_size)
        at = [x % page_size for x in slots]
        for pool, scale, new in ((pools[0], scales[0], k_new), (pools[1], scales[1], v_new)):
            rows = np.asarray(new)[src[entries]]
            for h in range(hkv):
                if kv_dtype == "bf16":
                    pool[page, h, at] = rows[:, h]
                    continue
                with np.errstate(invalid="ignore"):
                    x = bf16_to_f32(rows[:, h])
                    amax = np.float32(np.fmax.reduce(np.abs(x), axis=None, initial=np.float32(0)))
                    old = np.float32(scale[page, h])
                    now = old
                    if r == 0:
                        now = amax / _F448 if amax > 0 else np.float32(1.0)
                    elif not amax <= _F448 * old:
                        now = amax / _F448
                        before = e4m3_to_f64(pool[page, h, :r]).astype(np.float32) * old
                        pool[page, h, :r] = _encode(before / now)
                    pool[page, h, at] = _encode(x / now)
                scale[page, h] = now
    return pools[0], pools[1], scales[0], scales[1]


def page_tables_resize(block_table, free_pages, free_count, old_lens, new_lens, page_size=16, max_slots=None):
    """One page at a time: ``(status, block_table, free_pages, free_count, slot_offs, slots)``, status as
    {code, pages taken, pages given back, new tokens}; codes 0 done, 1 no pages, 2 bad length, 3 no slots,
    4 bad free list."""
    table, stack, count = block_table.copy(), free_pages.copy(), int(free_count)
    S, width = table.shape
    pages = lambda n: -(-int(n) // page_size)
    fits = [0 <= o <= width * page_size and 0 <= n <= width * page_size for o, n in zip(old_lens, new_lens)]
    moves = [(pages(o), pages(n)) if ok else (0, 0) for o, n, ok in zip(old_lens, new_lens, fits)]
    back, take = (sum(max(d * (h - w), 0) for h, w in moves) for d in (1, -1))
    fresh = [max(int(n) - int(o), 0) if ok else 0 for o, n, ok in zip(old_lens, new_lens, fits)]
    code = 0
    if not all(fits):
        code = 2
    elif count < 0 or count + back > len(stack):
        code = 4
    elif take > count + back:
        code = 1
    elif max_slots is not None and sum(fresh) > max_slots:
        code = 3
    status = [code, take, back, sum(fresh)]
    if code:
        return status, table, stack, count, np.zeros(S + 1, np.int64), np.zeros(0, np.int64)
    given = []
    for s, (have, want) in enumerate(moves):
        for p in range(want, have):
            given.append(int(table[s, p]))
            table[s, p] = -1
    for page in reversed(given):
        stack[count] = page
        count += 1
    for s, (have, want) in enumerate(moves):
        for p in range(have, want):
            count -= 1
            table[s, p] = stack[count]
    slots = [int(table[s, t // page_size]) * page_size + t % page_size
             for s in range(S) for t in range(int(old_lens[s]), int(new_lens[s]))]
    return status, table, stack, count, np.concatenate([[0], np.cumsum(fresh)]).astype(np.int64), \
        np.array(slots, np.int64)
