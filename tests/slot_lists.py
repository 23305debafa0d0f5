"""Pools and lists of slots for the tests of slot writes."""
import numpy as np


def pool(rng, pages, hkv, d, dtype, base=1.0):
    if dtype == "bf16":
        k, v = (rng.integers(0, 0x7F00, (pages, hkv, 16, d)).astype(np.uint16) for _ in range(2))
        return dict(k_pages=k, v_pages=v, k_scale=None, v_scale=None)
    k, v = (rng.integers(0, 0x7F, (pages, hkv, 16, d)).astype(np.uint8) for _ in range(2))
    ks, vs = ((base * np.exp(0.5 * rng.standard_normal((pages, hkv)))).astype(np.float32) for _ in range(2))
    return dict(k_pages=k, v_pages=v, k_scale=ks, v_scale=vs)


def skipping_list(rng, n, rows):
    """At least n entries, (slots, source rows, pages of the pool): one run per page, of every first row and length,
    in pages in any order; skipped entries between and inside runs, by their slot (-1 and others outside the pool)
    or by their source row, which may leave a gap of rows in the page. The first and last entry of a page are
    at most 63 places apart, some of them exactly so many."""
    runs = n // 4 + 2  # more than fit: the pool holds some pages that nothing touches
    order, slots, src = rng.permutation(runs), [], []
    outside = [-1, -2 ** 31, runs * 16, 2 ** 31 - 1]
    for i, page in enumerate(order):
        r = int(rng.integers(0, 16))
        run = list(range(page * 16 + r, page * 16 + r + int(rng.integers(1, 17 - r))))
        own = [int(x) for x in rng.integers(0, rows, len(run))]
        for j in range(len(run)):
            if rng.random() < 0.1:
                own[j] = [rows, -1, 2 ** 31 - 1, -2 ** 31][int(rng.integers(0, 4))]
        kind = rng.random()
        room = {0: 0, 1: int(rng.integers(1, 5)), 2: 64 - len(run)}[0 if kind < 0.4 else 1 if kind < 0.9 else 2]
        for _ in range(room if len(run) > 1 else 0):
            at = int(rng.integers(1, len(run)))
            run.insert(at, outside[int(rng.integers(0, 4))])
            own.insert(at, int(rng.integers(0, rows)))
        if rng.random() < 0.3:
            run.append(-1)
            own.append(0)
        slots += run
        src += own
        if len(slots) >= n and i >= 3:
            break
    return np.array(slots, np.int64), np.array(src, np.int64), runs


def accepted_in_place(rng, seqs, drafts):
    """Slots of the drafts of every sequence that are accepted, -1 for the others, in the drafts' own order; each
    sequence goes on behind some rows of a page of its own and into the next: (slots, pages of the pool)."""
    slots, per = [], (15 + drafts) // 16 + 1
    for s in range(seqs):
        at = s * per * 16 + int(rng.integers(0, 16))
        for yes in rng.random(drafts) < 0.5:
            slots.append(at if yes else -1)
            at += int(yes)
    return np.array(slots, np.int64), per * seqs
