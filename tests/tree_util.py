"""Shared helpers of the GPU tests of drafted token trees: random trees, the HIP path against the oracle."""
import sys

import numpy as np
import torch

import oracle
from tests.paged import bf16_bits


def say(msg):
    print(f"[case] {msg}", flush=True)
    sys.stdout.flush()


def random_trees(rng, counts):
    """Packed masks of a random tree per sequence: a draft sees its ancestors and itself."""
    masks = []
    for n in counts:
        own = []
        for i in range(n):
            parent = int(rng.integers(-1, i)) if i else -1
            own.append((own[parent] if parent >= 0 else 0) | 1 << i)
        masks += own
    return np.array(masks, np.uint64)


def drafts_for(wl, counts, seed, masks=None):
    rng = np.random.default_rng(seed)
    offs = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    T = int(offs[-1])
    q = bf16_bits(rng.standard_normal((T, wl.num_q_heads, wl.head_dim)))
    k, v = (bf16_bits(rng.standard_normal((T, wl.num_kv_heads, wl.head_dim))) for _ in range(2))
    return dict(draft_offs=offs, masks=random_trees(rng, counts) if masks is None else masks, q=q, k_draft=k, v_draft=v)


def run_tree(wl, dr, max_drafts, batch=None):
    """The HIP path on a workspace and outputs full of NaN; (batch, out, lse) on the host in fp64."""
    import paper_2606_26997_amd as rp
    b = rp.DeviceBatch.from_workload(wl) if batch is None else batch
    b.set_drafts(**{**dr, "masks": dr["masks"].view(np.int64)}, max_drafts=max_drafts)
    b.draft_workspace.fill_(0xFF)
    b.draft_out.fill_(float("nan"))
    b.draft_lse.fill_(float("nan"))
    b.tree_attention()
    torch.cuda.synchronize()
    return b, b.draft_out.float().cpu().numpy().astype(np.float64), b.draft_lse.cpu().numpy().astype(np.float64)


def compare_tree(out, lse, ref, d, label):
    """Tolerances by arithmetic. Scores: d products of exact bf16 values summed in fp32, off by at most
    d 2^-24 reach; the lse follows them, and exp2, log2 and the sums add less than 2^-20 (|lse| + 16) (a hundred
    fp32 steps). Output: probabilities rounded to bf16 (at most 2^-8 each, numerator and denominator) move it by
    2 2^-8 spread, score errors by 2 d 2^-24 reach spread, its own rounding to bf16 by 2^-8 |out|, and fp32 sums by
    less than 2^-14 spread."""
    r_out, r_lse, spread, reach = ref
    fin = np.isfinite(r_lse)
    assert np.array_equal(fin, np.isfinite(lse)), label
    assert np.all(out[~fin] == 0) and np.all(lse[~fin] == -np.inf), label
    score = d * 2.0 ** -24 * reach
    lim = score + 2.0 ** -20 * (np.abs(r_lse) + 16)
    off = np.abs(lse[fin] - r_lse[fin])
    assert np.all(off <= lim[fin]), f"{label}: lse off by {off.max():.3e}"
    tol = 2.0 ** -8 * np.abs(r_out) + (2 * 2.0 ** -8 + 2.0 ** -14 + 2 * score[..., None]) * spread
    worst = (np.abs(out - r_out) / np.maximum(tol, 1e-30)).max(initial=0)
    assert worst <= 1.0, f"{label}: out at {worst:.2f} of its tolerance"
    norm = np.linalg.norm(r_out)
    rel = np.linalg.norm(out - r_out) / norm if norm else 0.0
    # Independent roundings of the sizes above: a uniform one has an rms of its half step over sqrt 3.
    assert rel <= 5e-3, f"{label}: rel {rel:.2e}"


def check_tree(wl, counts, seed, label, max_drafts=None, masks=None):
    say(label)
    dr = drafts_for(wl, counts, seed, masks)
    b, out, lse = run_tree(wl, dr, max(counts) if max_drafts is None else max_drafts)
    compare_tree(out, lse, oracle.tree_for_workload(wl, **dr), wl.head_dim, label)
    return b, dr, out, lse
