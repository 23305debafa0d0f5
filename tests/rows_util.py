"""Shared helpers of the GPU tests of rows of logits: buffers with guarded gaps, the calls, error bounds.

Bounds, with u = 2^-24 and rows of V logits: a kernel forms d = (x - max) log2(e) / T in fp32 (a subtraction, a
product, a rounded constant: 3 u relative) and 2^d (2 u), so a term of S = sum 2^d is off by (3 |z - max z| + 2) u,
and S, whose terms average |z - max z| <= ln V, by (3 ln V + 2) u and the additions of one thread (V / 2048 + 16
for workgroups of 256 threads and vectors of 8). ln S, and with it every log-probability, is off by that.
"""
import math
import sys

import numpy as np
import torch

U = 2.0 ** -24
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SENTINEL = -77.0


def say(msg):
    print(f"[case] {msg}", flush=True)
    sys.stdout.flush()


def half_step(dtype):
    return torch.finfo(DTYPES[dtype]).eps / 2


def guarded(n, V, dtype, pad=0, offset=0, device="cuda"):
    """A [n][V] view of rows `pad` elements apart, beginning `offset` elements into its buffer, and the buffer."""
    buf = torch.full((offset + n * (V + pad) + 17,), SENTINEL, dtype=DTYPES[dtype], device=device)
    return buf.as_strided((n, V), (V + pad, 1), offset), buf


def gaps_untouched(view, buf):
    mask = torch.ones(buf.shape, dtype=torch.bool, device=buf.device)
    mask.as_strided(view.shape, view.stride(), view.storage_offset()).fill_(False)
    return bool((buf[mask] == SENTINEL).all())


def logits(rng, n, V, dtype, *, masked=0, scale=2.5, peaks=4, pad=0, offset=0, levels=None):
    """Values of a case on the host (float64, as the type holds them) and on the GPU in a guarded buffer."""
    x = scale * rng.standard_normal((n, V))
    if levels:
        x = np.round(x * levels) / levels  # many equal logits
    for r in range(n):
        x[r, rng.integers(0, V, min(peaks, V))] += 6 * rng.random(min(peaks, V))
        if masked:
            x[r, rng.permutation(V)[:masked]] = -np.inf
    view, buf = guarded(n, V, dtype, pad, offset)
    view.copy_(torch.from_numpy(x).to(DTYPES[dtype]))
    return view.double().cpu().numpy(), view, buf


def dev(a, dtype=torch.float32):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to("cuda", dtype)


def empty(n, dtype=torch.float32):
    return torch.full((n,), -5, dtype=dtype, device="cuda")


def workspace(view):
    import paper_2606_26997_amd as rp
    size = rp.logits_workspace_size(view)
    return torch.full((size,), 255, dtype=torch.uint8, device="cuda") if size else None


def lse_bound(V):
    return (3 * math.log(V) + 2 + V / 2048 + 16) * U


def entropy_bound(V):
    """ln S, and ln 2 sum p d: terms off by (3 |z| + 4) u of |z|, sums as above; |z| and z^2 average at most
    ln V + 1 and (ln V + 2)^2."""
    L = math.log(V) + 2
    return lse_bound(V) * (1 + L) + (3 * L * L + 4 * L) * U


def f32(a):
    return torch.from_numpy(np.asarray(a)).float().double().numpy()
