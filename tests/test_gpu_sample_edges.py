"""Sampling on the GPU where its forms could part from the definition: many rows that draw alike."""
import numpy as np
import pytest
import torch

import oracle
from tests.rows_util import dev, empty, logits, say, workspace

pytestmark = pytest.mark.gpu


def _draw(view, u, **how):
    """Tokens and both log-probabilities, in the tensors' own bits."""
    import paper_2606_26997_amd as rp
    n = view.shape[0]
    out = empty(n, torch.int32), empty(n), empty(n)
    given = {k: dev(v, torch.int32 if k == "top_k" else torch.float32) for k, v in how.items()}
    rp.sample_tokens(view, dev(u), *out, workspace=workspace(view), **given)
    torch.cuda.synchronize()
    return out


@pytest.mark.parametrize("n,V,dtype", [(2000, 4000, "bf16"), (700, 30000, "f16"), (200, 151936, "bf16"), (150, 151936, "bf16")])
def test_rows_alike_draw_alike(n, V, dtype):
    """One row n times with one random number, in each launch form: whatever the waves' pace, every workgroup takes the
    same way to the same token, call after call."""
    say(f"rows alike {n} x {V} {dtype}")
    rng = np.random.default_rng(V + n)
    x, one, _ = logits(rng, 1, V, dtype)
    view = one.repeat(n, 1)
    for how in (dict(top_k=50), dict(top_p=0.9), dict(top_p=0.4), dict(top_k=20, top_p=0.8), dict(top_k=100, min_p=0.01)):
        u = rng.random(1).astype(np.float32)
        want, _, _, margin = oracle.sample(x, u, **{k: np.array([v]) for k, v in how.items()})
        assert margin[0] > 1e-11
        alike = {k: np.full(n, v) for k, v in how.items()}
        for _ in range(5):
            tokens, lp, kept = _draw(view, np.repeat(u, n), **alike)
            assert (tokens == int(want[0])).all(), how
            assert (lp == lp[0]).all() and (kept == kept[0]).all(), how
