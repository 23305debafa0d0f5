"""Sampling on the GPU where its forms could part from the definition: many rows that draw alike, borders
between sums that differ by a rounding, temperatures far from 1."""
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

import oracle
from tests.rows_util import dev, empty, logits, say, workspace
from tests.test_gpu_sample import _check

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


def _weight(x):
    """2^(x log2 e) by the kernel's polynomial, products and sums rounded once together."""
    y = max(x * 1.4426950408889634, -1500.0)
    n = round(y)
    f = Fraction(y) - n
    p = 0.0
    for c in ("0x1.b63881021ff95p-24", "0x1.63d13637e6ed6p-20", "0x1.ffcb95154c637p-17", "0x1.4308ac85a8c94p-13",
              "0x1.5d87fe86fea1bp-10", "0x1.3b2ab7181b769p-7", "0x1.c6b08d7047e52p-5", "0x1.ebfbdff823cedp-3",
              "0x1.62e42fefa39efp-1", "0x1p0"):
        p = float(Fraction(p) * f + Fraction(float.fromhex(c)))
    return math.ldexp(p, n)


def _butterfly(s):
    """A wave's sum [..][64], lane by lane."""
    for o in (32, 16, 8, 4, 2, 1):
        s = s + s[..., np.arange(64) ^ o]
    return s[..., 0]


def _scan(s):
    """Running sums over the lanes, by doubling."""
    for o in (1, 2, 4, 8, 16, 32):
        if o < s.shape[-1]:
            s = np.concatenate([s[..., :o], s[..., o:] + s[..., :-o]], -1)
    return s


def _vector_sums(w):
    s = np.zeros(w.shape[:-1])
    for e in range(w.shape[-1]):
        s = s + w[..., e]
    return s


def _vectors(rng, count):
    """Logits in steps of 1/32 that bf16 holds, 0 the largest of every vector."""
    x = -rng.integers(1, 97, (count, 8)) / 32.0
    x[:, 0] = 0.0
    return x


def _gap_in_a_wave(rng, w_of):
    """Rows of two stretches of 64 vectors; behind the first one's last kept vector the scan's sums differ by a rounding,
    and half of the row's weight lies between them."""
    rows = []
    while len(rows) < 16:
        live = int(rng.integers(5, 40))
        at = np.sort(rng.permutation(60)[:live])
        x = np.full((128, 8), -np.inf)
        x[at] = _vectors(rng, live)
        sums = _vector_sums(w_of(x[:64]))
        upto, D0 = _scan(sums), _butterfly(sums)
        least, most = upto[at[-1]], upto[at[-1] + 1:].max()
        if not (D0 > least and most > least):
            continue
        for _ in range(200):
            x[64:] = -np.inf
            x[64 + rng.permutation(64)[:live]] = x[at][rng.permutation(live)]
            target = 0.5 * (D0 + _butterfly(_vector_sums(w_of(x[64:]))))
            over = np.flatnonzero(upto > target)
            if D0 > target and over.size and over[0] > at[-1]:
                rows.append(x.reshape(-1).copy())
                break
    return np.array(rows)


def _gap_between_stretches(rng, w_of):
    """Rows of eight stretches of 128 vectors, the fourth masked, whose running sum is a rounding above the third's; half of
    the row's weight lies between them."""
    rows = []
    while len(rows) < 16:
        x = np.full((8, 2, 64, 8), -np.inf)
        x[:3] = _vectors(rng, 3 * 128).reshape(3, 2, 64, 8)
        for _ in range(50):
            x[4:7] = x[:3].reshape(-1, 8)[rng.permutation(3 * 128)].reshape(3, 2, 64, 8)
            D = _vector_sums(w_of(x))
            D = _butterfly(D[:, 0] + D[:, 1])
            upto = _scan(D)
            target = 0.5 * upto[-1]
            if np.flatnonzero(upto > target)[0] == 3:
                rows.append(x.reshape(-1).copy())
                break
    return np.array(rows)


@pytest.mark.parametrize("rows_of", [_gap_in_a_wave, _gap_between_stretches])
def test_a_border_between_two_roundings(rows_of):
    """Running sums that were added in different orders may differ by a rounding from one masked token to the next; a
    border that falls between two such sums still draws a token that can occur."""
    say(f"borders: {rows_of.__name__}")
    table = np.array([_weight(-i / 32.0) for i in range(97)] + [0.0])
    w_of = lambda x: table[np.where(np.isfinite(x), -32 * np.maximum(x, -3.0), 97).astype(int)]
    x = rows_of(np.random.default_rng(17), w_of)
    view = torch.from_numpy(x).to("cuda", torch.bfloat16)
    tokens = _draw(view, np.full(len(x), 0.5))[0].tolist()
    assert all(0 <= t < x.shape[1] and r[t] > -np.inf for t, r in zip(tokens, x)), tokens
    # It is one of the two beside the border: exact arithmetic does not tell which.
    for t, r in zip(tokens, x):
        w = np.exp(r)
        before, upto = w[:t].sum() / w.sum(), w[:t + 1].sum() / w.sum()
        assert before - 1e-12 <= 0.5 <= upto + 1e-12


@pytest.mark.parametrize("masked", [0, 3])
@pytest.mark.parametrize("n,V,dtype", [(10, 9, "f16"), (10, 9000, "bf16"), (10, 70001, "f16"), (10, 60000, "f32")])
def test_temperatures_without_a_bound(n, V, dtype, masked):
    """T = +inf makes every token that can occur equally likely, whatever is filtered; temperatures at both ends of fp32."""
    say(f"temperature inf {n} x {V} {dtype} masked {masked}")
    rng = np.random.default_rng(V + masked)
    x, view, _ = logits(rng, n, V, dtype, masked=masked)
    live = V - masked
    # Shares of a vocabulary that are no whole number of tokens.
    p = ((rng.integers(0, live, n) + 0.5) / live).astype(np.float32)
    k = np.array([1, 2, 3, 40, 200, 700, live // 2, live - 1, live, V + 1], np.int32)
    q = np.array([0, 1e-30, 0.1, 0.5, 0.999, 1, 1, 0.3, 2, 0.7], np.float32)
    half = np.full(n, 0.5 + 0.25 / live, np.float32)
    for T in (np.full(n, np.inf, np.float32), np.array([np.inf, 1e30, 3e38, 1e38, 2e30, 1e-39, 1e-45, 1e-30, 1e10, np.inf], np.float32)):
        u = rng.random(n).astype(np.float32)
        for how in (dict(top_k=k), dict(top_p=p), dict(min_p=q), dict(top_k=k, top_p=half), dict(top_k=k, min_p=q),
                    dict(top_p=p, min_p=q), dict(top_k=k, top_p=half, min_p=q)):
            _check(x, view, u, dict(temperature=T, **how), str(list(how)))


def test_temperatures_of_rows_at_the_ends_of_fp32():
    """Logits further apart than fp32's largest number: at T = 1e38 each counts."""
    say("temperature, logits of +-3e38")
    n, V = 6, 5000
    view = torch.linspace(-3.2e38, 3.2e38, V, dtype=torch.float64).float().cuda().repeat(n, 1)
    x = view.double().cpu().numpy()
    T = np.array([1e38, 3e38, np.inf, 1e37, 1e36, 2e38], np.float32)
    u = np.random.default_rng(2).random(n).astype(np.float32)
    f = lambda v: np.full(n, v, np.float32)
    for how in (dict(), dict(top_k=np.full(n, 70, np.int32)), dict(top_p=f(0.37)), dict(min_p=f(0.3))):
        _check(x, view, u, dict(temperature=T, **how), str(list(how)))
