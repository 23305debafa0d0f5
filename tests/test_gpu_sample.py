"""Sampling on the GPU against the float64 oracle: tokens equal it (no case's random number lies within 1e-11 of a
border), log-probabilities to the bounds of rows_util."""
import math

import numpy as np
import pytest
import torch

import oracle
from tests.rows_util import U, dev, empty, gaps_untouched, guarded, logits, lse_bound, say, workspace

pytestmark = pytest.mark.gpu


def _params(rng, n, filters):
    p = dict(temperature=None, top_k=None, top_p=None, min_p=None)
    if filters == "none":
        return p
    f = lambda a: np.asarray(a, np.float32)
    p["temperature"] = f(0.5 + rng.random(n))
    if filters in ("topk", "all"):
        p["top_k"] = rng.integers(0, 40, n).astype(np.int32)
    if filters in ("topp", "all"):
        p["top_p"] = f(0.3 + 0.75 * rng.random(n))
    if filters in ("minp", "all"):
        p["min_p"] = f(0.2 * rng.random(n) ** 2)
    if filters == "all":
        p["temperature"][rng.random(n) < 0.2] = 0.0
    return p


def _call(view, u, p, **kw):
    import paper_2606_26997_amd as rp
    n = view.shape[0]
    tokens, lp, kept = empty(n, torch.int32), empty(n), empty(n)
    rp.sample_tokens(view, dev(u), tokens, lp, kept, temperature=dev(p.get("temperature")),
                     top_k=dev(p.get("top_k"), torch.int32), top_p=dev(p.get("top_p")), min_p=dev(p.get("min_p")),
                     workspace=workspace(view), **kw)
    torch.cuda.synchronize()
    return tokens.cpu().numpy(), lp.double().cpu().numpy(), kept.double().cpu().numpy()


def _check(x, view, u, p, label, kept_bound=1e-10):
    got = _call(view, u, p)
    tok, lp, kept, margin = oracle.sample(x, u, **p)
    sure = margin > 1e-11
    assert sure.mean() > 0.99, f"{label}: inputs on borders"
    assert np.array_equal(got[0][sure], tok[sure]), f"{label}: tokens {got[0]} {tok}"
    same = got[0] == tok
    # One rounding to fp32 of what is held in 64 bits; ln of the whole row's sum may come from fp32 terms.
    for g, e, what, slack in ((got[1], lp, "logprobs", lse_bound(x.shape[1])), (got[2], kept, "kept", kept_bound)):
        fine = same & np.isfinite(e)
        assert np.array_equal(np.isnan(g[same]), np.isnan(e[same])) and np.array_equal(g[same & ~fine & ~np.isnan(e)], e[same & ~fine & ~np.isnan(e)]), (label, what)
        off = np.abs(g[fine] - e[fine]) - (U * np.abs(e[fine]) + slack)
        assert off.size == 0 or off.max() <= 0, f"{label} {what}: {off.max()}"


SIZES = [  # rows, vocab, dtype, pad, offset, masked
    (1, 1, "bf16", 0, 0, 0), (3, 2, "f32", 1, 1, 0), (5, 7, "bf16", 2, 3, 2), (64, 63, "f16", 0, 1, 5),
    (300, 40, "bf16", 0, 0, 0), (4, 1000, "f32", 0, 0, 900), (7, 8191, "bf16", 1, 0, 0), (2, 32769, "f16", 7, 5, 100),
    (3, 50257, "f32", 0, 0, 0), (2, 151936, "bf16", 0, 0, 267), (1, 163841, "bf16", 0, 1, 0), (40, 20000, "bf16", 0, 0, 0),
]


@pytest.mark.parametrize("filters", ["none", "topk", "topp", "minp", "all"])
@pytest.mark.parametrize("n,V,dtype,pad,offset,masked", SIZES)
def test_sampling(n, V, dtype, pad, offset, masked, filters):
    say(f"sample {n} x {V} {dtype} pad {pad} offset {offset} masked {masked} {filters}")
    rng = np.random.default_rng(V * 5 + n)
    x, view, buf = logits(rng, n, V, dtype, masked=masked, pad=pad, offset=offset)
    _check(x, view, rng.random(n).astype(np.float32), _params(rng, n, filters), filters)
    assert gaps_untouched(view, buf)


@pytest.mark.parametrize("scale", [0.5, 2.5])
@pytest.mark.parametrize("n,V,dtype", [(90, 90001, "bf16"), (170, 90001, "f16"), (270, 40001, "f32"), (520, 9001, "bf16")])
def test_batches_that_fill_the_units(n, V, dtype, scale):
    """Rows scanned apart above 64 of them, and a workgroup of each size to a row; flat rows and rows with peaks."""
    say(f"batch {n} x {V} {dtype} scale {scale}")
    rng = np.random.default_rng(n)
    x, view, buf = logits(rng, n, V, dtype, scale=scale, peaks=4 if scale > 1 else 0)
    u = rng.random(n).astype(np.float32)
    for filters in ("none", "topp", "all"):
        _check(x, view, u, _params(rng, n, filters), filters)
    assert gaps_untouched(view, buf)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("filters", ["topk", "topp", "minp", "all"])
def test_many_equal_logits(dtype, filters):
    """The cut falls among equals: the lowest indices are kept."""
    say(f"equal logits {dtype} {filters}")
    rng = np.random.default_rng(3)
    x, view, _ = logits(rng, 60, 3000, dtype, levels=2, peaks=0)
    _check(x, view, rng.random(60).astype(np.float32), _params(rng, 60, filters), filters)
    flat = torch.zeros(8, 5000, dtype=view.dtype, device="cuda")
    k = np.array([1, 2, 3, 63, 64, 65, 4999, 5000], np.int32)
    u = np.full(8, 0.99999, np.float32)
    _check(flat.double().cpu().numpy(), flat, u, dict(top_k=k), "flat, top-k")
    _check(flat.double().cpu().numpy(), flat, u, dict(top_p=(k / 5000).astype(np.float32) * np.float32(0.9993)), "flat, top-p")


@pytest.mark.parametrize("V", [100, 20000, 160000])
def test_large_nuclei(V):
    """Flat rows: half of the vocabulary and more is kept; top-k far above a list's length."""
    say(f"large nuclei {V}")
    rng = np.random.default_rng(V)
    n = 6
    x, view, _ = logits(rng, n, V, "bf16", scale=0.5, peaks=0)
    u = rng.random(n).astype(np.float32)
    _check(x, view, u, dict(top_p=np.array([0.5, 0.9, 0.99, 0.999, 0.9999, 0.1], np.float32)), "top-p")
    _check(x, view, u, dict(top_k=np.array([V // 2, V // 3, V - 1, V, V + 5, 5000], np.int32)), "top-k")
    _check(x, view, u, dict(top_k=np.array([V // 2] * n, np.int32), top_p=np.full(n, 0.7, np.float32),
                            min_p=np.array([0, 0.01, 0.05, 0.1, 0.2, 0.3], np.float32)), "all")


@pytest.mark.parametrize("V", [5, 1500, 40000])
def test_rows_that_are_empty_or_bad(V):
    say(f"bad rows {V}")
    rng = np.random.default_rng(11)
    x, view, _ = logits(rng, 8, V, "bf16")
    view[0] = -math.inf
    view[1, V // 2] = math.nan
    view[2, V - 1] = math.inf
    view[3] = -math.inf
    view[3, V - 1] = 2.0
    view[4] = math.nan
    view[5, 1:] = -3.0e38
    x = view.double().cpu().numpy()
    for p in (dict(), dict(temperature=np.zeros(8, np.float32)), dict(top_k=np.full(8, 2, np.int32)),
              dict(top_p=np.full(8, 0.5, np.float32)), dict(min_p=np.full(8, 0.1, np.float32)),
              dict(top_k=np.full(8, 3, np.int32), top_p=np.full(8, 0.9, np.float32), min_p=np.full(8, 0.5, np.float32))):
        _check(x, view, rng.random(8).astype(np.float32), p, str(list(p)))


@pytest.mark.parametrize("V", [9, 9000])
def test_parameters_out_of_the_ordinary(V):
    say(f"odd parameters {V}")
    rng = np.random.default_rng(5)
    f = lambda *a: np.array(a, np.float32)
    x, view, _ = logits(rng, 8, V, "f16")
    u = f(0.0, 1.0, -1.0, math.nan, 5.0, 1 - 2.0 ** -24, 0.5, math.inf)
    _check(x, view, u, dict(), "u")
    _check(x, view, u, dict(top_k=np.full(8, 3, np.int32)), "u, top-k")
    u = rng.random(8).astype(np.float32)
    _check(x, view, u, dict(temperature=f(math.inf, 1e30, 1e-30, math.nan, -0.0, 1e-40, 100, 0.01)), "temperature")
    _check(x, view, u, dict(top_p=f(0, -1, 1, 2, math.nan, 1e-30, 1 - 2.0 ** -24, math.inf)), "top-p")
    _check(x, view, u, dict(top_k=np.array([0, -1, 1, V, V + 1, 2 ** 31 - 1, -2 ** 31, 2], np.int32)), "top-k")
    _check(x, view, u, dict(min_p=f(0, -1, 1, 2, math.nan, 1e-30, 0.999, math.inf)), "min-p")


def test_large_vocabulary_and_optional_outputs():
    import paper_2606_26997_amd as rp
    say("vocabulary of 1048576")
    rng = np.random.default_rng(8)
    x, view, _ = logits(rng, 1, 1 << 20, "f32", peaks=200)
    u = f32 = rng.random(1).astype(np.float32)
    for p in (dict(), dict(top_k=np.array([700], np.int32), top_p=np.array([0.95], np.float32))):
        _check(x, view, u, p, str(list(p)))
    tokens = empty(1, torch.int32)
    rp.sample_tokens(view, dev(u), tokens, workspace=workspace(view))
    assert tokens.item() == oracle.sample(x, f32)[0][0]


def test_the_same_call_twice_and_on_another_stream():
    import paper_2606_26997_amd as rp
    say("repeats and streams")
    rng = np.random.default_rng(21)
    n, V = 20, 30000
    x, view, _ = logits(rng, n, V, "bf16")
    p = _params(rng, n, "all")
    u = rng.random(n).astype(np.float32)
    first = _call(view, u, p)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = _call(view, u, p)
    third = _call(view, u, p, stream=0)
    for a, b, c in zip(first, second, third):
        assert np.array_equal(a, b, equal_nan=True) and np.array_equal(a, c, equal_nan=True)
    out = empty(n, torch.int32)
    rp.sample_tokens(view[:0], dev(u[:0]), out[:0])
    assert (out == -5).all()


def test_the_drawn_tokens_follow_the_distribution():
    """4096 rows of one distribution with evenly spaced random numbers: each token as often as its probability says."""
    say("distribution")
    rng = np.random.default_rng(2)
    n, V = 4096, 50
    x, one, _ = logits(rng, 1, V, "bf16", scale=1.0, peaks=0)
    view = one.repeat(n, 1)
    u = ((np.arange(n) + 0.5) / n).astype(np.float32)
    tok, lp, _ = _call(view, u, {})
    p = np.exp(oracle.token_logprobs(np.repeat(x, V, 0), np.arange(V))[0])
    assert np.abs(np.bincount(tok, minlength=V) - n * p).max() <= 1.01
    assert np.allclose(np.exp(lp), p[tok], atol=1e-6)
