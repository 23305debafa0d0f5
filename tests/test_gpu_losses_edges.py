"""Losses over rows of logits on the GPU at the ends of their ranges, against the float64 oracle: a list far above all other
tokens, a teacher's values that are no numbers, temperatures past fp32's range, logits further apart than that,
ratios that are no finite numbers."""
import math

import numpy as np
import pytest
import torch

import oracle
from tests.rows_util import U, dev, empty, entropy_bound, f32, guarded, half_step, logits, lse_bound, say, workspace
from tests.test_gpu_losses import _distill_run, _near, _policy_case, _policy_check, _policy_run

pytestmark = pytest.mark.gpu


def _far_check(x, dtype, ids, values, kind, w, T, got, what):
    """From logarithms: with m_o the largest logit outside the list and S_o the sum of exp((x - m_o) / T) there (off by
    lse_bound relative, its terms by (3 z + 4) u), q_o = S_o exp((m_o - m) / T) / s and the gradient outside is
    w / T e_i / S_o times a number of the row that is as exact as q_o; sums over the list are in 64 bits."""
    V, lb = x.shape[1], lse_bound(x.shape[1])
    loss, grad = oracle.distill_loss(x, ids, values, kind=kind, weights=w, temperature=T)
    tiny = 2.0 ** -25 if dtype == "f16" else 1e-37
    for r in range(len(x)):
        others = np.isfinite(x[r])
        others[ids[r]] = False
        z = np.where(others, (x[r][others].max() - np.where(others, x[r], 0.0)) / T, 0.0)
        l = oracle.rows.log_softmax(x[r], T)
        t, lq = values[r].astype(np.float64), l[ids[r]]
        qo, lqo = np.exp(l[others]).sum(), np.abs(oracle.rows.log_sum(l[others]))
        if kind == "topk":
            size, listed = 1.0, np.exp(lq)
        elif kind == "tail":
            size, listed = np.exp(t).sum() + 1.0, np.exp(lq) * (np.exp(t).sum() + 1)
        else:
            size = (np.exp(lq) * (np.abs(lq) + np.abs(t) + 1)).sum() + qo * (lqo + 17)
            listed = np.exp(lq) * (np.abs(lq) + np.abs(t) + 1 + size)
        _near(got[0][r:r + 1], loss[r:r + 1], w[r] * 2 * size * lb + U * abs(loss[r]) + w[r] * 1e-12, f"{what} losses")
        bound = (3 * z + 8) * U * np.abs(grad[r]) + 2 * lb * np.abs(grad[r])
        if kind != "topk":
            share = np.where(others, np.exp(-z), 0.0)
            bound += w[r] / T * share / share.sum() * qo * 2 * lb * (2.0 if kind == "tail" else lqo + 18 + size)
        bound[ids[r]] += w[r] / T * listed * 2 * lb
        _near(got[1][r], grad[r], bound + half_step(dtype) * 1.01 * np.abs(grad[r]) + tiny, f"{what} dlogits")


@pytest.mark.parametrize("kind", ["topk", "tail", "reverse"])
@pytest.mark.parametrize("V,dtype,masked", [(8, "f32", 0), (3000, "bf16", 7), (40001, "f32", 100), (140000, "f16", 0)])
def test_tokens_far_below_the_list(V, dtype, masked, kind):
    """What is outside the list keeps its class however small its mass: gaps of 80 and more, also through temperatures
    below 1, and a weight over T that a factor of the row's maximum would take past fp32's range."""
    say(f"far outside {V} {dtype} masked {masked} {kind}")
    rng = np.random.default_rng(V)
    for gap, T, weight in ((30.0, 1.0, 1.0), (80.0, 1.0, 1.0), (87.0, 1.0, 30.0), (90.0, 1.0, 1.0), (103.0, 1.0, 500.0),
                           (200.0, 1.0, 1.0), (900.0, 1.0, 1.0), (20.0, 0.2, 3.0), (9.0, 0.1, 10.0), (90.0, 0.1, 1.0)):
        n, k = 3, min(3, V // 4)
        view, _ = guarded(n, V, dtype)
        x = 0.5 * T * rng.standard_normal((n, V))
        ids = np.stack([rng.permutation(V - masked)[:k] for _ in range(n)]).astype(np.int32)
        np.put_along_axis(x, ids.astype(np.int64), gap + 0.2 * T * rng.random((n, k)), 1)
        if masked:
            x[:, V - masked:] = -np.inf
        view.copy_(torch.from_numpy(x))
        x = view.double().cpu().numpy()
        values = np.log(np.full((n, k), 0.9 / k) * (0.9 + 0.1 * rng.random((n, k)))).astype(np.float32)
        w = np.full(n, weight, np.float32)
        grad, _ = guarded(n, V, dtype)
        got = _distill_run(view, ids, values, kind, w, T, grad)
        _far_check(x, dtype, ids, values, kind, w.astype(np.float64), T, got, f"gap {gap} T {T}")
        alone = _distill_run(view, ids, values, kind, w, T, None)
        assert np.array_equal(alone[0], got[0])


def test_a_divergence_beside_a_far_outside():
    """One listed token of probability 1/2 that the student takes for certain: the loss is 43, not below 0."""
    say("far outside, by hand")
    view = torch.zeros(1, 8, device="cuda")
    view[0, 0] = 90.0
    ids, values = np.zeros((1, 1), np.int32), np.full((1, 1), math.log(0.5), np.float32)
    grad, _ = guarded(1, 8, "f32")
    got = _distill_run(view, ids, values, "tail", None, 1.0, grad)
    assert abs(got[0][0] - (math.log(0.5) + 0.5 * (90 - math.log(7)))) < 1e-4
    assert np.abs(got[1][0] - np.array([0.5] + [-0.5 / 7] * 7)).max() < 1e-6


@pytest.mark.parametrize("kind", ["topk", "tail", "reverse"])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_teachers_values_that_are_no_numbers(kind, bad):
    """A NaN or +inf among a teacher's values is no empty list: the loss is not finite, nor is the entry's gradient."""
    say(f"teacher of {bad} {kind}")
    rng = np.random.default_rng(1)
    n, V, k = 4, 600, 8
    x, view, _ = logits(rng, n, V, "f32")
    ids = np.stack([rng.permutation(V)[:k] for _ in range(n)]).astype(np.int32)
    values = np.log(np.full((n, k), 0.1)).astype(np.float32)
    values[0, 0] = values[1, k - 1] = values[2, 3] = bad
    view[2, int(ids[2, 3])] = -math.inf      # an entry that the student rules out
    values[2, 5] = -math.inf
    grad, _ = guarded(n, V, "f32")
    loss, g = _distill_run(view, ids, values, kind, None, 1.0, grad)
    want, _ = oracle.distill_loss(view.double().cpu().numpy(), ids, values, kind=kind)
    assert not np.isfinite(loss[:3]).any() and np.isfinite(loss[3]), loss
    assert not np.isfinite(want[:3]).any() and np.isfinite(want[3])
    for r, j in ((0, 0), (1, k - 1)):
        assert not np.isfinite(g[r, ids[r, j]])
    assert np.isfinite(g[3]).all()
    assert np.array_equal(_distill_run(view, ids, values, kind, None, 1.0, None)[0], loss, equal_nan=True)


@pytest.mark.parametrize("T", [1e39, 1e45, 1e46, 1e60, 1e300])
@pytest.mark.parametrize("V,dtype", [(50, "bf16"), (3001, "f32"), (40001, "f16")])
def test_temperatures_past_fp32(V, dtype, T):
    """log2(e) / T passes fp32's least number: tokens that can occur become equally likely, the others stay out."""
    import paper_2606_26997_amd as rp
    say(f"temperature {T} {V} {dtype}")
    rng = np.random.default_rng(V)
    n = 3
    x, view, _ = logits(rng, n, V, dtype, masked=5)
    tokens = np.array([int(np.flatnonzero(np.isfinite(r))[3]) for r in x], np.int32)
    lp, H = empty(n), empty(n)
    rp.token_logprobs(view, dev(tokens, torch.int32), lp, H, temperature=T, workspace=workspace(view))
    want = oracle.token_logprobs(x, tokens, T)
    _near(lp.double().cpu(), want[0], lse_bound(V) + U * np.abs(want[0]), "logprobs")
    _near(H.double().cpu(), want[1], entropy_bound(V) + U * np.abs(want[1]), "entropy")
    case = (tokens, want[0].astype(np.float32), want[0].astype(np.float32), np.zeros(n, np.int32), np.ones(1, np.float32),
            np.ones(n, np.float32))
    grad, _ = guarded(n, V, dtype)
    _policy_check(x, view, dtype, T, case, _policy_run(view, dtype, T, case, 0.05, 0.01, grad), 0.05, 0.01)
    ids = np.stack([np.flatnonzero(np.isfinite(r))[:4] for r in x]).astype(np.int32)
    values = np.log(np.full((n, 4), 0.2)).astype(np.float32)
    for kind in ("topk", "tail", "reverse"):
        loss, g = _distill_run(view, ids, values, kind, None, T, grad)
        want, wg = oracle.distill_loss(x, ids, values, kind=kind, temperature=T)
        _near(loss, want, 4 * lse_bound(V) * (1 + math.log(V)) + U * np.abs(want), kind + " losses")
        assert np.abs(g - wg).max() <= 1e-37


@pytest.mark.parametrize("V", [8, 5000, 50000])
def test_logits_further_apart_than_fp32_reaches(V):
    """Logits between -3.3e38 and 3.3e38 at temperatures where each of them counts. |z| is at most 6.6e38 / T, not ln V on
    average; a weight of T / 10 makes the gradient a number."""
    import paper_2606_26997_amd as rp
    say(f"logits of +-3.3e38, {V}")
    rng = np.random.default_rng(V)
    n = 3
    view, _ = guarded(n, V, "f32")
    ends = np.where(rng.random((n, V)) < 0.5, 3.3e38, -3.3e38)
    view.copy_(torch.from_numpy(ends * (1 - 0.3 * rng.random((n, V)))))
    view[2, 7] = -math.inf
    x = view.double().cpu().numpy()
    for T in (4e37, 1e38, 1e39):
        case = list(_policy_case(rng, x, T, n))
        case[5] = np.full(n, T / 10, np.float32)
        far = 6.6e38 / T
        sums = lse_bound(V) + (3 * far + 2) * U
        lp, H = empty(n), empty(n)
        rp.token_logprobs(view, dev(case[0], torch.int32), lp, H, temperature=T, workspace=workspace(view))
        want = oracle.token_logprobs(x, case[0], T)
        _near(lp.double().cpu(), want[0], sums + U * np.abs(want[0]), f"T {T} logprobs")
        _near(H.double().cpu(), want[1], (1 + far) * sums + U * np.abs(want[1]), f"T {T} entropy")
        grad, _ = guarded(n, V, "f32")
        got = _policy_run(view, "f32", T, case, 0.05, 0.0, grad)["grad"]
        want = oracle.policy_loss(x, case[0], case[1].astype(np.float64), case[4], row_seq=case[3],
                                  weights=case[5].astype(np.float64), ref=case[2].astype(np.float64), temperature=T,
                                  clip_low=0.2, clip_high=0.25, kl_beta=0.05)[3]
        # Terms off by (3 z + 8) u, the row's sum and, with a slope of at most 3.3, its factor by `sums`.
        slack = (3 * far + 10) * U + 5 * sums
        _near(got, want, slack * np.abs(want) + 0.1 * 4 * sums * np.abs(want / want.max()) + 1e-37, f"T {T} dlogits")
        ids, values = np.array([[1, 2]] * n, np.int32), np.log(np.full((n, 2), 0.3)).astype(np.float32)
        for kind in ("topk", "tail", "reverse"):
            loss, g = _distill_run(view, ids, values, kind, case[5], T, grad)
            want = oracle.distill_loss(x, ids, values, kind=kind, weights=case[5].astype(np.float64), temperature=T)
            # At T = 1e39 losses of 1e38 times 7 round to infinity.
            _near(loss, f32(want[0]), case[5] * sums * (4 + 2 * far) + 2 * U * np.abs(want[0]), f"T {T} {kind}")
            assert np.abs(g - want[1]).max() <= 0.1 * (3 * far + 10 + far) * 4 * sums, (T, kind)


def test_ratios_that_are_no_finite_numbers():
    """A token that cannot occur has r = 0 whatever the old policy gave it, and an advantage of 0 has no surrogate, also
    beside a ratio past fp64's range."""
    say("ratios")
    n, V = 8, 40
    x, view, _ = logits(np.random.default_rng(3), n, V, "f32")
    view[0, 5] = view[1, 5] = -math.inf
    view[6, 9] = math.nan
    x = view.double().cpu().numpy()
    tokens = np.full(n, 5, np.int32)
    old = np.array([-np.inf, -1.0, -np.inf, -np.inf, -1e30, -2.0, -1.0, -2.0], np.float32)
    adv = np.array([1.0, 1.0, 0.0, 1.0, 0.0, 0.0, 0.0, -1.0], np.float32)
    case = (tokens, old, np.zeros(n, np.float32), np.arange(n, dtype=np.int32), adv, np.ones(n, np.float32))
    grad, _ = guarded(n, V, "f32")
    got = _policy_run(view, "f32", 1.0, case, 0.0, 0.01, grad)
    fine = np.arange(n) != 6
    assert np.isfinite(got["losses"][fine]).all() and np.isfinite(got["grad"][fine]).all(), got
    _policy_check(x, view, "f32", 1.0, case, got, 0.0, 0.01)
