"""Log-probabilities, policy loss and distillation on the GPU against the float64 oracle; bounds from rows_util."""
import math

import numpy as np
import pytest
import torch

import oracle
from tests.rows_util import (DTYPES, U, dev, empty, entropy_bound, f32, gaps_untouched, guarded, half_step, logits,
                             lse_bound, say, workspace)

pytestmark = pytest.mark.gpu

SIZES = [  # rows, vocab, dtype, pad, offset, masked, temperature
    (1, 1, "bf16", 0, 0, 0, 1.0), (3, 2, "f32", 1, 1, 0, 0.5), (5, 7, "bf16", 2, 3, 2, 1.0), (9, 63, "f16", 0, 1, 5, 2.0),
    (300, 40, "bf16", 0, 0, 0, 0.7), (4, 1000, "f32", 3, 0, 900, 1.0), (3, 8191, "bf16", 1, 0, 0, 1.1),
    (2, 32769, "f16", 7, 5, 100, 1.0), (3, 50257, "f32", 0, 0, 0, 0.9), (2, 151936, "bf16", 0, 0, 267, 1.0),
    (2, 163841, "bf16", 0, 1, 0, 1.0), (1, 90001, "f32", 0, 0, 7, 1.3), (1, 1 << 20, "bf16", 0, 0, 0, 1.0),
    (270, 4097, "bf16", 0, 0, 11, 1.0),
]


def _tokens(rng, x):
    best = x.argmax(1)
    any_live = np.array([int(rng.choice(np.flatnonzero(np.isfinite(r)))) if np.isfinite(r).any() else 0 for r in x])
    return np.where(rng.random(len(x)) < 0.5, best, any_live).astype(np.int32)


def _near(got, want, bound, what):
    got, want, bound = np.asarray(got), np.asarray(want), np.broadcast_to(bound, np.shape(want))
    fine = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)), f"{what}: NaN"
    rest = ~fine & ~np.isnan(want)
    assert np.array_equal(got[rest], want[rest]), f"{what}: infinities"
    off = np.abs(got[fine] - want[fine]) - bound[fine]
    assert off.size == 0 or off.max() <= 0, f"{what}: over the bound by {off.max()}, bound {bound[fine][off.argmax()]}"


def _z(x, T):
    """|z - max z| where it is finite."""
    with np.errstate(invalid="ignore"):
        z = (x.max(1, keepdims=True) - x) / T
    return np.where(np.isfinite(z), z, 0.0)


@pytest.mark.parametrize("n,V,dtype,pad,offset,masked,T", SIZES)
def test_logprobs(n, V, dtype, pad, offset, masked, T):
    import paper_2606_26997_amd as rp
    say(f"logprobs {n} x {V} {dtype}")
    rng = np.random.default_rng(V + n)
    x, view, buf = logits(rng, n, V, dtype, masked=masked, pad=pad, offset=offset)
    tokens = _tokens(rng, x)
    if n > 2:
        tokens[0], tokens[1] = -1, V
    lp, H = empty(n), empty(n)
    rp.token_logprobs(view, dev(tokens, torch.int32), lp, H, temperature=T, workspace=workspace(view))
    want = oracle.token_logprobs(x, tokens, T)
    _near(lp.double().cpu(), want[0], lse_bound(V) + U * np.abs(want[0]), "logprobs")
    _near(H.double().cpu(), want[1], entropy_bound(V) + U * np.abs(want[1]), "entropy")
    alone = empty(n)
    rp.token_logprobs(view, dev(tokens, torch.int32), alone, temperature=T, workspace=workspace(view))
    assert torch.equal(alone, lp) and gaps_untouched(view, buf)


def _policy_case(rng, x, T, n):
    tokens = _tokens(rng, x)
    lp = oracle.token_logprobs(x, tokens, T)[0]
    lp = np.where(np.isfinite(lp), lp, -1.0)
    # Ratios of 0.5 to 1.6, none within 1e-3 of a border.
    ratio = 0.5 + 1.1 * rng.random(n)
    for border in (0.8, 1.25):
        ratio = np.where(np.abs(ratio - border) < 2e-3, border + 4e-3, ratio)
    old = (lp - np.log(ratio)).astype(np.float32)
    ref = (lp + 0.3 * rng.standard_normal(n)).astype(np.float32)
    seq = rng.integers(0, 4, n).astype(np.int32)
    adv = rng.standard_normal((2, 2)).astype(np.float32)
    return tokens, old, ref, seq, adv, rng.random(n).astype(np.float32)


def _policy_check(x, view, dtype, T, case, got, beta, ent, use_ref=True, weights=True, what=""):
    tokens, old, ref, seq, adv, w = case
    V = x.shape[1]
    weight = w.astype(np.float64) if weights else np.ones(len(x))
    loss, lp, H, grad = oracle.policy_loss(x, tokens, old.astype(np.float64), adv, row_seq=seq,
                                           weights=weight, ref=ref.astype(np.float64),
                                           temperature=T, clip_low=0.2, clip_high=0.25, kl_beta=beta, entropy_coef=ent)
    A = np.abs(adv.reshape(-1).astype(np.float64)[np.clip(seq, 0, adv.size - 1)])
    with np.errstate(over="ignore", invalid="ignore"):
        ratio, gap = np.exp(np.where(np.isfinite(lp), lp - old, 0.0)), np.exp(np.where(np.isfinite(lp), ref - lp, 0.0))
    lb, hb = lse_bound(V), entropy_bound(V)
    tidy = lambda a: np.where(np.isfinite(a), a, 0.0)
    slope = A * tidy(ratio) + beta * (1 + gap)  # an infinite ratio is clipped, or its loss infinite
    _near(got["losses"], loss, weight * (slope * lb * 1.01 + ent * hb) + U * np.abs(tidy(loss)), what + "losses")
    _near(got["logprobs"], lp, lb + U * np.abs(tidy(lp)), what + "logprobs")
    _near(got["entropy"], H, hb + U * np.abs(tidy(H)), what + "entropy")
    # Every element: its probability is off by (3 |z| + 4) u and the row's sum, its factor by the slope's.
    z = _z(x, T)
    with np.errstate(invalid="ignore"):
        p = np.where(np.isfinite(x), np.exp(-z), 0.0)
    p = p / np.maximum(p.sum(1, keepdims=True), 1.0)
    size = slope[:, None] + ent * (np.abs(tidy(H))[:, None] + math.log(V) + z)
    onehot = np.zeros_like(p)
    onehot[np.arange(len(x)), np.clip(tokens, 0, V - 1)] = 1.0
    bound = (weight / T)[:, None] * ((p * size) * ((3 * z + 8) * U + 2 * lb + U) + p * ent * hb + onehot * (slope[:, None] * lb * 1.01))
    tiny = 2.0 ** -25 if dtype == "f16" else 1e-37
    _near(got["grad"], grad, bound + half_step(dtype) * 1.01 * np.abs(tidy(grad)) + tiny, what + "dlogits")


def _policy_run(view, dtype, T, case, beta, ent, grad, **kw):
    import paper_2606_26997_amd as rp
    tokens, old, ref, seq, adv, w = case
    n = view.shape[0]
    out = dict(losses=empty(n), logprobs=empty(n), entropy=empty(n))
    args = dict(row_seq=dev(seq, torch.int32), weights=dev(w), ref_logprobs=dev(ref) if beta else None)
    args.update(kw)
    rp.policy_loss(view, dev(tokens, torch.int32), dev(old), dev(adv), out["losses"], grad, logprobs=out["logprobs"],
                   entropy=out["entropy"], temperature=T, clip_low=0.2, clip_high=0.25, kl_beta=beta, entropy_coef=ent,
                   workspace=workspace(view), **args)
    torch.cuda.synchronize()
    out = {k: v.double().cpu().numpy() for k, v in out.items()}
    if grad is not None:
        out["grad"] = grad.double().cpu().numpy()
    return out


@pytest.mark.parametrize("beta,ent", [(0.0, 0.0), (0.05, 0.02)])
@pytest.mark.parametrize("n,V,dtype,pad,offset,masked,T", SIZES)
def test_policy(n, V, dtype, pad, offset, masked, T, beta, ent):
    say(f"policy {n} x {V} {dtype} beta {beta} entropy {ent}")
    rng = np.random.default_rng(V + 7 * n)
    x, view, buf = logits(rng, n, V, dtype, masked=masked, pad=pad, offset=offset)
    case = _policy_case(rng, x, T, n)
    if n > 4:
        case[0][0], case[0][1], case[3][2], case[3][3] = -1, V, -1, 4
        case[5][4] = 0.0
    grad, gbuf = guarded(n, V, dtype, pad + 1, offset + 1)
    got = _policy_run(view, dtype, T, case, beta, ent, grad)
    _policy_check(x, view, dtype, T, case, got, beta, ent)
    assert gaps_untouched(grad, gbuf) and gaps_untouched(view, buf)
    assert np.array_equal(view.double().cpu().numpy(), x, equal_nan=True)
    # The losses alone, and the gradient in the logits' place: the same numbers.
    alone = _policy_run(view, dtype, T, case, beta, ent, None)
    assert all(np.array_equal(alone[k], got[k]) for k in alone)
    there = _policy_run(view, dtype, T, case, beta, ent, view)
    assert all(np.array_equal(there[k], got[k]) for k in there) and gaps_untouched(view, buf)


@pytest.mark.parametrize("V", [6, 900, 40000])
def test_policy_rows_that_are_empty_or_bad(V):
    say(f"policy bad rows {V}")
    rng = np.random.default_rng(V)
    n, T = 9, 1.0
    x, view, _ = logits(rng, n, V, "bf16")
    view[0] = -math.inf
    view[1, V // 2] = math.nan
    view[2, 0] = math.inf
    view[3] = -math.inf
    view[3, V - 1] = 2.0
    view[4] = math.nan
    view[5, 1:] = -3.0e38
    view[6, 0] = math.nan
    x = view.double().cpu().numpy()
    case = _policy_case(rng, x, T, n)
    case[5][6] = 0.0                       # a weight of 0 beside a NaN
    case[0][4] = -1                        # a skipped row of NaN
    case[0][3], case[0][5] = V - 1, 0      # the only token left
    for beta, ent in ((0.0, 0.0), (0.05, 0.02)):
        grad, _ = guarded(n, V, "bf16")
        got = _policy_run(view, "bf16", T, case, beta, ent, grad)
        _policy_check(x, view, "bf16", T, case, got, beta, ent, what=f"beta {beta} ")


def test_policy_without_sequences_and_weights():
    say("policy, advantages by row")
    rng = np.random.default_rng(4)
    n, V = 4, 333
    x, view, _ = logits(rng, n, V, "f32")
    case = list(_policy_case(rng, x, 1.0, n))
    case[3] = np.arange(4, dtype=np.int32)
    grad, _ = guarded(n, V, "f32")
    got = _policy_run(view, "f32", 1.0, case, 0.05, 0.0, grad, row_seq=None, weights=None)
    _policy_check(x, view, "f32", 1.0, case, got, 0.05, 0.0, weights=False)


def test_policy_gradient_against_differences():
    """Central differences of the fp32 losses themselves: h = 2^-6, losses off by 2e-6, third derivatives below 20."""
    import paper_2606_26997_amd as rp
    say("policy differences")
    rng = np.random.default_rng(9)
    V, h = 12, 2.0 ** -6
    x, view, _ = logits(rng, 1, V, "f32", scale=1.0, peaks=0)
    case = [a[:1] if a.ndim == 1 else a for a in _policy_case(rng, x, 1.0, 1)]
    grad, _ = guarded(1, V, "f32")
    got = _policy_run(view, "f32", 1.0, case, 0.05, 0.02, grad)["grad"][0]
    many = view.repeat(2 * V, 1)
    for i in range(V):
        many[2 * i, i] += h
        many[2 * i + 1, i] -= h
    rep = [np.repeat(a, 2 * V, 0) if a.ndim == 1 else a for a in case]
    losses = _policy_run(many, "f32", 1.0, rep, 0.05, 0.02, None)["losses"]
    diff = (losses[0::2] - losses[1::2]) / (2 * h)
    assert np.abs(diff - got).max() <= 2e-6 / h + 20 * h * h / 6


# ---- distillation ----------------------------------------------------------
def _lists(rng, x, k, kind, T):
    n, V = x.shape
    teacher = np.where(np.isfinite(x), x / T + 0.8 * rng.standard_normal(x.shape), -np.inf)
    ids = np.argsort(-teacher, 1, kind="stable")[:, :k]
    top = teacher.max(1, keepdims=True)
    lse = top + np.log(np.exp(teacher - top).sum(1, keepdims=True))
    values = np.take_along_axis(teacher, ids, 1)
    values = values * T if kind == "topk" else values - lse
    shuffle = np.argsort(rng.random(ids.shape), 1)
    return (np.take_along_axis(ids, shuffle, 1).astype(np.int32), np.take_along_axis(values, shuffle, 1).astype(np.float32))


def _distill_run(view, ids, values, kind, w, T, grad):
    import paper_2606_26997_amd as rp
    losses = empty(view.shape[0])
    rp.distill_loss(view, dev(ids, torch.int32), dev(values), losses, grad, kind=kind, weights=dev(w), temperature=T,
                    workspace=workspace(view))
    torch.cuda.synchronize()
    return losses.double().cpu().numpy(), None if grad is None else grad.double().cpu().numpy()


def _distill_check(x, dtype, ids, values, kind, w, T, got, what=""):
    n, V = x.shape
    weight = np.ones(n) if w is None else w.astype(np.float64)
    loss, grad = oracle.distill_loss(x, ids, values, kind=kind, weights=weight, temperature=T)
    tidy = lambda a: np.where(np.isfinite(a), a, 0.0)
    lb, z = lse_bound(V), _z(x, T)
    with np.errstate(invalid="ignore"):
        p = np.where(np.isfinite(x), np.exp(-z), 0.0)
    p = p / np.maximum(p.sum(1, keepdims=True), 1.0)
    listed = np.zeros(x.shape, bool)
    P = np.zeros(x.shape)
    for r in range(n):
        for i, t in zip(ids[r], values[r]):
            if 0 <= i < V and t > -math.inf and not listed[r, i]:
                listed[r, i] = True
                P[r, i] = math.exp(float(t)) if kind != "topk" else 0.0
    out = (p * ~listed).sum(1)
    rest = np.maximum(1 - P.sum(1), 2.0 ** -24)
    gap = np.abs(np.log(np.where(out > 0, out, rest) / rest))
    lq = np.abs(np.log(np.maximum(p, 1e-300)))
    lp = np.abs(np.log(np.maximum(P, 1e-300)))
    if kind == "reverse":
        worth = (p * listed * (lq + lp + 1)).sum(1) + out * (gap + 1)
        factor = np.where(listed, lq + lp + np.abs(tidy(loss / np.maximum(weight, 1e-30)))[:, None] + 1,
                          gap[:, None] + np.abs(tidy(loss / np.maximum(weight, 1e-30)))[:, None] + 1) + worth[:, None]
    else:
        worth = 1.0 + (rest if kind == "tail" else 0.0)
        ratio = rest / np.maximum(out, 1e-300) if kind == "tail" else np.ones(n)
        factor = np.where(listed, 2.0, np.where(out > 0, 1 + ratio, 0.0)[:, None])
    _near(got[0], loss, weight * 2 * worth * lb + U * np.abs(tidy(loss)) + weight * 1e-12, what + "losses")
    bound = (weight / T)[:, None] * p * factor * ((3 * z + 8) * U + 4 * lb)
    tiny = 2.0 ** -25 if dtype == "f16" else 1e-37
    if got[1] is not None:
        _near(got[1], grad, bound + half_step(dtype) * 1.01 * np.abs(tidy(grad)) + tiny, what + "dlogits")


@pytest.mark.parametrize("kind", ["topk", "tail", "reverse"])
@pytest.mark.parametrize("n,V,dtype,pad,offset,masked,T", SIZES)
def test_distillation(n, V, dtype, pad, offset, masked, T, kind):
    say(f"distill {n} x {V} {dtype} {kind}")
    rng = np.random.default_rng(V + 3 * n)
    x, view, buf = logits(rng, n, V, dtype, masked=masked, pad=pad, offset=offset)
    k = max(1, min((V - masked) // 2, 1024 if V > 100000 else 50))
    ids, values = _lists(rng, x, k, kind, T)
    w = rng.random(n).astype(np.float32)
    if n > 2:
        w[1] = 0.0
    grad, gbuf = guarded(n, V, dtype, pad + 1, offset + 1)
    got = _distill_run(view, ids, values, kind, w, T, grad)
    _distill_check(x, dtype, ids, values, kind, w, T, got)
    assert gaps_untouched(grad, gbuf) and gaps_untouched(view, buf)
    assert np.array_equal(view.double().cpu().numpy(), x, equal_nan=True)
    assert np.array_equal(_distill_run(view, ids, values, kind, w, T, None)[0], got[0])
    there = _distill_run(view, ids, values, kind, w, T, view)
    assert np.array_equal(there[0], got[0]) and np.array_equal(there[1], got[1]) and gaps_untouched(view, buf)


@pytest.mark.parametrize("kind", ["topk", "tail", "reverse"])
@pytest.mark.parametrize("V", [30, 5000])
def test_lists_with_entries_that_do_not_count(V, kind):
    """Ids listed twice, out of range, values of -inf; nothing listed; everything listed; a long list of one id."""
    say(f"odd lists {V} {kind}")
    rng = np.random.default_rng(V)
    x, view, _ = logits(rng, 6, V, "f32")
    ids, values = _lists(rng, x, 16, kind, 1.0)
    ids[0, 3], ids[0, 9], ids[1, 2], ids[1, 5] = ids[0, 1], ids[0, 1], -1, V
    values[2, 4] = -math.inf
    ids[3], ids[4], values[5] = -7, ids[4, 0], -math.inf
    if kind != "topk":
        values -= 1.0  # what does not count leaves mass outside
    grad, _ = guarded(6, V, "f32")
    _distill_check(x, "f32", ids, values, kind, None, 1.0, _distill_run(view, ids, values, kind, None, 1.0, grad))
    if V == 30:
        ids, values = _lists(rng, x, 30, kind, 1.0)
        _distill_check(x, "f32", ids, values, kind, None, 1.0, _distill_run(view, ids, values, kind, None, 1.0, grad), "all ")


@pytest.mark.parametrize("kind", ["topk", "tail", "reverse"])
def test_distillation_of_rows_that_are_empty_or_bad(kind):
    say(f"distill bad rows {kind}")
    rng = np.random.default_rng(6)
    n, V = 7, 700
    x, view, _ = logits(rng, n, V, "bf16")
    ids, values = _lists(rng, x, 8, kind, 1.0)
    view[0] = -math.inf
    view[1, 600] = math.nan
    view[2, int(ids[2, 0])] = math.inf
    view[3] = math.nan
    view[4] = -math.inf
    view[4, torch.from_numpy(ids[4].astype(np.int64)).cuda()] = 1.0   # nothing outside the list
    w = np.ones(n, np.float32)
    w[3] = 0.0
    x = view.double().cpu().numpy()
    grad, _ = guarded(n, V, "bf16")
    _distill_check(x, "bf16", ids, values, kind, w, 1.0, _distill_run(view, ids, values, kind, w, 1.0, grad))


def test_a_small_mass_outside_the_list():
    """Logits of 20 and more in the list, of 0 outside: a mass of about 1e-6 there keeps its digits."""
    say("distill small tail")
    rng = np.random.default_rng(12)
    V, k = 3000, 8
    x, view, _ = logits(rng, 2, V, "f32", scale=0.3, peaks=0)
    ids = np.stack([rng.permutation(V)[:k] for _ in range(2)]).astype(np.int32)
    view.scatter_(1, dev(ids, torch.int64), 22.0 + torch.rand(2, k, device="cuda"))
    x = view.double().cpu().numpy()
    values = np.log(np.full((2, k), (1 - 1e-5) / k)).astype(np.float32)
    for kind in ("tail", "reverse"):
        grad, _ = guarded(2, V, "f32")
        _distill_check(x, "f32", ids, values, kind, None, 1.0, _distill_run(view, ids, values, kind, None, 1.0, grad), kind + " ")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [600, 30001, 200000])
def test_one_token_with_nearly_all_the_mass(V, dtype):
    """ln p of a token of probability 1 - 1e-4 and closer, the entropy and the gradient there keep their digits: the other
    terms' sum is off by (3 |z| + 2 + V / 2048 + 16) u, with |z| below 40."""
    import paper_2606_26997_amd as rp
    say(f"dominant token {V} {dtype}")
    rng = np.random.default_rng(V)
    n = 4
    x, view, _ = logits(rng, n, V, dtype, scale=0.5, peaks=0)
    at = np.array([0, V - 1, V // 2, 7])
    for r in range(n):
        view[r, int(at[r])] = 22.0 + 3 * r
    x = view.double().cpu().numpy()
    rel = 3 * ((3 * 40 + 2 + V / 2048 + 16) * U)
    lp, H = empty(n), empty(n)
    rp.token_logprobs(view, dev(at, torch.int32), lp, H, workspace=workspace(view))
    want = oracle.token_logprobs(x, at)
    # The oracle's own ln(1 + small) is off by 2^-53 of 1.
    _near(lp.double().cpu(), want[0], rel * np.abs(want[0]) + 2e-16, "logprobs")
    _near(H.double().cpu(), want[1], 3 * rel * np.abs(want[1]) + 1e-14, "entropy")
    case = (at.astype(np.int32), want[0].astype(np.float32), want[0].astype(np.float32), np.arange(n, dtype=np.int32),
            np.ones(n, np.float32), np.ones(n, np.float32))
    grad, _ = guarded(n, V, "f32")
    if dtype == "f32":
        got = _policy_run(view, "f32", 1.0, case, 0.0, 0.0, grad)["grad"]
        ref = oracle.policy_loss(x, at, case[1].astype(np.float64), case[4])[3]
        r = np.arange(n)
        _near(got[r, at], ref[r, at], rel * np.abs(ref[r, at]) + 1e-15, "the token's gradient")
    tokens, slp, kept = empty(n, torch.int32), empty(n), empty(n)
    rp.sample_tokens(view, dev(np.full(n, 0.5)), tokens, slp, kept, workspace=workspace(view))
    assert tokens.tolist() == at.tolist()
    _near(slp.double().cpu(), want[0], rel * np.abs(want[0]) + 2e-16, "sampled")
    rp.sample_tokens(view, dev(np.full(n, 0.5)), tokens, slp, kept, top_k=dev(np.full(n, 5), torch.int32), workspace=workspace(view))
    assert tokens.tolist() == at.tolist()
    _near(slp.double().cpu(), want[0], rel * np.abs(want[0]) + 2e-16, "sampled, top-k")


@pytest.mark.parametrize("V", [40, 5000])
def test_logits_near_the_end_of_fp32(V):
    """Rows of +-3e38 (all alike, and beside ordinary ones) are sums like any other."""
    import paper_2606_26997_amd as rp
    say(f"huge logits {V}")
    n = 4
    view = torch.zeros(n, V, device="cuda")
    view[0], view[1], view[2] = -3.0e38, 3.0e38, -3.0e38
    view[2, 5] = 1.0
    view[3] = -3.4028234663852886e38
    x = view.double().cpu().numpy()
    tokens = np.array([3, 3, 5, 3])
    lp, H = empty(n), empty(n)
    rp.token_logprobs(view, dev(tokens, torch.int32), lp, H, workspace=workspace(view))
    want = oracle.token_logprobs(x, tokens)
    _near(lp.double().cpu(), want[0], lse_bound(V) + U * np.abs(want[0]), "logprobs")
    _near(H.double().cpu(), want[1], entropy_bound(V) + U * np.abs(want[1]), "entropy")
    case = (tokens.astype(np.int32), want[0].astype(np.float32), want[0].astype(np.float32), np.zeros(n, np.int32),
            np.ones(1, np.float32), np.ones(n, np.float32))
    grad, _ = guarded(n, V, "f32")
    _policy_check(x, view, "f32", 1.0, case, _policy_run(view, "f32", 1.0, case, 0.05, 0.01, grad), 0.05, 0.01)
    got = rp_sample(view)
    assert got[2] == 5 and all(0 <= t < V for t in got)


def rp_sample(view):
    import paper_2606_26997_amd as rp
    tokens = empty(view.shape[0], torch.int32)
    rp.sample_tokens(view, dev(np.full(view.shape[0], 0.4)), tokens, workspace=workspace(view))
    return tokens.tolist()
