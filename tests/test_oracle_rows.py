"""The float64 oracle of the operators on rows of logits, against closed forms, brute force, differentiation by
torch in float64 and central differences. CPU only."""
import math

import numpy as np
import pytest
import torch

import oracle


def _rows(rng, n, V, scale=2.0, masked=0):
    x = scale * rng.standard_normal((n, V))
    if masked:
        for r in range(n):
            x[r, rng.permutation(V)[:masked]] = -np.inf
    return x


def test_greedy_and_ties_take_the_lowest_index():
    x = np.array([[1.0, 3.0, 3.0, -0.0], [0.0, -0.0, -1.0, 0.0]])
    tok, lp, kept, _ = oracle.sample(x, np.array([0.99, 0.99]), temperature=np.array([0.0, -1.0]))
    assert tok.tolist() == [1, 0] and kept.tolist() == [0, 0]
    assert np.allclose(lp, [3 - math.log(math.e + 2 * math.e ** 3 + 1), -math.log(3 + math.exp(-1))])


def test_borders_of_equal_tokens():
    x = np.zeros((1, 4))
    for u, want in [(0.0, 0), (0.2499, 0), (0.25, 1), (0.5, 2), (0.75, 3), (0.99, 3), (1.0, 3), (7.0, 3), (-1.0, 0), (math.nan, 0)]:
        assert oracle.sample(x, np.array([u]))[0][0] == want, u


@pytest.mark.parametrize("how,want", [
    (dict(top_k=3), [2, 4, 0]), (dict(top_k=1), [2]), (dict(top_k=99), [2, 4, 0, 1, 3, 5]), (dict(top_p=0.0), [2]),
    (dict(top_p=0.5), [2, 4]), (dict(min_p=0.6), [2]), (dict(min_p=0.4), [2, 4, 0, 1]), (dict(min_p=2.0), [2]),
    (dict(top_k=4, top_p=0.8), [2, 4, 0]), (dict(top_k=2, min_p=0.4), [2, 4]),
])
def test_kept_tokens_by_hand(how, want):
    x = np.log(np.array([0.2, 0.2, 0.4, 0.0, 0.2, 0.0]) + np.array([0, 0, 0, 1e-9, 1e-6, 1e-9]))
    assert oracle.kept_tokens(x, **how).tolist() == want


def test_sampling_follows_the_kept_distribution(rng):
    x = _rows(rng, 1, 9)
    n = 20000
    u = (np.arange(n) + 0.5) / n
    tok, _, kept, _ = oracle.sample(np.repeat(x, n, 0), u, temperature=np.full(n, 0.7), top_k=np.full(n, 5))
    ids = np.sort(oracle.kept_tokens(x[0], 0.7, 5))
    w = np.exp(x[0][ids] / 0.7)
    count = np.array([(tok == i).sum() for i in ids])
    assert count.sum() == n and np.abs(count / n - w / w.sum()).max() < 2 / n
    assert np.allclose(np.exp(kept), (w / w.sum())[np.searchsorted(ids, tok)])


def test_rows_without_and_with_bad_logits():
    x = np.array([[-np.inf, -np.inf], [np.nan, 0.0], [np.inf, 0.0], [-np.inf, 2.0]])
    tok, lp, kept, _ = oracle.sample(x, np.full(4, 0.5))
    assert tok.tolist() == [-1, -1, -1, 1] and lp[3] == 0 and kept[3] == 0
    assert lp[0] == -np.inf and np.isnan(lp[1:3]).all()
    lp, H = oracle.token_logprobs(x, np.array([0, 0, 1, 1]))
    assert lp[0] == -np.inf and H[0] == 0 and np.isnan(lp[1:3]).all() and np.isnan(H[1:3]).all() and H[3] == 0


@pytest.mark.parametrize("V,masked,T", [(1, 0, 1.0), (2, 0, 0.5), (33, 5, 1.3), (257, 100, 1.0)])
@pytest.mark.parametrize("beta,ent", [(0.0, 0.0), (0.1, 0.0), (0.05, 0.02)])
def test_policy_gradient_by_differentiation(rng, V, masked, T, beta, ent):
    n = 12
    x = _rows(rng, n, V, masked=masked)
    tokens = np.array([int(rng.choice(np.flatnonzero(np.isfinite(r)))) for r in x])
    tokens[3] = -1
    old = np.minimum(oracle.token_logprobs(x, tokens, T)[0] + 0.4 * rng.standard_normal(n), 0.5)
    ref, adv, w = old + 0.2 * rng.standard_normal(n), rng.standard_normal(5), rng.random(n)
    seq = rng.integers(0, 5, n)
    got = oracle.policy_loss(x, tokens, old, adv, row_seq=seq, weights=w, ref=ref, temperature=T, clip_low=0.2,
                             clip_high=0.3, kl_beta=beta, entropy_coef=ent)
    t = torch.from_numpy(x).requires_grad_()
    lp = torch.log_softmax(t / T, 1)
    # A skipped row's place is taken by its largest logit, whose derivative is finite.
    mine = lp.gather(1, torch.from_numpy(np.where(tokens >= 0, tokens, x.argmax(1)))[:, None])[:, 0]
    H = -torch.where(torch.isfinite(lp), torch.exp(lp) * torch.where(torch.isfinite(lp), lp, 0.0), 0.0).sum(1)
    r, A = torch.exp(mine - torch.from_numpy(old)), torch.from_numpy(adv[seq])
    gap = torch.from_numpy(ref) - mine
    loss = -torch.minimum(r * A, r.clamp(0.8, 1.3) * A) + beta * (torch.exp(gap) - gap - 1) - ent * H
    loss = torch.where(torch.from_numpy(tokens >= 0), torch.from_numpy(w) * loss, 0.0)
    (g,) = torch.autograd.grad(loss.sum(), t)
    assert np.allclose(got[0], loss.detach().numpy(), atol=1e-12)
    assert np.allclose(got[3], g.numpy(), atol=1e-12)


@pytest.mark.parametrize("kind", ["topk", "tail", "reverse"])
@pytest.mark.parametrize("V,k,masked,T", [(2, 1, 0, 1.0), (40, 7, 0, 0.8), (40, 40, 0, 1.0), (300, 32, 60, 1.5)])
def test_distillation_gradient_by_differentiation(rng, kind, V, k, masked, T):
    n = 6
    x = _rows(rng, n, V, masked=masked)
    teacher = np.where(np.isfinite(x), x + rng.standard_normal((n, V)), -np.inf)
    ids = np.argsort(-teacher, 1)[:, :k]
    logp = np.array([oracle.token_logprobs(np.repeat(t[None], V, 0), np.arange(V), T)[0] for t in teacher])
    values = np.take_along_axis(teacher if kind == "topk" else logp, ids, 1)
    w = rng.random(n)
    loss, grad = oracle.distill_loss(x, ids, values, kind=kind, weights=w, temperature=T)
    t = torch.from_numpy(x).requires_grad_()
    lq = torch.log_softmax(t / T, 1)
    v, at = torch.from_numpy(values), torch.from_numpy(ids)
    if kind == "topk":
        lp = torch.log_softmax(v / T, 1)
        ref = (torch.exp(lp) * (lp - lq.gather(1, at))).sum(1)
    else:
        P = torch.exp(v)
        rest = (1 - P.sum(1)).clamp(min=2.0 ** -24)
        out = torch.exp(lq).scatter(1, at, 0.0).sum(1)
        if k == V:
            ref = (P * (v - lq.gather(1, at))).sum(1) if kind == "tail" else \
                (torch.exp(lq.gather(1, at)) * (lq.gather(1, at) - v)).sum(1)
        elif kind == "tail":
            ref = (P * (v - lq.gather(1, at))).sum(1) + rest * torch.log(rest / out)
        else:
            ref = (torch.exp(lq.gather(1, at)) * (lq.gather(1, at) - v)).sum(1) + out * torch.log(out / rest)
    ref = torch.from_numpy(w) * ref
    (g,) = torch.autograd.grad(ref.sum(), t)
    assert np.allclose(loss, ref.detach().numpy(), atol=1e-11)
    assert np.allclose(grad, g.numpy(), atol=1e-11)


@pytest.mark.parametrize("kind", ["topk", "tail", "reverse"])
def test_entries_that_do_not_count(rng, kind):
    x = _rows(rng, 1, 20)
    clean = oracle.distill_loss(x, np.array([[3, 7, 1]]), np.array([[-1.0, -2.0, -3.0]]), kind=kind)
    mixed = oracle.distill_loss(x, np.array([[3, -1, 7, 3, 20, 1, 5]]),
                                np.array([[-1.0, -0.5, -2.0, -9.0, -0.1, -3.0, -np.inf]]), kind=kind)
    assert np.array_equal(clean[0], mixed[0]) and np.array_equal(clean[1], mixed[1])
    loss, grad = oracle.distill_loss(x, np.array([[-1]]), np.array([[0.0]]), kind=kind)
    assert abs(loss[0]) < 1e-12 and np.abs(grad).max() < 1e-12


def test_gradients_by_differences(rng):
    x, h = _rows(rng, 1, 11), 1e-5
    args = dict(old=np.array([-1.5]), advantages=np.array([-0.7]), ref=np.array([-2.0]), kl_beta=0.2, entropy_coef=0.1)
    policy = lambda z: oracle.policy_loss(z, np.array([4]), temperature=0.9, **args)
    lists = dict(ids=np.array([[2, 9, 4]]), values=np.array([[-0.7, -1.6, -2.5]]), temperature=1.2)
    for f, grad in [(policy, 3)] + [(lambda z, k=k: oracle.distill_loss(z, kind=k, **lists), 1) for k in ("topk", "tail", "reverse")]:
        got = f(x)[grad][0]
        for i in range(11):
            up, down = x.copy(), x.copy()
            up[0, i] += h
            down[0, i] -= h
            assert abs((f(up)[0][0] - f(down)[0][0]) / (2 * h) - got[i]) < 1e-8, i
