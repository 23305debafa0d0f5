"""The calls on rows of logits as a program makes them: a sampled batch, its advantages, the update and a distillation
after it; captured into a graph and replayed; on two streams at once; far apart in memory."""
import numpy as np
import pytest
import torch

import oracle
from tests.rows_util import U, dev, empty, guarded, logits, lse_bound, say, workspace
from tests.test_gpu_losses import _distill_check, _lists, _policy_check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("V,dtype", [(700, "f32"), (33001, "bf16")])
def test_a_rollout_step_its_update_and_a_distillation(V, dtype):
    """Tokens of 4 groups of 8 are drawn on-policy; their log-probabilities are what token_logprobs says of them, so
    the update's ratios are 1 and its losses - w A; groups' advantages come from grpo_advantage as they lie."""
    import paper_2606_26997_amd as rp
    say(f"rollout and update {V} {dtype}")
    rng = np.random.default_rng(V)
    R, K, T = 4, 8, 1.25
    n = R * K
    x, view, _ = logits(rng, n, V, dtype)
    ws, u = workspace(view), rng.random(n).astype(np.float32)
    tokens, lp, kept = empty(n, torch.int32), empty(n), empty(n)
    rp.sample_tokens(view, dev(u), tokens, lp, kept, temperature=dev(np.full(n, T)), workspace=ws)
    want = oracle.sample(x, u, temperature=np.full(n, T, np.float32))
    assert want[3].min() > 1e-11 and np.array_equal(tokens.cpu().numpy(), want[0])
    again, H = empty(n), empty(n)
    rp.token_logprobs(view, tokens, again, H, temperature=T, workspace=ws)
    a, b = lp.double().cpu().numpy(), again.double().cpu().numpy()
    # Nothing is filtered: drawn with the probability that the row gives, to the bounds of both.
    assert np.abs(a - b).max() <= (2 * U * np.abs(a) + 2 * lse_bound(V)).max()
    assert np.abs(a - kept.double().cpu().numpy()).max() <= (2 * U * np.abs(a) + 1e-10).max()
    rewards = dev(rng.integers(0, 2, (R, K)).astype(np.float32))
    adv = torch.empty(R, K, device="cuda")
    rp.grpo_advantage(rewards, adv)
    seq, w = dev(np.arange(n), torch.int32), dev(np.full(n, 1.0 / n))
    losses, grad = empty(n), guarded(n, V, dtype)[0]
    out = dict(losses=losses, logprobs=empty(n), entropy=empty(n))
    rp.policy_loss(view, tokens, again, adv, losses, grad, row_seq=seq, weights=w, ref_logprobs=lp,
                   logprobs=out["logprobs"], entropy=out["entropy"], temperature=T, clip_low=0.2, clip_high=0.25,
                   kl_beta=0.05, entropy_coef=0.01, workspace=ws)
    assert torch.equal(out["logprobs"], again) and torch.equal(out["entropy"], H)
    got = {k: v.double().cpu().numpy() for k, v in out.items()}
    got["grad"] = grad.double().cpu().numpy()
    case = (tokens.cpu().numpy(), again.cpu().numpy(), lp.cpu().numpy(), np.arange(n, dtype=np.int32),
            adv.cpu().numpy(), w.cpu().numpy())
    _policy_check(x, view, dtype, T, case, got, 0.05, 0.01)
    # One step down the gradient, and a distillation on the rows that it leaves, its gradient in their place.
    view -= 0.5 * grad
    x = view.double().cpu().numpy()
    ids, values = _lists(rng, x, 20, "reverse", 1.0)
    rp.distill_loss(view, dev(ids, torch.int32), dev(values), losses, view, kind="reverse", workspace=ws)
    _distill_check(x, dtype, ids, values, "reverse", None, 1.0,
                   (losses.double().cpu().numpy(), view.double().cpu().numpy()))


def _static(rng, n, V, dtype):
    s = dict(x=logits(rng, n, V, dtype)[1], u=dev(rng.random(n)), tokens=empty(n, torch.int32), lp=empty(n), kept=empty(n),
             old=empty(n), H=empty(n), losses=empty(n), dl=empty(n), grad=guarded(n, V, dtype)[0],
             grad2=guarded(n, V, dtype)[0], adv=dev(rng.standard_normal(n)), top_p=dev(np.full(n, 0.9)),
             top_k=dev(np.full(n, 40), torch.int32), ids=dev(np.argsort(rng.random((n, V)), 1)[:, :6], torch.int32),
             values=dev(np.log(np.full((n, 6), 0.1))))
    s["ws"] = workspace(s["x"])
    return s


def _pass(s, stream=None):
    import paper_2606_26997_amd as rp
    kw = dict(workspace=s["ws"], stream=stream)
    rp.sample_tokens(s["x"], s["u"], s["tokens"], s["lp"], s["kept"], top_p=s["top_p"], top_k=s["top_k"], **kw)
    rp.token_logprobs(s["x"], s["tokens"], s["old"], s["H"], **kw)
    rp.policy_loss(s["x"], s["tokens"], s["lp"], s["adv"], s["losses"], s["grad"], entropy_coef=0.01, **kw)
    rp.distill_loss(s["x"], s["ids"], s["values"], s["dl"], s["grad2"], **kw)


OUT = ("tokens", "lp", "kept", "old", "H", "losses", "dl", "grad", "grad2")


def _taken(s):
    return [s[k].clone() for k in OUT]


@pytest.mark.parametrize("n,V,dtype", [(3, 500, "f32"), (20, 40000, "bf16"), (300, 9000, "f16")])
def test_captured_and_replayed(n, V, dtype):
    """Every replay, with other inputs and eager work between, gives what the eager calls give, bit for bit."""
    say(f"graph {n} x {V} {dtype}")
    rng = np.random.default_rng(n)
    s = _static(rng, n, V, dtype)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _pass(s)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _pass(s)
    for r in range(4):
        s["x"].copy_(torch.from_numpy(2.5 * rng.standard_normal((n, V))).to(s["x"].dtype))
        s["u"].copy_(dev(rng.random(n)))
        for k in OUT:
            s[k].fill_(-3)
        graph.replay()
        torch.cuda.synchronize()
        replayed = _taken(s)
        for k in OUT:
            s[k].fill_(-4)
        _pass(s)
        torch.cuda.synchronize()
        for k, a, b in zip(OUT, replayed, _taken(s)):
            assert torch.equal(a, b), (r, k)


def test_two_streams_at_once():
    """Two batches on two streams, each with its workspace, interleaved: what each gives alone."""
    say("two streams")
    rng = np.random.default_rng(77)
    batches = [_static(rng, 12, 60000, "bf16"), _static(rng, 40, 35000, "bf16")]
    alone = []
    for s in batches:
        _pass(s)
        torch.cuda.synchronize()
        alone.append(_taken(s))
    streams = [torch.cuda.Stream() for _ in batches]
    torch.cuda.synchronize()
    for _ in range(3):
        for s in batches:
            for k in OUT:
                s[k].fill_(-1)
        torch.cuda.synchronize()
        for _ in range(4):
            for s, st in zip(batches, streams):
                _pass(s, stream=st)
        torch.cuda.synchronize()
        for s, want in zip(batches, alone):
            for k, a, b in zip(OUT, _taken(s), want):
                assert torch.equal(a, b), k


def test_rows_far_apart():
    """Rows 2^30 elements apart: offsets pass 32 bits."""
    import paper_2606_26997_amd as rp
    say("rows far apart")
    rng = np.random.default_rng(5)
    n, V, stride = 3, 1000, 1 << 30
    bufs = [torch.zeros((n - 1) * stride + V, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    far, grad = (b.as_strided((n, V), (stride, 1)) for b in bufs)
    near = torch.from_numpy(2 * rng.standard_normal((n, V))).to("cuda", torch.bfloat16)
    far.copy_(near)
    u, adv, old = dev(rng.random(n)), dev(rng.standard_normal(n)), dev(np.full(n, -5.0))
    res = []
    for x, g in ((near, torch.empty_like(near)), (far, grad)):
        tokens, lp, losses = empty(n, torch.int32), empty(n), empty(n)
        rp.sample_tokens(x, u, tokens, lp)
        rp.policy_loss(x, tokens, old, adv, losses, g)
        torch.cuda.synchronize()
        res.append((tokens, lp, losses, g.clone()))
    for a, b in zip(*res):
        assert torch.equal(a, b)
    assert not bufs[1][V:stride].any() and not bufs[1][stride + V:2 * stride].any()


def test_tensors_that_are_refused():
    import paper_2606_26997_amd as rp
    n, V = 4, 50
    x, f, i = torch.zeros(n, V, device="cuda"), empty(n), empty(n, torch.int32)
    for bad, needle in ((x[:1].expand(n, V), "overlap"), (x.cpu(), "current GPU"), (x.double(), "dtype")):
        with pytest.raises(ValueError, match=needle):
            rp.sample_tokens(bad, f, i)
    for kw in (dict(temperature=f[:3]), dict(top_k=f), dict(top_p=f.double()), dict(min_p=f.cpu()),
               dict(temperature=torch.zeros(n, 2, device="cuda")[:, 0])):
        with pytest.raises(ValueError):
            rp.sample_tokens(x, f, i, **kw)
    with pytest.raises(ValueError, match="dlogits"):
        rp.policy_loss(x, i, f, f, f, torch.zeros(n, V + 1, device="cuda"))
    with pytest.raises(ValueError, match="dlogits"):
        rp.policy_loss(x, i, f, f, f, torch.zeros(n, V, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(rp.RpError, match="num_advantages"):
        rp.policy_loss(x, i, f, f[:2], f)
    with pytest.raises(ValueError, match="values"):
        rp.distill_loss(x, torch.zeros(n, 3, dtype=torch.int32, device="cuda"), torch.zeros(n, 2, device="cuda"), f)
    with pytest.raises(ValueError, match="ids"):
        rp.distill_loss(x, i, f, f)
    wide = torch.zeros(2, 1 << 20, device="cuda")
    with pytest.raises(rp.RpError) as e:
        rp.sample_tokens(wide, f[:2], i[:2])
    assert e.value.status == rp.RP_ERR_WORKSPACE
