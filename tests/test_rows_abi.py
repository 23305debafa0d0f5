"""Refusals of the calls on rows of logits, on the CPU: every check comes before a launch, and fake addresses are
never read."""
import ctypes
import math

import pytest
import torch

import paper_2606_26997_amd as rp
from paper_2606_26997_amd import _binding as B
from tests.test_abi import A

G = A + (1 << 30)  # a gradient elsewhere


def _logits(**kw):
    d = dict(data=A, num_rows=4, vocab=100, row_stride=104, dtype=0)
    d.update(kw)
    return B.RpLogits(d["data"], d["num_rows"], d["vocab"], d["row_stride"], d["dtype"])


def _ref(x):
    return None if x is None else ctypes.byref(x)


def _sample(logits, how=None, u=A, tokens=A, lp=A, kept=A, ws=A, ws_bytes=1 << 40):
    return rp.load().rp_sample_tokens(_ref(logits), _ref(how), u, tokens, lp, kept, ws, ws_bytes, None)


def _logprobs(logits, tokens=A, t=1.0, lp=A, ent=A, ws=A, ws_bytes=1 << 40):
    return rp.load().rp_token_logprobs(_ref(logits), tokens, t, lp, ent, ws, ws_bytes, None)


def _batch(**kw):
    d = dict(tokens=A, old=A, ref=A, adv=A, seq=A, num=3, weights=A, t=1.0, lo=0.2, hi=0.2, beta=0.1, ent=0.0)
    d.update(kw)
    return B.RpPolicyBatch(*d.values())


def _policy(logits, batch, losses=A, lp=A, ent=A, grad=G, stride=104, ws=A, ws_bytes=1 << 40):
    return rp.load().rp_policy_loss(_ref(logits), _ref(batch), losses, lp, ent, grad, stride, ws, ws_bytes, None)


def _teacher(**kw):
    d = dict(ids=A, values=A, k=8, kind=1, weights=A, t=1.0)
    d.update(kw)
    return B.RpTeacher(*d.values())


def _distill(logits, teacher, losses=A, grad=G, stride=104, ws=A, ws_bytes=1 << 40):
    return rp.load().rp_distill_loss(_ref(logits), _ref(teacher), losses, grad, stride, ws, ws_bytes, None)


def _size(logits):
    n = ctypes.c_size_t(12345)
    return rp.load().rp_logits_workspace_size(_ref(logits), ctypes.byref(n)), n.value


ROWS = [
    (dict(data=None), rp.RP_ERR_INVALID_ARG, "data"), (dict(data=A + 1), rp.RP_ERR_INVALID_ARG, "aligned"),
    (dict(data=A + 2, dtype=2), rp.RP_ERR_INVALID_ARG, "aligned"), (dict(num_rows=-1), rp.RP_ERR_INVALID_ARG, "num_rows"),
    (dict(vocab=0), rp.RP_ERR_INVALID_ARG, "vocab"), (dict(row_stride=99), rp.RP_ERR_INVALID_ARG, "row_stride"),
    (dict(row_stride=1 << 31), rp.RP_ERR_INVALID_ARG, "row_stride"),
    (dict(vocab=(1 << 20) + 1, row_stride=1 << 21), rp.RP_ERR_UNSUPPORTED, "limit"),
    (dict(dtype=3), rp.RP_ERR_UNSUPPORTED, "dtype"), (dict(dtype=-1), rp.RP_ERR_UNSUPPORTED, "dtype"),
]


@pytest.mark.parametrize("kw,status,needle", ROWS)
def test_rows_refused_by_every_call(kw, status, needle):
    l = _logits(**kw)
    for st in (lambda: _sample(l), lambda: _logprobs(l), lambda: _policy(l, _batch()), lambda: _distill(l, _teacher()),
               lambda: _size(l)[0]):
        assert st() == status and needle in rp.last_error()


def test_null_structs():
    for st in (_sample(None), _logprobs(None), _policy(None, _batch()), _distill(None, _teacher()), _size(None)[0],
               _policy(_logits(), None), _distill(_logits(), None),
               rp.load().rp_logits_workspace_size(_ref(_logits()), None)):
        assert st == rp.RP_ERR_INVALID_ARG


@pytest.mark.parametrize("kw", [dict(u=None), dict(u=A + 2), dict(tokens=None), dict(tokens=A + 1), dict(lp=A + 2),
                                dict(kept=A + 3), dict(how=B.RpSampling(A + 2, None, None, None)),
                                dict(how=B.RpSampling(None, A + 1, None, None)),
                                dict(how=B.RpSampling(None, None, A + 2, None)),
                                dict(how=B.RpSampling(None, None, None, A + 3))])
def test_sampling_refusals(kw):
    assert _sample(_logits(), **kw) == rp.RP_ERR_INVALID_ARG and rp.last_error()


BAD_T = [0.0, -1.0, math.inf, math.nan, 1e-320]


@pytest.mark.parametrize("kw", [dict(tokens=None), dict(lp=None), dict(lp=A + 2), dict(ent=A + 1)] + [dict(t=t) for t in BAD_T])
def test_logprob_refusals(kw):
    assert _logprobs(_logits(), **kw) == rp.RP_ERR_INVALID_ARG and rp.last_error()


@pytest.mark.parametrize("batch,call,needle", [
    (dict(tokens=None), {}, "tokens"), (dict(old=None), {}, "old_logprobs"), (dict(old=A + 2), {}, "aligned"),
    (dict(adv=None), {}, "advantages"), (dict(num=-1), {}, "num_advantages"), (dict(seq=None, num=3), {}, "num_advantages"),
    (dict(ref=None), {}, "ref_logprobs"), (dict(weights=A + 1), {}, "weights"), (dict(lo=-0.1), {}, "clip_low"),
    (dict(lo=math.nan), {}, "clip"), (dict(hi=-1.0), {}, "clip_high"), (dict(beta=math.inf), {}, "kl_beta"),
    (dict(beta=math.nan), {}, "kl_beta"), (dict(ent=math.nan), {}, "entropy_coef"), ({}, dict(losses=None), "losses"),
    ({}, dict(lp=A + 2), "logprobs"), ({}, dict(ent=A + 2), "entropy"), ({}, dict(grad=G + 1), "dlogits"),
    ({}, dict(stride=99), "dlogits_stride"), ({}, dict(stride=1 << 31), "dlogits_stride"),
    ({}, dict(grad=A, stride=105), "stride"), ({}, dict(grad=A + 2), "overlaps"), ({}, dict(grad=A - 10), "overlaps"),
] + [(dict(t=t), {}, "temperature") for t in BAD_T])
def test_policy_refusals(batch, call, needle):
    assert _policy(_logits(), _batch(**batch), **call) == rp.RP_ERR_INVALID_ARG and needle in rp.last_error()


@pytest.mark.parametrize("teacher,call,status,needle", [
    (dict(ids=None), {}, 1, "ids"), (dict(values=None), {}, 1, "values"), (dict(values=A + 2), {}, 1, "aligned"),
    (dict(k=0), {}, 1, "k must"), (dict(k=1025), {}, 2, "limit"), (dict(kind=3), {}, 2, "kind"),
    (dict(kind=-1), {}, 2, "kind"), (dict(weights=A + 2), {}, 1, "weights"), ({}, dict(losses=None), 1, "losses"),
    ({}, dict(grad=G + 1), 1, "dlogits"), ({}, dict(stride=99), 1, "dlogits_stride"),
    ({}, dict(grad=A + 200), 1, "overlaps"),
] + [(dict(t=t), {}, 1, "temperature") for t in BAD_T])
def test_distillation_refusals(teacher, call, status, needle):
    assert _distill(_logits(), _teacher(**teacher), **call) == status and needle in rp.last_error()


def test_no_rows_is_fine_without_anything_else():
    l = _logits(num_rows=0, data=None)
    assert _size(l) == (rp.RP_OK, 0)
    assert _sample(l, u=None, tokens=None, ws=None, ws_bytes=0) == rp.RP_OK
    assert _logprobs(l, tokens=None, lp=None, ws=None, ws_bytes=0) == rp.RP_OK
    assert _policy(l, _batch(), losses=None, ws=None, ws_bytes=0) == rp.RP_OK
    assert _distill(l, _teacher(), losses=None, ws=None, ws_bytes=0) == rp.RP_OK


def test_short_workspaces_are_refused():
    l = _logits(num_rows=1, vocab=1 << 20, row_stride=1 << 20)
    st, need = _size(l)
    assert st == rp.RP_OK
    if need == 0:
        pytest.skip("no shape of this size needs a workspace")
    for ws, size, status in [(None, 1 << 40, rp.RP_ERR_WORKSPACE), (A, need - 1, rp.RP_ERR_WORKSPACE),
                             (A + 128, need, rp.RP_ERR_INVALID_ARG)]:
        for st in (lambda: _sample(l, ws=ws, ws_bytes=size), lambda: _logprobs(l, ws=ws, ws_bytes=size),
                   lambda: _policy(l, _batch(), stride=1 << 20, ws=ws, ws_bytes=size),
                   lambda: _distill(l, _teacher(), stride=1 << 20, ws=ws, ws_bytes=size)):
            assert st() == status and "workspace" in rp.last_error()


CPU = dict(logits=torch.zeros(3, 8), i=torch.zeros(3, dtype=torch.int32), f=torch.zeros(3))


def test_binding_refuses_tensors_elsewhere_or_of_other_types():
    x, i, f = CPU["logits"], CPU["i"], CPU["f"]
    for call in (lambda l: rp.logits_workspace_size(l), lambda l: rp.sample_tokens(l, f, i),
                 lambda l: rp.token_logprobs(l, i, f), lambda l: rp.policy_loss(l, i, f, f, f),
                 lambda l: rp.distill_loss(l, i[:, None], f[:, None], f)):
        for logits, needle in [(x.double(), "dtype"), (x[0], "shape"), (x.t(), "contiguous"), (x, "current GPU")]:
            with pytest.raises(ValueError, match=needle):
                call(logits)
    with pytest.raises(ValueError, match="kind"):
        rp.distill_loss(x, i[:, None], f[:, None], f, kind="sideways")
