"""Operators on rows of logits, of a GRPO rollout and its training: cases, inputs, plain forms, work.

  sample    one token per row, with temperature, top-k, top-p and min-p, from a given uniform number
  logprobs  the log-probabilities of given tokens, and the rows' entropies
  policy    GRPO's clipped policy loss with its KL and entropy terms, and its gradient
  distill   the divergence from a teacher of whom the top log-probabilities are known, and its gradient

Rows have a bulk of normally distributed logits, and `peak` > 0 lifts 32 tokens of each row by up to that much, as
a trained model's rows have a few likely tokens; without it a row is that of a model early in its training.
"""
import math

import torch

own = False
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
TAIL = 2.0 ** -24  # the least mass that a teacher leaves to the tokens that it does not list


# ---- cases -----------------------------------------------------------------
def _case(name, op, rows, vocab, dtype, peak=18.0, pad=0, masked=0, **more):
    return dict(name=name, op=op, rows=rows, vocab=vocab, dtype=dtype, peak=peak, pad=pad, masked=masked, **more)


def listed():
    return [
        # One sequence being decoded alone: all latency.
        _case("sample_one", "sample", 1, 32000, "bf16", filters="topk"),
        # Frontier dispatch, two groups of eight in flight: on-policy samples, nothing left out.
        _case("sample_frontier", "sample", 16, 151936, "bf16", masked=267, filters="none"),
        # A decode step of a batch whose requests ask for different things.
        _case("sample_step", "sample", 256, 151936, "bf16", masked=267, filters="mixed"),
        # Large nuclei of flat fp32 rows of an odd length.
        _case("sample_nucleus", "sample", 512, 50257, "f32", peak=0.0, filters="topp"),
        # The tokens of one short step under the present policy.
        _case("logprobs_step", "logprobs", 16, 32000, "f16", temperature=1.0),
        # The tokens of a few responses under the reference policy.
        _case("logprobs_round", "logprobs", 8192, 151936, "bf16", masked=267, temperature=1.0),
        # The loss of a few tokens.
        _case("policy_small", "policy", 24, 32000, "bf16", temperature=1.0, beta=0.0, entropy=0.0, skipped=0.0),
        # One micro-batch of a training step with every term, its last rows padding.
        _case("policy_update", "policy", 2048, 151936, "bf16", masked=267, temperature=0.9, beta=0.02, entropy=0.01,
              skipped=0.05),
        # fp32 logits with an odd row stride.
        _case("policy_f32", "policy", 1000, 50257, "f32", pad=6, temperature=1.0, beta=0.02, entropy=0.0, skipped=0.0),
        # A few tokens against a short list.
        _case("distill_small", "distill", 24, 32000, "bf16", temperature=1.0, k=16, kind="topk", skipped=0.0),
        # A micro-batch against a list and the mass outside it.
        _case("distill_tail", "distill", 2048, 151936, "bf16", masked=267, temperature=1.0, k=64, kind="tail",
              skipped=0.05),
        # The reverse divergence of on-policy distillation, long lists, rows of an odd length.
        _case("distill_reverse", "distill", 1500, 100003, "f16", temperature=1.0, k=200, kind="reverse", skipped=0.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["sample", "logprobs", "policy", "distill"])
    most = 4.0e7 if op == "sample" else 2.0e8  # elements of the logits
    while True:
        rows, vocab = _log(rng, 1, 8192), _log(rng, 16, 262144)
        if 2.0e3 <= rows * vocab <= most:
            break
    c = _case("", op, rows, vocab, rng.choice(["bf16", "bf16", "f16", "f32"]), peak=rng.choice([0.0, 10.0, 18.0]),
              pad=rng.choice([0, 0, rng.randint(1, 64)]), masked=rng.choice([0, vocab // 100]))
    if op == "sample":
        c["filters"] = rng.choice(["none", "topk", "topp", "minp", "mixed"])
    else:
        c["temperature"] = rng.choice([1.0, round(rng.uniform(0.6, 1.5), 3)])
    if op == "policy":
        c["beta"], c["entropy"] = rng.choice([0.0, 0.02]), rng.choice([0.0, 0.01])
    if op == "distill":
        c["k"], c["kind"] = min(_log(rng, 1, 256), vocab // 2), rng.choice(["topk", "tail", "reverse"])
    if op in ("policy", "distill"):
        c["skipped"] = rng.choice([0.0, 0.1])
    c.pop("name")
    return c


def _skipped(c):
    return int(c.get("skipped", 0.0) * c["rows"])


def work(c):
    """Logits read once (padding rows not at all), gradients written once, and what goes with each row."""
    size = 4 if c["dtype"] == "f32" else 2
    read, n = float((c["rows"] - _skipped(c)) * c["vocab"]), c["rows"]
    written = float(n * c["vocab"]) if c["op"] in ("policy", "distill") else 0.0
    each = {"sample": 28, "logprobs": 12, "policy": 32, "distill": 8 * c.get("k", 0) + 8}[c["op"]]
    return {"bytes": (read + written) * size + n * each, "flops": 2.0 * read + 4.0 * written}


# ---- inputs ----------------------------------------------------------------
def _logits(c, gen, pad):
    n, V = c["rows"], c["vocab"]
    buf = torch.randn(n, V + pad, generator=gen, device="cuda", dtype=DTYPES[c["dtype"]])
    buf *= 1.8 if c["peak"] else 2.5
    x = buf[:, :V]
    if c["peak"]:
        at = torch.randint(V, (n, min(32, V)), generator=gen, device="cuda")
        x.scatter_(1, at, (c["peak"] * torch.rand(at.shape, generator=gen, device="cuda")).to(x.dtype))
    if c["masked"]:
        x[:, V - c["masked"]:] = -math.inf
    return x


def _lse(x, temperature):
    """ln sum exp of each row's scaled logits, a few rows at a time."""
    return torch.cat([torch.logsumexp(y.float() / temperature, 1) for y in x.split(256)])


def prepare(case, seed):
    c = case
    n, V = c["rows"], c["vocab"]
    gen = torch.Generator("cuda").manual_seed(seed)
    f32 = dict(device="cuda", dtype=torch.float32)

    def rand(*shape):
        return torch.rand(*shape, generator=gen, device="cuda")

    def ints(lo, hi, *shape):
        return torch.randint(lo, hi, shape, generator=gen, device="cuda", dtype=torch.int32)

    s = dict(op=c["op"], logits=_logits(c, gen, c["pad"]))
    x, live = s["logits"], V - c["masked"]
    if c["op"] == "sample":
        s["u"] = rand(n)
        s["temperature"] = s["top_k"] = s["top_p"] = s["min_p"] = None
        if c["filters"] != "none":
            pick = {"topk": 2, "topp": 3, "minp": 4}.get(c["filters"])
            what = ints(0, 6, n) if pick is None else torch.full((n,), pick, device="cuda")
            # 0 greedy, 1 temperature alone, 2 top-k with a wide top-p, 3 top-p, 4 min-p, 5 all of them
            s["temperature"] = torch.where(what == 0, 0.0, 0.6 + 0.6 * rand(n))
            if pick in (None, 2):
                s["top_k"] = torch.where((what == 2) | (what == 5), ints(1, 100, n), 0).int()
            if pick in (None, 2, 3):
                s["top_p"] = torch.where(what == 3, 0.8 + 0.19 * rand(n),
                                         torch.where((what == 2) | (what == 5), 0.9 + 0.1 * rand(n), 1.0))
            if pick in (None, 4):
                s["min_p"] = torch.where((what == 4) | (what == 5), 0.01 + 0.1 * rand(n), 0.0)
    else:
        s["temperature"] = c["temperature"]
        s["skip"] = _skipped(c)
    if c["op"] in ("logprobs", "policy"):
        best = torch.cat([y.argmax(1) for y in x.split(256)]).int()
        s["tokens"] = torch.where(rand(n) < 0.7, best, ints(0, live, n))
    if c["op"] == "policy":
        logp = (x.gather(1, s["tokens"].long()[:, None])[:, 0].float() / c["temperature"] - _lse(x, c["temperature"]))
        s["old"] = logp + 0.15 * torch.randn(n, generator=gen, **f32)
        s["ref"] = logp + 0.3 * torch.randn(n, generator=gen, **f32) if c["beta"] else None
        # Responses of 1 to 64 tokens; a response's advantage is shared by its tokens, its mean is the loss.
        length = ints(1, 65, n)
        s["row_seq"] = torch.repeat_interleave(torch.arange(n, device="cuda"), length.long())[:n].int()
        s["advantages"] = torch.randn(n, generator=gen, **f32)
        s["weights"] = 1.0 / length[s["row_seq"].long()].float()
        s["tokens"][n - s["skip"]:] = -1
        s["terms"] = dict(clip_low=0.2, clip_high=0.28, kl_beta=c["beta"], entropy_coef=c["entropy"])
    if c["op"] == "distill":
        k, kind = min(c["k"], live), c["kind"]
        values, ids = [], []
        for y in x.split(256):
            t = y.float() / c["temperature"] + 0.7 * torch.randn(y.shape, generator=gen, **f32)
            v, i = t.topk(k, 1)
            values.append(v * c["temperature"] if kind == "topk" else v - torch.logsumexp(t, 1, keepdim=True))
            ids.append(i)
        s["values"], s["ids"] = torch.cat(values).float(), torch.cat(ids).int()
        s["weights"], s["kind"] = rand(n), kind
        s["weights"][n - s["skip"]:] = 0.0
    if own:
        _handles(s)
    return s


def _handles(s):
    """What a program keeps between calls: outputs and the workspace."""
    import paper_2606_26997_amd as rp
    n, f32 = s["logits"].shape[0], dict(dtype=torch.float32, device="cuda")
    s["rp"] = rp
    if s["op"] == "sample":
        s["tokens"] = torch.empty(n, dtype=torch.int32, device="cuda")
    s["a"], s["b"], s["c"] = (torch.empty(n, **f32) for _ in range(3))
    if s["op"] in ("policy", "distill"):
        s["grad"] = torch.empty(s["logits"].shape, dtype=s["logits"].dtype, device="cuda")
    s["work"] = torch.empty(max(rp.logits_workspace_size(s["logits"]), 256), dtype=torch.uint8, device="cuda")


# ---- one pass --------------------------------------------------------------
def run(state):
    s = state
    if own:
        rp = s["rp"]
        if s["op"] == "sample":
            rp.sample_tokens(s["logits"], s["u"], s["tokens"], s["a"], s["b"], temperature=s["temperature"],
                             top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"], workspace=s["work"])
            return {"tokens": s["tokens"], "logprobs": s["a"], "kept_logprobs": s["b"]}
        if s["op"] == "logprobs":
            rp.token_logprobs(s["logits"], s["tokens"], s["a"], s["b"], temperature=s["temperature"],
                              workspace=s["work"])
            return {"logprobs": s["a"], "entropy": s["b"]}
        if s["op"] == "policy":
            rp.policy_loss(s["logits"], s["tokens"], s["old"], s["advantages"], s["a"], s["grad"],
                           row_seq=s["row_seq"], weights=s["weights"], ref_logprobs=s["ref"], logprobs=s["b"],
                           entropy=s["c"], temperature=s["temperature"], workspace=s["work"], **s["terms"])
            return {"losses": s["a"], "logprobs": s["b"], "entropy": s["c"], "dlogits": s["grad"]}
        rp.distill_loss(s["logits"], s["ids"], s["values"], s["a"], s["grad"], kind=s["kind"], weights=s["weights"],
                        temperature=s["temperature"], workspace=s["work"])
        return {"losses": s["a"], "dlogits": s["grad"]}
    return {"sample": _plain_sample, "logprobs": _plain_logprobs, "policy": _plain_policy,
            "distill": _plain_distill}[s["op"]](s)


# ---- plain forms -----------------------------------------------------------
def _plain_sample(s):
    """In 64 bits throughout: a token hangs on which side of a border the random number lies."""
    x, dev = s["logits"].float(), s["logits"].device
    n, V = x.shape
    heat = torch.ones(n, device=dev) if s["temperature"] is None else s["temperature"]
    greedy = heat <= 0
    t = torch.where(greedy, 1.0, heat).double()[:, None]
    value, order = torch.sort(x, dim=1, descending=True, stable=True)
    top = value[:, :1].double()
    w = torch.exp((value.double() - top) / t)
    whole, best = w.sum(1), order[:, 0]
    keep = torch.ones(n, V, dtype=torch.bool, device=dev)
    if s["top_k"] is not None:
        k = torch.where(s["top_k"] > 0, s["top_k"], V)
        keep &= torch.arange(V, device=dev)[None] < k[:, None]
    if s["top_p"] is not None:
        p = s["top_p"].double()[:, None]
        left = torch.where(keep, w, 0.0)
        total = left.cumsum(1)
        keep &= (total - left < p * total[:, -1:]) | (p >= 1)
        del left, total
    if s["min_p"] is not None:
        keep &= w >= s["min_p"].double()[:, None]
    w = torch.zeros_like(w).scatter_(1, order, torch.where(keep, w, 0.0))
    del order, keep, value
    total = w.cumsum(1)
    kept = total[:, -1]
    token = (total <= s["u"].double()[:, None] * kept[:, None]).sum(1).clamp(max=V - 1)
    token = torch.where(greedy, best, token)
    mine = ((x.gather(1, token[:, None]).double() - top) / t)[:, 0]
    return {"tokens": token.int(), "logprobs": (mine - torch.log(whole)).float(),
            "kept_logprobs": torch.where(greedy, 0.0, mine - torch.log(kept)).float()}


def _rows(s):
    """Scaled logits less the row's largest, their exponentials, and those rounded sums that lose in 32 bits in 64."""
    x = s["logits"].float()
    top = x.amax(1, keepdim=True)
    d = (x - top) / s["temperature"]
    e = torch.exp(d)
    return x, top, d, e, e.sum(1, dtype=torch.float64)


def _of_tokens(s, x, top, total):
    at = s["tokens"].clamp(min=0).long()[:, None]
    return at, ((x.gather(1, at) - top).double() / s["temperature"])[:, 0] - torch.log(total)


def _entropy(d, e, total):
    return torch.log(total) - torch.where(e > 0, e * d, 0.0).sum(1, dtype=torch.float64) / total


def _plain_logprobs(s):
    x, top, d, e, total = _rows(s)
    return {"logprobs": _of_tokens(s, x, top, total)[1].float(), "entropy": _entropy(d, e, total).float()}


def _plain_policy(s):
    x, top, d, e, total = _rows(s)
    at, logp = _of_tokens(s, x, top, total)
    del x
    c, live = s["terms"], s["tokens"] >= 0
    H = _entropy(d, e, total)
    A, w = s["advantages"][s["row_seq"].long()].double(), torch.where(live, s["weights"], 0.0).double()
    r = torch.exp(logp - s["old"].double())
    free, held = r * A, r.clamp(1 - c["clip_low"], 1 + c["clip_high"]) * A
    loss = -torch.minimum(free, held) - c["entropy_coef"] * H
    g = torch.where(free <= held, -free, 0.0)
    if s["ref"] is not None:
        gap = s["ref"].double() - logp
        loss = loss + c["kl_beta"] * (torch.exp(gap) - gap - 1)
        g = g + c["kl_beta"] * (1 - torch.exp(gap))
    p = e / total.float()[:, None]
    grad = -g.float()[:, None] * p
    if c["entropy_coef"]:
        more = p * (d + (H - torch.log(total)).float()[:, None])
        grad += c["entropy_coef"] * torch.where(p > 0, more, 0.0)
        del more
    grad.scatter_add_(1, at, g.float()[:, None])
    grad *= (w / s["temperature"]).float()[:, None]
    return {"losses": torch.where(live, w * loss, 0.0).float(), "logprobs": torch.where(live, logp, 0.0).float(),
            "entropy": torch.where(live, H, 0.0).float(), "dlogits": grad.to(s["logits"].dtype)}


def _plain_distill(s):
    x, top, d, e, total = _rows(s)
    ids, w = s["ids"].long(), s["weights"].double()
    lq = (x.gather(1, ids) - top).double() / s["temperature"] - torch.log(total)[:, None]
    q = torch.exp(lq)
    del x, d
    t = s["values"].double()
    if s["kind"] == "topk":
        t = t / s["temperature"]
        t = t - t.amax(1, keepdim=True)
        lp = t - torch.log(torch.exp(t).sum(1, keepdim=True))
        P = torch.exp(lp)
        loss, others, mine = (P * (lp - lq)).sum(1), torch.ones_like(total), q - P
    else:
        lp, P = t, torch.exp(t)
        rest = (1 - P.sum(1)).clamp(min=TAIL)
        tail = e.scatter(1, ids, 0.0).sum(1, dtype=torch.float64) / total
        if s["kind"] == "tail":
            loss = (P * (lp - lq)).sum(1) + rest * (torch.log(rest) - torch.log(tail))
            whole = P.sum(1) + rest
            others, mine = whole - rest / tail, whole[:, None] * q - P
        else:
            gap = torch.log(tail) - torch.log(rest)
            loss = (q * (lq - lp)).sum(1) + tail * gap
            others, mine = gap - loss, q * (lq - lp - loss[:, None])
    scale = w / s["temperature"]
    grad = e * (scale * others / total).float()[:, None]
    grad.scatter_(1, ids, (scale[:, None] * mine).float())
    return {"losses": (w * loss).float(), "dlogits": grad.to(s["logits"].dtype)}


# ---- the definition in 64 bits ---------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    if s["op"] == "sample":
        return _exact_sample(s)
    parts = [_exact_rows(s, a, min(a + 64, case["rows"])) for a in range(0, case["rows"], 64)]
    return {key: torch.cat([p[key] for p in parts]) for key in parts[0]}


def _exact_sample(s):
    """Row by row, from the sizes of the three sets of likeliest tokens."""
    n, V = s["logits"].shape
    u = s["u"].tolist()
    heat, top_k, top_p, min_p = (None if s[k] is None else s[k].tolist()
                                 for k in ("temperature", "top_k", "top_p", "min_p"))
    logprobs, kept_logprobs = [], []
    for r in range(n):
        x = s["logits"][r].double()
        t = 1.0 if heat is None else heat[r]
        if t <= 0:
            logprobs.append(float(x.max() - torch.logsumexp(x, 0)))
            kept_logprobs.append(0.0)
            continue
        p = torch.softmax(x / t, 0)
        order = torch.argsort(-x, stable=True)
        sorted_p, size = p[order], V
        if top_k is not None and 0 < top_k[r] < V:
            size = top_k[r]
        if top_p is not None and top_p[r] < 1:
            mass = sorted_p[:size].cumsum(0)
            size = 1 + int((mass[:-1] < top_p[r] * mass[-1]).sum())
        if min_p is not None:
            size = min(size, int((sorted_p >= min_p[r] * sorted_p[0]).sum()))
        kept = torch.zeros(V, dtype=torch.float64, device="cuda")
        kept[order[:size]] = sorted_p[:size]
        mass = kept.cumsum(0)
        i = min(V - 1, int(torch.searchsorted(mass, u[r] * mass[-1], right=True)))
        logprobs.append(float(torch.log(p[i])))
        kept_logprobs.append(float(torch.log(p[i] / mass[-1])))
    return {"tokens": None, "logprobs": torch.tensor(logprobs, dtype=torch.float64),
            "kept_logprobs": torch.tensor(kept_logprobs, dtype=torch.float64)}


def _exact_rows(s, a, b):
    """Rows a .. b-1 from the losses' own formulas, gradients by differentiation."""
    x = s["logits"][a:b].double().requires_grad_()
    lp = torch.log_softmax(x / s["temperature"], 1)
    seen = torch.where(torch.isfinite(lp), lp, 0.0)
    entropy = -(torch.exp(lp) * seen).sum(1)
    if s["op"] == "distill":
        ids, t = s["ids"][a:b].long(), s["values"][a:b].double()
        lq = lp.gather(1, ids)
        if s["kind"] == "topk":
            target = torch.log_softmax(t / s["temperature"], 1)
            loss = (torch.exp(target) * (target - lq)).sum(1)
        else:
            rest = (1 - torch.exp(t).sum(1)).clamp(min=TAIL)
            tail = torch.exp(lp).scatter(1, ids, 0.0).sum(1)
            if s["kind"] == "tail":
                loss = (torch.exp(t) * (t - lq)).sum(1) + rest * torch.log(rest / tail)
            else:
                loss = (torch.exp(lq) * (lq - t)).sum(1) + tail * torch.log(tail / rest)
        loss = s["weights"][a:b].double() * loss
        return {"losses": loss.detach(), "dlogits": torch.autograd.grad(loss.sum(), x)[0]}
    tokens = s["tokens"][a:b].long()
    live = tokens >= 0
    logp = lp.gather(1, tokens.clamp(min=0)[:, None])[:, 0]
    if s["op"] == "logprobs":
        return {"logprobs": logp.detach(), "entropy": entropy.detach()}
    c, A = s["terms"], s["advantages"].double()[s["row_seq"][a:b].long()]
    r = torch.exp(logp - s["old"][a:b].double())
    loss = -torch.where(A >= 0, r.clamp(max=1 + c["clip_high"]), r.clamp(min=1 - c["clip_low"])) * A
    loss = loss - c["entropy_coef"] * entropy
    if s["ref"] is not None:
        gap = s["ref"][a:b].double() - logp
        loss = loss + c["kl_beta"] * (torch.exp(gap) - gap - 1)
    loss = torch.where(live, s["weights"][a:b].double() * loss, 0.0)
    return {"losses": loss.detach(), "logprobs": torch.where(live, logp, 0.0).detach(),
            "entropy": torch.where(live, entropy, 0.0).detach(), "dlogits": torch.autograd.grad(loss.sum(), x)[0]}
