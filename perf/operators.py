"""Operators of speculative decoding over the paged, group-shared KV cache: cases, inputs, plain forms, work.

  tree    attention of every sequence's tree of drafted tokens over the cache and the tree itself
  write   K/V rows written into the cache by slot: prompts, accepted drafts, single tokens
  tables  block tables and slot maps from lengths, pages taken from and given back to a free list

Lengths are the quantiles of a case's distribution in an order drawn from the seed, so every seed has the
same work and other data.
"""
import math

import numpy as np
import torch

own = False
PAGE = 16


# ---- cases -----------------------------------------------------------------
def _tree(name, *, hq, hkv, d, groups, size, prefix, resp, drafts, dtype="bf16"):
    return dict(name=name, op="tree", hq=hq, hkv=hkv, d=d, groups=groups, size=size, prefix_lo=prefix[0],
                prefix_hi=prefix[1], resp_lo=resp[0], resp_hi=resp[1], drafts_lo=drafts[0], drafts_hi=drafts[1],
                dtype=dtype)


def _write(name, *, hkv, d, seqs, start, new, dtype="bf16", gather=False):
    return dict(name=name, op="write", hkv=hkv, d=d, seqs=seqs, start_lo=start[0], start_hi=start[1], new_lo=new[0],
                new_hi=new[1], dtype=dtype, gather=gather)


def _tables(name, *, seqs, old, new, ending, spare):
    return dict(name=name, op="tables", seqs=seqs, old_lo=old[0], old_hi=old[1], new_lo=new[0], new_hi=new[1],
                ending=ending, spare=spare)


def listed():
    return [
        # One small group early in its rollout, four drafts each: all latency.
        _tree("tree_tiny", hq=4, hkv=2, d=64, groups=1, size=4, prefix=(128, 128), resp=(32, 64), drafts=(4, 4)),
        # Frontier dispatch: two groups of eight in flight, ragged trees of 1 to 16 drafts.
        _tree("tree_frontier", hq=16, hkv=8, d=128, groups=2, size=8, prefix=(512, 512), resp=(0, 6016),
              drafts=(1, 16)),
        # An ordinary batch in mid-rollout, chains and trees of eight drafts.
        _tree("tree_groups", hq=16, hkv=8, d=128, groups=32, size=8, prefix=(64, 512), resp=(0, 4096), drafts=(8, 8)),
        # Large trees and eight query heads per kv-head: the matrix products count.
        _tree("tree_wide", hq=32, hkv=4, d=128, groups=4, size=8, prefix=(1024, 1024), resp=(0, 2048),
              drafts=(64, 64)),
        # Long contexts in an fp8 cache, ragged trees.
        _tree("tree_fp8_long", hq=16, hkv=8, d=128, groups=4, size=16, prefix=(256, 256), resp=(8192, 32768),
              drafts=(1, 32), dtype="fp8"),
        # One token for each of four sequences: the smallest write.
        _write("write_tiny", hkv=2, d=64, seqs=4, start=(32, 64), new=(1, 1)),
        # The accepted drafts of a batch, picked out of all drafts, into an fp8 cache.
        _write("write_accepted", hkv=8, d=128, seqs=256, start=(0, 31), new=(1, 8), dtype="fp8", gather=True),
        # The prompts of a round.
        _write("write_prompts", hkv=8, d=128, seqs=64, start=(0, 0), new=(64, 1024)),
        # Long prompts into an fp8 cache, behind a part that is there already.
        _write("write_fp8_long", hkv=8, d=128, seqs=32, start=(0, 100), new=(2048, 4096), dtype="fp8"),
        # Room for the drafts of a frontier batch, given back when none is accepted.
        _tables("tables_step", seqs=16, old=(0, 6016), new=(1, 16), ending=0.0, spare=64),
        # A step of a large batch in which a quarter of the responses end; then those are admitted again.
        _tables("tables_round", seqs=1024, old=(1, 2048), new=(1, 8), ending=0.25, spare=2048),
        # The prompts of a large round admitted at once, and ended.
        _tables("tables_prompts", seqs=512, old=(0, 0), new=(64, 4096), ending=0.0, spare=0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _odd(rng, lo, hi):
    """Two lengths between lo and hi, in order, spread over the logarithm."""
    a, b = sorted((_log(rng, lo, hi), _log(rng, lo, hi)))
    return a, b


def draw(rng):
    op = rng.choice(["tree", "tree", "write", "tables"])
    while True:
        if op == "tree":
            hkv, size = rng.choice([1, 2, 4, 8]), _log(rng, 1, 16)
            c = _tree("", hq=hkv * rng.choice([1, 2, 4, 8]), hkv=hkv, d=rng.choice([64, 128]),
                      groups=_log(rng, 1, 32), size=size, prefix=_odd(rng, 1, 1024), resp=_odd(rng, 1, 16384),
                      drafts=_odd(rng, 1, 64), dtype=rng.choice(["bf16", "fp8"]))
            if rng.random() < 0.2:
                c["prefix_lo"] = 0
            if rng.random() < 0.2:
                c["resp_lo"] = 0
            S = c["groups"] * c["size"]
            padded = S * (c["prefix_hi"] + c["resp_hi"] + c["drafts_hi"])
            w = work(c)
            fits = (w["bytes"] <= 2e9 and w["flops"] <= 6e10 and padded * hkv * c["d"] <= 2e9
                    and padded * c["hq"] * c["drafts_hi"] <= 2e9)
        elif op == "write":
            start = (0, 0) if rng.random() < 0.3 else _odd(rng, 1, 64)
            c = _write("", hkv=rng.choice([1, 2, 4, 8]), d=rng.choice([64, 128]), seqs=_log(rng, 1, 512), start=start,
                       new=_odd(rng, 1, 4096), dtype=rng.choice(["bf16", "fp8"]), gather=rng.random() < 0.5)
            fits = work(c)["bytes"] <= 5e8
        else:
            old = (0, 0) if rng.random() < 0.2 else _odd(rng, 1, 8192)
            c = _tables("", seqs=_log(rng, 1, 2048), old=old, new=_odd(rng, 1, 4096),
                        ending=0.0 if old[1] == 0 else rng.choice([0.0, 0.1, 0.5]), spare=_log(rng, 1, 4096))
            fits = work(c)["bytes"] <= 1.1e7
        if fits:
            c.pop("name")
            return c


def _quantiles(lo, hi, n):
    return np.floor(lo + (hi - lo + 1) * (np.arange(n) + 0.5) / n).astype(np.int64).clip(lo, hi)


def _pages(x):
    return (x + PAGE - 1) // PAGE


def _shuffled(x):
    """The same order for every seed: what a case has to move goes by how its lengths are paired."""
    return x[np.argsort((np.arange(len(x)) * 7919) % 10007, kind="stable")]


def _write_lens(c):
    """Tokens there already, and new ones, of each sequence."""
    return (_shuffled(_quantiles(c["start_lo"], c["start_hi"], c["seqs"])),
            _quantiles(c["new_lo"], c["new_hi"], c["seqs"]))


def _resize_lens(c):
    """Lengths before and after the first of the two resizes; the first `ending` of the sequences end."""
    old = _shuffled(_quantiles(c["old_lo"], c["old_hi"], c["seqs"]))
    new = old + _quantiles(c["new_lo"], c["new_hi"], c["seqs"])
    new[:int(c["ending"] * c["seqs"])] = 0
    return old, new


def work(c):
    if c["op"] == "tree":
        S, e = c["groups"] * c["size"], 1 if c["dtype"] == "fp8" else 2
        P, L = _quantiles(c["prefix_lo"], c["prefix_hi"], c["groups"]), _quantiles(c["resp_lo"], c["resp_hi"], S)
        n = _quantiles(c["drafts_lo"], c["drafts_hi"], S)
        T, cached = int(n.sum()), int(P.sum() + L.sum())
        rows = 2 * c["hkv"] * c["d"]
        mean = float(P.mean() + L.mean())  # keys per draft; prefixes, lengths and trees are paired by the seed
        return {"bytes": float(cached * rows * e + T * rows * 2 + T * c["hq"] * (c["d"] * 4 + 4)
                               + (_pages(P).sum() + _pages(L).sum()) * (4 + (8 * c["hkv"] if e == 1 else 0)) + T * 8),
                "flops": 4.0 * T * c["hq"] * c["d"] * mean}
    if c["op"] == "write":
        T, e = int(_quantiles(c["new_lo"], c["new_hi"], c["seqs"]).sum()), 1 if c["dtype"] == "fp8" else 2
        return {"bytes": float(T * 2 * c["hkv"] * c["d"] * (2 + e) + T * (8 if c["gather"] else 4)), "flops": 0.0}
    old, new = _resize_lens(c)
    moved = int(np.abs(_pages(new) - _pages(old)).sum())
    return {"bytes": float(2 * (8 * c["seqs"] + 4 * (c["seqs"] + 1) + 8 * moved) + 4 * int(np.abs(new - old).sum())),
            "flops": 0.0}


# ---- inputs ----------------------------------------------------------------
def _pool(gen, pages, hkv, d, dtype, spread):
    """K or V pages: bf16, or e4m3fn codes and their (page, head) scales (amax / 448)."""
    if dtype == "bf16":
        return torch.randn(pages, hkv, PAGE, d, generator=gen, device="cuda", dtype=torch.bfloat16), None
    x = torch.randn(pages, hkv, PAGE, d, generator=gen, device="cuda", dtype=torch.bfloat16).float()
    if spread:
        x *= torch.exp(0.5 * torch.randn(pages, hkv, 1, 1, generator=gen, device="cuda"))
    scale = x.abs().amax((2, 3)) / 448
    return (x / scale[:, :, None, None]).to(torch.float8_e4m3fn).view(torch.uint8), scale


def _dev(x, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(x)).to("cuda", dtype)


def _block_table(ids, pages):
    """Rows of a block table: sequence s takes the next pages[s] of ids."""
    table = np.zeros((len(pages), max(1, int(pages.max()))), np.int64)
    at = np.arange(table.shape[1])[None] < pages[:, None]
    table[at] = ids[:int(pages.sum())]
    return table


def _ancestors(rng, counts):
    """Random trees: bit u of row (s, i) says that draft i of s sees draft u, itself included; packed."""
    S, n = len(counts), int(counts.max())
    mask = np.zeros((S, n), np.uint64)
    for i in range(n):
        parent = rng.integers(-1, i, S) if i else np.full(S, -1)
        chain = rng.random(S) < 0.5  # half of the drafts follow the one before
        parent = np.where(chain, i - 1, parent)
        up = np.where(parent >= 0, mask[np.arange(S), np.maximum(parent, 0)], np.uint64(0))
        mask[:, i] = up | (np.uint64(1) << np.uint64(i))
    return mask[np.arange(n)[None] < counts[:, None]]


def prepare(case, seed):
    c, rng = case, np.random.default_rng(seed)
    gen = torch.Generator("cuda").manual_seed(seed)
    if c["op"] == "tree":
        G, S = c["groups"], c["groups"] * c["size"]
        P = rng.permutation(_quantiles(c["prefix_lo"], c["prefix_hi"], G))
        L = rng.permutation(_quantiles(c["resp_lo"], c["resp_hi"], S))
        n = rng.permutation(_quantiles(c["drafts_lo"], c["drafts_hi"], S))
        pages = max(1, int(_pages(P).sum() + _pages(L).sum()))
        ids = rng.permutation(pages)
        s = dict(group=_dev(rng.permutation(np.repeat(np.arange(G), c["size"]))), prefix=_dev(P), resp=_dev(L),
                 prefix_table=_dev(_block_table(ids, _pages(P))),
                 resp_table=_dev(_block_table(ids[int(_pages(P).sum()):], _pages(L))),
                 offs=_dev(np.concatenate([[0], np.cumsum(n)])),
                 masks=torch.from_numpy(_ancestors(rng, n).view(np.int64)).to("cuda"), most=int(n.max()))
        s["k"], s["k_scale"] = _pool(gen, pages, c["hkv"], c["d"], c["dtype"], True)
        s["v"], s["v_scale"] = _pool(gen, pages, c["hkv"], c["d"], c["dtype"], True)
        T, new = int(n.sum()), dict(generator=gen, device="cuda", dtype=torch.bfloat16)
        s["q"] = torch.randn(T, c["hq"], c["d"], **new)
        s["kd"], s["vd"] = (torch.randn(T, c["hkv"], c["d"], **new) for _ in range(2))
        s["sigma"] = 1.0 / math.sqrt(c["d"])
    elif c["op"] == "write":
        S = c["seqs"]
        start, new = (x[p] for p in [rng.permutation(S)] for x in _write_lens(c))
        count = _pages(start + new)
        ids = rng.permutation(int(count.sum()))
        table, T = _block_table(ids, count), int(new.sum())
        seq = np.repeat(np.arange(S), new)
        t = start[seq] + np.arange(T) - np.repeat(np.cumsum(new) - new, new)
        rows = 2 * T if c["gather"] else T
        s = dict(slots=_dev(table[seq, t // PAGE] * PAGE + t % PAGE),
                 src=_dev(np.sort(rng.permutation(rows)[:T])) if c["gather"] else None)
        s["k"], s["k_scale"] = _pool(gen, int(count.sum()), c["hkv"], c["d"], c["dtype"], True)
        s["v"], s["v_scale"] = _pool(gen, int(count.sum()), c["hkv"], c["d"], c["dtype"], True)
        s["k_new"], s["v_new"] = (torch.randn(rows, c["hkv"], c["d"], generator=gen, device="cuda",
                                              dtype=torch.bfloat16) for _ in range(2))
    else:
        old, new = (x[p] for p in [rng.permutation(c["seqs"])] for x in _resize_lens(c))
        have, want = _pages(old), _pages(new)
        pages = int(np.maximum(have, want).sum()) + c["spare"]
        ids = rng.permutation(pages)
        held = int(have.sum())
        table = np.full((c["seqs"], max(1, int(max(have.max(), want.max())))), -1, np.int64)
        mine = _block_table(ids, have)
        table[:, :mine.shape[1]] = np.where(np.arange(mine.shape[1])[None] < have[:, None], mine, -1)
        free = np.zeros(pages, np.int64)
        free[:pages - held] = ids[held:]
        up, down = (int(np.maximum(x, 0).sum()) for x in (new - old, old - new))
        s = dict(old=_dev(old), new=_dev(new), table=_dev(table), free=_dev(free), count=_dev([pages - held]),
                 offs=[torch.empty(c["seqs"] + 1, dtype=torch.int32, device="cuda") for _ in range(2)],
                 slots=[torch.empty(x, dtype=torch.int32, device="cuda") for x in (up, down)],
                 status=[torch.empty(4, dtype=torch.int32, device="cuda") for _ in range(2)])
    s["op"] = c["op"]
    if own:
        _handles(s)
    return s


def _handles(s):
    """What a program keeps between calls: descriptors of its buffers, outputs and the workspace."""
    import paper_2606_26997_amd as rp
    s["rp"] = rp
    if s["op"] == "tables":
        s["tables"] = rp.page_tables(s["table"], s["free"], s["count"])
        return
    s["kv"] = rp.paged_kv(s["k"], s["v"], s["k_scale"], s["v_scale"])
    if s["op"] == "tree":
        s["layout"] = rp.group_layout(s["group"], s["prefix"], s["prefix_table"], s["resp"], s["resp_table"],
                                      num_q_heads=s["q"].shape[1])
        s["tree"] = rp.draft_tree(s["offs"], s["masks"], max_drafts=s["most"])
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(s["q"].shape[:2], dtype=torch.float32, device="cuda")
        size = rp.group_tree_attn_workspace_size(s["kv"], s["layout"], s["tree"])
        s["work"] = torch.empty(max(size, 256), dtype=torch.uint8, device="cuda")


# ---- one pass --------------------------------------------------------------
def run(state):
    s = state
    if own:
        rp = s["rp"]
        if s["op"] == "tree":
            rp.group_tree_attn(s["kv"], s["layout"], s["tree"], s["q"], s["kd"], s["vd"], s["sigma"], s["out"],
                               s["lse"], s["work"])
            return {"out": s["out"], "lse": s["lse"]}
        if s["op"] == "write":
            rp.kv_write_slots(s["kv"], s["slots"], s["k_new"], s["v_new"], s["src"])
            return _pools(s)
        rp.page_tables_resize(s["tables"], s["old"], s["new"], s["status"][0], s["offs"][0], s["slots"][0])
        rp.page_tables_resize(s["tables"], s["new"], s["old"], s["status"][1], s["offs"][1], s["slots"][1])
        return _table_outputs(s)
    if s["op"] == "tree":
        return _plain_tree(s)
    if s["op"] == "write":
        if s["k_scale"] is None:
            _plain_write(s["k"], s["slots"], s["k_new"], s["src"])
            _plain_write(s["v"], s["slots"], s["v_new"], s["src"])
        else:
            _plain_write_fp8(s["k"], s["k_scale"], s["slots"], s["k_new"], s["src"])
            _plain_write_fp8(s["v"], s["v_scale"], s["slots"], s["v_new"], s["src"])
        return _pools(s)
    _plain_resize(s, s["old"], s["new"], s["status"][0], s["offs"][0], s["slots"][0])
    _plain_resize(s, s["new"], s["old"], s["status"][1], s["offs"][1], s["slots"][1])
    return _table_outputs(s)


def _pools(s):
    if s["k_scale"] is None:
        return {"k": s["k"], "v": s["v"]}
    return {"k": s["k"].view(torch.float8_e4m3fn), "v": s["v"].view(torch.float8_e4m3fn), "k_scale": s["k_scale"],
            "v_scale": s["v_scale"]}


def _table_outputs(s):
    return {"table": s["table"], "free": s["free"], "count": s["count"], "offs": s["offs"], "slots": s["slots"],
            "status": s["status"]}


# ---- plain forms -----------------------------------------------------------
def _decoded(pages, scale, table):
    """The tokens of a block table's rows in fp32: [rows][Hkv][tokens][d]."""
    ids = table.long().reshape(-1)
    x = pages[ids].view(torch.float8_e4m3fn).float() if scale is not None else pages[ids].float()
    if scale is not None:
        x = x * scale[ids][:, :, None, None]
    n, m, hkv, d = table.shape[0], table.shape[1], pages.shape[1], pages.shape[3]
    return x.view(n, m, hkv, PAGE, d).transpose(1, 2).reshape(n, hkv, m * PAGE, d)


def _plain_tree(s):
    """Masked softmax over [prefix | response | drafts], padded to the longest of each."""
    S, (T, hq, d), hkv, n = s["group"].shape[0], s["q"].shape, s["k"].shape[1], s["most"]
    group, rep, dev = s["group"].long(), hq // hkv, s["q"].device
    first, count = s["offs"][:-1].long(), (s["offs"][1:] - s["offs"][:-1]).long()
    i = torch.arange(n, device=dev)
    live = i[None] < count[:, None]                                    # [S][n]
    token = torch.where(live, first[:, None] + i[None], 0)
    q = s["q"][token].float().view(S, n, hkv, rep, d).permute(0, 2, 1, 3, 4).reshape(S, hkv, n * rep, d)

    def keys(pages, scale, drafts):
        return torch.cat([_decoded(pages, scale, s["prefix_table"])[group], _decoded(pages, scale, s["resp_table"]),
                          drafts[token].float().transpose(1, 2)], 2)

    tp, tr = s["prefix_table"].shape[1] * PAGE, s["resp_table"].shape[1] * PAGE
    cached = torch.cat([torch.arange(tp, device=dev)[None] < s["prefix"][group][:, None],
                        torch.arange(tr, device=dev)[None] < s["resp"][:, None]], 1)
    sees = ((s["masks"][token][:, :, None] >> i[None, None]) & 1).bool() & live[:, :, None] & live[:, None, :]
    allowed = torch.cat([cached[:, None].expand(S, n, tp + tr), sees], 2)    # [S][n][N]
    scores = (q @ keys(s["k"], s["k_scale"], s["kd"]).transpose(2, 3)) * s["sigma"]
    scores = scores.view(S, hkv, n, rep, -1).masked_fill(~allowed[:, None, :, None], -math.inf)
    top = scores.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp(scores - top)
    total = p.sum(-1, keepdim=True)
    lse = (top + torch.log(total)).squeeze(-1)
    o = (p / torch.where(total == 0, 1.0, total)).view(S, hkv, n * rep, -1) @ keys(s["v"], s["v_scale"], s["vd"])
    o = o.view(S, hkv, n, rep, d).permute(0, 2, 1, 3, 4).reshape(S, n, hq, d)
    seq = torch.searchsorted(s["offs"][1:].contiguous(), torch.arange(T, device=dev, dtype=torch.int32), right=True)
    at = torch.arange(T, device=dev) - first[seq]
    return {"out": o[seq, at].to(torch.bfloat16), "lse": lse.permute(0, 2, 1, 3).reshape(S, n, hq)[seq, at]}


def _plain_write(pages, slots, rows, src):
    slot = slots.long()
    pages[slot // PAGE, :, slot % PAGE] = rows if src is None else rows[src.long()]


def _plain_write_fp8(codes, scale, slots, rows, src):
    """One scale per (page, head): set by a run from row 0, else kept or raised with the rows before requantised."""
    slot, x = slots.long(), (rows if src is None else rows[src.long()]).float()     # [T][Hkv][d]
    page, row = slot // PAGE, slot % PAGE
    n, hkv = scale.shape
    amax = torch.zeros(n, hkv, device=x.device).scatter_reduce(0, page[:, None].expand(-1, hkv), x.abs().amax(2), "amax")
    first = torch.full((n,), PAGE, device=x.device).scatter_reduce(0, page, row, "amin")[:, None]
    fresh = torch.where(amax > 0, amax / 448, 1.0)
    raised = (first > 0) & (first < PAGE) & ~(amax <= 448 * scale)
    now = torch.where((first == 0) | raised, torch.where(first == 0, fresh, amax / 448), scale)
    values = codes.view(torch.float8_e4m3fn).float() * scale[:, :, None, None]
    before = raised[:, :, None, None] & (torch.arange(PAGE, device=x.device)[None, None, :, None] < first[:, :, None, None])
    codes.copy_(torch.where(before, _e4m3(values / now[:, :, None, None]), codes))
    codes[page, :, row] = _e4m3(x / now[page][:, :, None])
    scale.copy_(now)


def _e4m3(x):
    return x.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)


def _plain_resize(s, old, new, status, offs, slots):
    table, dev = s["table"], s["table"].device
    have, want = _pages(old.long()), _pages(new.long())
    back, more = (have - want).clamp(min=0), (want - have).clamp(min=0)
    at = torch.arange(table.shape[1], device=dev)[None]
    gone = (at >= want[:, None]) & (at < have[:, None])
    come = (at >= have[:, None]) & (at < want[:, None])
    count, spare = s["count"].long(), s["free"].shape[0]
    returned, taken = back.sum(), more.sum()
    top = count + returned
    # Every table entry has a place of the stack: where its page goes or comes from; others one behind its end.
    rank = ((back.cumsum(0) - back)[:, None] + at - want[:, None])
    place = torch.where(gone, top - 1 - rank, spare)
    stack = torch.cat([s["free"], s["free"].new_zeros(1)])
    stack[place.reshape(-1)] = table.reshape(-1)
    rank = ((more.cumsum(0) - more)[:, None] + at - have[:, None])
    place = torch.where(come, top - 1 - rank, spare)
    page = stack[place]
    s["free"].copy_(stack[:-1])
    table.copy_(torch.where(come, page, torch.where(gone, -1, table)))
    s["count"].copy_(top - taken)
    fresh = (new - old).long().clamp(min=0)
    offs[0] = 0
    offs[1:] = fresh.cumsum(0)
    t = torch.arange(slots.shape[0], device=dev)
    seq = torch.searchsorted(offs[1:].contiguous(), t.int(), right=True)
    pos = old.long()[seq] + t - offs[:-1].long()[seq]
    slots.copy_(table.long()[seq, pos // PAGE] * PAGE + pos % PAGE)
    status.copy_(torch.stack([torch.zeros_like(taken), taken, returned, fresh.sum()]))


# ---- the definition in 64 bits ---------------------------------------------
def exact(case, seed):
    if case["op"] == "tables":
        return None  # whole numbers throughout
    s = prepare(case, seed)
    return _exact_tree(s) if case["op"] == "tree" else _exact_write(s)


def _tokens(pages, scale, table, length):
    """The first `length` tokens of one row of a block table, in 64 bits: [Hkv][length][d]."""
    ids = table[:(length + PAGE - 1) // PAGE].long()
    x = pages[ids]
    x = x.double() if scale is None else x.view(torch.float8_e4m3fn).double() * scale[ids].double()[:, :, None, None]
    return torch.cat(list(x), 1)[:, :length] if len(ids) else x.new_zeros(pages.shape[1], 0, pages.shape[3])


def _exact_tree(s):
    hkv = s["k"].shape[1]
    group, P, L, offs = (s[k].tolist() for k in ("group", "prefix", "resp", "offs"))
    masks = s["masks"].cpu().numpy().view(np.uint64)
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    for i, g in enumerate(group):
        a, b = offs[i], offs[i + 1]
        if a == b:
            continue
        k, v = (torch.cat([_tokens(s[x], s[x + "_scale"], s["prefix_table"][g], P[g]),
                           _tokens(s[x], s[x + "_scale"], s["resp_table"][i], L[i]),
                           s[x + "d"][a:b].double().transpose(0, 1)], 1) for x in ("k", "v"))
        hide = np.array([[not (int(masks[r]) >> u) & 1 for u in range(b - a)] for r in range(a, b)])
        for h in range(hkv):
            rep = s["q"].shape[1] // hkv
            q = s["q"][a:b, h * rep:(h + 1) * rep].double().reshape(-1, k.shape[2])
            score = torch.mm(q, k[h].t().contiguous()) * s["sigma"]
            score = score.view(b - a, rep, -1)
            score[:, :, P[g] + L[i]:].masked_fill_(torch.from_numpy(hide).to("cuda")[:, None], -math.inf)
            z = torch.logsumexp(score, 2)
            w = torch.where(torch.isfinite(z)[:, :, None], torch.exp(score - z[:, :, None]), 0.0)
            out[a:b, h * rep:(h + 1) * rep] = torch.mm(w.view((b - a) * rep, -1), v[h]).view(b - a, rep, -1)
            lse[a:b, h * rep:(h + 1) * rep] = z
    return {"out": out, "lse": lse}


def _exact_write(s):
    """bf16: the rows themselves. fp8: scales, and each element's unrounded multiple of its page's scale."""
    slots = s["slots"].long()
    src = torch.arange(slots.shape[0], device="cuda") if s["src"] is None else s["src"].long()
    page, row = slots // PAGE, slots % PAGE
    result = {}
    for x in ("k", "v"):
        rows = s[x + "_new"].double()[src]
        if s[x + "_scale"] is None:
            result[x] = s[x].double()
            result[x][page, :, row] = rows
            continue
        held, scale = s[x].view(torch.float8_e4m3fn).double(), s[x + "_scale"].double()
        dense = torch.full(held.shape, math.nan, dtype=torch.float64, device="cuda")
        dense[page, :, row] = rows
        touched = ~torch.isnan(dense[:, 0, :, 0])                      # [pages][rows]
        peak = dense.abs().nan_to_num(-1.0).amax((2, 3))
        begins, used = touched[:, :1], touched.any(1, keepdim=True)
        grown = torch.where(peak > 0, peak / 448, 1.0)
        # The comparison is the rule's own, of fp32 products.
        keeps = peak.float() <= 448 * s[x + "_scale"]
        now = torch.where(used & (begins | ~keeps), grown, scale)
        result[x] = torch.where(torch.isnan(dense), held * (scale / now)[:, :, None, None], dense / now[:, :, None, None])
        # Rows behind a page's run keep their codes whatever the scale.
        after = (torch.cummax(touched.int(), 1).values.bool() & ~touched)[:, None, :, None]
        result[x] = torch.where(after, held, result[x])
        result[x + "_scale"] = now
    return result
