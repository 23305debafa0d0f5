"""Attention of trees of drafted tokens over the paged, group-shared cache, from the definition.

Draft ``i`` of sequence ``s`` (row ``t = draft_offs[s] + i``) attends to the keys of
``decode_attention`` for ``s`` and to the drafts ``u`` of ``s`` with bit ``u`` of ``masks[t]``:
``lse = log sum exp(sigma q k)``, ``out = sum exp(sigma q k - lse) v``; no key: 0 and -inf.
"""
import numpy as np

from .attention import _gather, key_slots
from .formats import bf16_to_f64


def tree_attention(*, k_pages, v_pages, k_scale, v_scale, kv_dtype, page_size, seq_to_group, prefix_lens,
                   prefix_block_table, resp_lens, resp_block_table, draft_offs, masks, q, k_draft, v_draft,
                   softmax_scale):
    """fp64 ``(out [T][Hq][d], lse [T][Hq], spread, reach)``, and two measures of how far roundings can move them:
    ``spread = sum exp(s - lse) |v|`` and ``reach = max_u sigma sum_i |q_i k_ui|`` over the row's keys."""
    T, Hq, d = q.shape
    Hkv = k_pages.shape[1]
    rep, sigma = Hq // Hkv, np.float64(np.float32(softmax_scale))
    out, spread = np.zeros((T, Hq, d)), np.zeros((T, Hq, d))
    lse, reach = np.full((T, Hq), -np.inf), np.zeros((T, Hq))
    qf, kd, vd = bf16_to_f64(q), bf16_to_f64(k_draft), bf16_to_f64(v_draft)
    for s in range(len(seq_to_group)):
        a, b = int(draft_offs[s]), int(draft_offs[s + 1])
        if a == b:
            continue
        pages, rows = key_slots(seq_to_group, prefix_lens, prefix_block_table, resp_lens, resp_block_table, s,
                                page_size)
        for h in range(Hkv):
            K = _gather(k_pages, k_scale, kv_dtype, pages, rows, h)
            V = _gather(v_pages, v_scale, kv_dtype, pages, rows, h)
            for t in range(a, b):
                see = np.array([bool(int(masks[t]) >> u & 1) for u in range(b - a)])
                Kt = np.concatenate([K, kd[a:b, h][see]])
                Vt = np.concatenate([V, vd[a:b, h][see]])
                if not len(Kt):
                    continue
                for j in range(h * rep, (h + 1) * rep):
                    with np.errstate(invalid="ignore", over="ignore"):
                        sc = sigma * (Kt @ qf[t, j])
                        m = sc.max()
                        lse[t, j] = m + np.log(np.exp(sc - m).sum())
                        w = np.exp(sc - lse[t, j])
                        out[t, j] = (w[:, None] * Vt).sum(0)
                        spread[t, j] = (w[:, None] * np.abs(Vt)).sum(0)
                        reach[t, j] = (sigma * (np.abs(Kt) @ np.abs(qf[t, j]))).max()
    return out, lse, spread, reach


def tree_for_workload(wl, draft_offs, masks, q, k_draft, v_draft):
    """Oracle result for a generated workload's cache (``resp_lens`` cached tokens) and the given drafts."""
    return tree_attention(k_pages=wl.k_pages, v_pages=wl.v_pages, k_scale=wl.k_scale, v_scale=wl.v_scale,
                          kv_dtype=wl.kv_dtype, page_size=wl.page_size, seq_to_group=wl.seq_to_group,
                          prefix_lens=wl.prefix_lens, prefix_block_table=wl.prefix_block_table,
                          resp_lens=wl.resp_lens, resp_block_table=wl.resp_block_table, draft_offs=draft_offs,
                          masks=masks, q=q, k_draft=k_draft, v_draft=v_draft, softmax_scale=wl.softmax_scale)
