"""The operators together, as a rollout with drafted tokens uses them: tables from lengths, prompts and accepted
drafts written by slot, the drafts' attention and the decode step over the same cache; against dense fp64 keys."""
import numpy as np
import pytest
import torch

from oracle import e4m3_to_f64
from tests.paged import bf16_bits, bf16_value
from tests.tree_util import random_trees, say

pytestmark = pytest.mark.gpu


def _softmax_attention(q, K, V, sigma):
    s = sigma * np.einsum("hd,nhd->hn", q, K)
    m = s.max(1, keepdims=True)
    e = np.exp(s - m)
    return np.einsum("hn,nhd->hd", e / e.sum(1, keepdims=True), V), (m + np.log(e.sum(1, keepdims=True)))[:, 0]


def _bf16(x):
    return torch.from_numpy(x.view(np.int16)).view(torch.bfloat16).cuda()


@pytest.mark.parametrize("dtype,hq,hkv,d", [("bf16", 8, 4, 128), ("bf16", 16, 2, 64), ("fp8", 8, 2, 128)])
def test_rollout_with_drafts(dtype, hq, hkv, d):
    import paper_2606_26997_amd as rp
    say(f"speculative rollout {dtype} {hq} {hkv} {d}")
    rng = np.random.default_rng(hq + d)
    G, K, pages = 3, 4, 160
    S, rep, sigma = G * K, hq // hkv, float(np.float32(1 / np.sqrt(d)))
    P = np.array([37, 64, 5])
    if dtype == "bf16":
        k_pages, v_pages = (torch.full((pages, hkv, 16, d), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        k_scale = v_scale = None
    else:
        k_pages, v_pages = (torch.full((pages, hkv, 16, d), 0x7F, dtype=torch.uint8, device="cuda") for _ in range(2))
        k_scale, v_scale = (torch.full((pages, hkv), float("nan"), device="cuda") for _ in range(2))
    kv = rp.paged_kv(k_pages, v_pages, k_scale, v_scale)
    prefix = rp.PageTables(num_seqs=G, max_pages=6, num_pages=pages)
    resp = rp.PageTables(num_seqs=S, max_pages=12, stack=prefix.stack)
    group = torch.arange(S, dtype=torch.int32, device="cuda") // K
    layout = rp.group_layout(group, prefix.lens, prefix.block_table, resp.lens, resp.block_table, num_q_heads=hq)

    # Prompts: pages from their lengths, rows by slot.
    T = int(P.sum())
    new = [bf16_bits(rng.standard_normal((T, hkv, d))) for _ in range(2)]
    slots = torch.empty(T, dtype=torch.int32, device="cuda")
    prefix.resize(torch.from_numpy(P.astype(np.int32)).cuda(), slots)
    rp.kv_write_slots(kv, slots, _bf16(new[0]), _bf16(new[1]))
    rows = {("p", g): [x[sum(P[:g]):sum(P[:g + 1])] for x in new] for g in range(G)}
    for s in range(S):
        rows["r", s] = [np.zeros((0, hkv, d), np.uint16) for _ in range(2)]

    def cached(s):
        """The sequence's cached keys and values: what was written, or, in fp8, what the pages hold of it."""
        if dtype == "bf16":
            return [bf16_value(np.concatenate([rows["p", s // K][i], rows["r", s][i]])) for i in range(2)]
        out = []
        for codes, scale in ((k_pages, k_scale), (v_pages, v_scale)):
            x = e4m3_to_f64(codes.cpu().numpy()) * scale.cpu().numpy().astype(np.float64)[:, :, None, None]
            t = [prefix.block_table[s // K, u // 16].item() * 16 + u % 16 for u in range(P[s // K])]
            t += [resp.block_table[s, u // 16].item() * 16 + u % 16 for u in range(len(rows["r", s][0]))]
            t = np.array(t)
            out.append(x[t // 16, :, t % 16])
            written = bf16_value(np.concatenate([rows["p", s // K][len(out) - 1], rows["r", s][len(out) - 1]]))
            # A stored value is off by at most 2^-4 of itself, or half the smallest step, a few times over
            # (once more for each time that its page's scale rose behind it: at most 3 rounds here).
            step = 2.0 ** -9 * np.nanmax(scale.cpu().numpy())  # pages never written have a scale of NaN
            off = np.abs(out[-1] - written) / (2.0 ** -4 * np.abs(written) + step)
            assert off.max(initial=0) <= 4
        return out

    for step in range(3):
        counts = rng.integers(1, 9, S)
        counts[step] = 0
        offs = np.concatenate([[0], np.cumsum(counts)])
        T = int(offs[-1])
        masks = random_trees(rng, counts)
        q = bf16_bits(rng.standard_normal((T, hq, d)))
        kd, vd = (bf16_bits(rng.standard_normal((T, hkv, d))) for _ in range(2))
        tree = rp.draft_tree(torch.from_numpy(offs.astype(np.int32)).cuda(), torch.from_numpy(masks.view(np.int64)).cuda(),
                             max_drafts=8)
        out = torch.empty(T, hq, d, dtype=torch.bfloat16, device="cuda")
        lse = torch.empty(T, hq, device="cuda")
        work = torch.empty(max(256, rp.group_tree_attn_workspace_size(kv, layout, tree)), dtype=torch.uint8, device="cuda")
        args = _bf16(q), _bf16(kd), _bf16(vd)
        rp.group_tree_attn(kv, layout, tree, *args, sigma, out, lse, work)
        torch.cuda.synchronize()
        got, got_lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
        for s in range(S):
            if counts[s] == 0:
                continue
            K_, V_ = cached(s)
            for t in range(offs[s], offs[s + 1]):
                see = [u for u in range(counts[s]) if int(masks[t]) >> u & 1]
                Kt = np.concatenate([K_, bf16_value(kd[offs[s]:offs[s + 1]][see])]).repeat(rep, 1)
                Vt = np.concatenate([V_, bf16_value(vd[offs[s]:offs[s + 1]][see])]).repeat(rep, 1)
                o, l = _softmax_attention(bf16_value(q[t]), Kt, Vt, sigma)
                # Roundings to bf16 of the probabilities and the output, 2^-8 each, of values up to max |v|.
                assert np.abs(got[t] - o).max() <= 3 * 2.0 ** -8 * np.abs(Vt).max()
                assert np.abs(got_lse[t] - l).max() <= 1e-4
        # One leaf of each tree is accepted: its path joins the cache, by slot, straight from the drafts.
        paths = []
        for s in range(S):
            m = int(masks[offs[s] + int(rng.integers(0, counts[s]))]) if counts[s] else 0
            paths.append([offs[s] + u for u in range(counts[s]) if m >> u & 1])
            for i, x in enumerate((kd, vd)):
                rows["r", s][i] = np.concatenate([rows["r", s][i], x[paths[-1]]])
        src = np.array([t for p in paths for t in p], np.int32)
        new_lens = torch.tensor([len(rows["r", s][0]) for s in range(S)], dtype=torch.int32, device="cuda")
        slots = torch.empty(T, dtype=torch.int32, device="cuda")  # room for all drafts: the rest is -1
        resp.resize(new_lens, slots)
        pad = np.zeros(T, np.int32)
        pad[:len(src)] = src
        rp.kv_write_slots(kv, slots, args[1], args[2], torch.from_numpy(pad).cuda())
        torch.cuda.synchronize()
        assert resp.status[0].item() == rp.RP_TABLES_OK
        rp.validate_layout(kv, layout)

    # The decode attention reads the same cache.
    q = bf16_bits(rng.standard_normal((S, hq, d)))
    out = torch.empty(S, hq, d, dtype=torch.bfloat16, device="cuda")
    lse = torch.empty(S, hq, device="cuda")
    work = torch.empty(rp.group_decode_attn_workspace_size(kv, layout), dtype=torch.uint8, device="cuda")
    rp.group_decode_attn(kv, layout, _bf16(q), sigma, out, lse, work)
    torch.cuda.synchronize()
    for s in range(S):
        K_, V_ = cached(s)
        o, l = _softmax_attention(bf16_value(q[s]), K_.repeat(rep, 1), V_.repeat(rep, 1), sigma)
        assert np.abs(out[s].double().cpu().numpy() - o).max() <= 3 * 2.0 ** -8 * np.abs(V_).max()
        assert np.abs(lse[s].double().cpu().numpy() - l).max() <= 1e-4
    # Sequences that end give their pages back.
    resp.resize(torch.zeros_like(resp.lens))
    prefix.resize(torch.zeros_like(prefix.lens))
    torch.cuda.synchronize()
    assert prefix.stack[1].item() == pages and sorted(prefix.stack[0].tolist()) == list(range(pages))
