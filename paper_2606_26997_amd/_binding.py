"""ctypes binding for librp.so: argument marshalling only.

Every computation runs in the HIP library. torch is imported first so that the
library's HIP runtime dependency resolves to the runtime torch already loaded;
tensors are passed by ``data_ptr()`` and streams by their raw HIP handle.
If the library is missing or cannot be loaded, every call raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import torch  # noqa: F401  (loads torch's HIP runtime before librp.so)

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "librp.so")

RP_OK = 0
RP_ERR_INVALID_ARG = 1
RP_ERR_UNSUPPORTED = 2
RP_ERR_WORKSPACE = 3
RP_ERR_HIP = 4
RP_ERR_LAYOUT = 5
RP_KV_BF16 = 0
RP_KV_FP8_E4M3 = 1
RP_NOALLOC_SCRATCH_BYTES = 64 << 20   # include/rp.h: static scratch of rp_group_decode_attn_noalloc

EXPORTED = ("rp_status_string", "rp_last_error", "rp_kv_append",
            "rp_group_decode_attn_workspace_size", "rp_group_decode_attn", "rp_lse_combine",
            "rp_plan", "rp_attn_parts", "rp_combine_parts", "rp_plan_layout", "rp_validate_layout",
            "rp_prefill_kv_write", "rp_prefill_attn", "rp_decode_qk_prep", "rp_sched_simulate",
            "rp_grpo_advantage", "rp_prefill", "rp_group_decode_attn_noalloc", "rp_decode_qk_prep_plan",
            "rp_selftest_mfma", "rp_stream_read", "rp_group_tree_attn_workspace_size", "rp_group_tree_attn",
            "rp_kv_write_slots", "rp_page_tables_resize")
# include/rp.h rp_tables_status, as the device's status[0] holds it
RP_TABLES_OK, RP_TABLES_NO_PAGES, RP_TABLES_BAD_LENGTH, RP_TABLES_NO_SLOTS, RP_TABLES_BAD_FREE_LIST = range(5)
RP_STREAM_READ_SINK_WORDS = 2048 * 4   # include/rp.h
# include/rp.h rp_selftest_shape: name -> (code, M, N, K)
RP_SELFTEST_SHAPES = {"16x16x32": (0, 16, 16, 32), "16x16x16": (1, 16, 16, 16), "16x16x32_lds_tr": (2, 16, 16, 32)}
RP_SCHED_MODES = {"slime": 0, "cgp": 1, "cgp_fgd": 2}


class RpPagedKV(ctypes.Structure):
    _fields_ = [("k_pages", ctypes.c_void_p), ("v_pages", ctypes.c_void_p),
                ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
                ("num_pages", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("kv_dtype", ctypes.c_int32)]


class RpGroupLayout(ctypes.Structure):
    _fields_ = [("num_seqs", ctypes.c_int32), ("num_groups", ctypes.c_int32),
                ("num_q_heads", ctypes.c_int32),
                ("seq_to_group", ctypes.c_void_p), ("prefix_lens", ctypes.c_void_p),
                ("prefix_block_table", ctypes.c_void_p), ("max_prefix_pages", ctypes.c_int32),
                ("resp_lens", ctypes.c_void_p), ("resp_block_table", ctypes.c_void_p),
                ("max_resp_pages", ctypes.c_int32)]


class RpPrefillLayout(ctypes.Structure):
    _fields_ = [("num_groups", ctypes.c_int32), ("num_q_heads", ctypes.c_int32), ("num_tokens", ctypes.c_int32),
                ("prompt_offs", ctypes.c_void_p), ("prefix_block_table", ctypes.c_void_p),
                ("max_prefix_pages", ctypes.c_int32)]


class RpDraftTree(ctypes.Structure):
    _fields_ = [("num_drafts", ctypes.c_int32), ("max_drafts", ctypes.c_int32), ("draft_offs", ctypes.c_void_p),
                ("masks", ctypes.c_void_p)]


class RpPageTables(ctypes.Structure):
    _fields_ = [("num_seqs", ctypes.c_int32), ("max_pages", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("num_pages", ctypes.c_int32), ("block_table", ctypes.c_void_p), ("free_pages", ctypes.c_void_p),
                ("free_count", ctypes.c_void_p)]


class RpPlanInfo(ctypes.Structure):
    _fields_ = [(n, ctypes.c_size_t) for n in ("hdr", "grp_off", "grp_members", "prefix_items", "resp_items",
                                                 "seq_parts", "part_o", "part_lse")] + \
               [(n, ctypes.c_int32) for n in ("max_prefix_items", "max_resp_items", "parts_per_row", "max_parts")]


class RpSchedConfig(ctypes.Structure):
    _fields_ = [("mode", ctypes.c_int32), ("num_groups", ctypes.c_int32), ("group_size", ctypes.c_int32),
                ("update_groups", ctypes.c_int32), ("frontier_width", ctypes.c_int32),
                ("max_running", ctypes.c_int32)] + \
               [(n, ctypes.c_double) for n in ("step_base", "step_per_seq", "step_per_ctx_token", "prefill_per_token",
                                                "mat_base", "mat_per_token", "train_base", "train_per_token",
                                                "opt_step")]


class RpSchedSummary(ctypes.Structure):
    _fields_ = [(n, ctypes.c_double) for n in ("t_first_u", "t_complete", "t_start", "delta_cgp", "t_train_end",
                                                "compute", "wait", "w_train", "wait_ratio")] + \
               [("steps", ctypes.c_int64)]


class RpError(RuntimeError):
    def __init__(self, status: int, func: str, detail: str):
        self.status = status
        super().__init__(f"{func}: {status_string(status)}: {detail}")


_lib = None


def load() -> ctypes.CDLL:
    """Load librp.so (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with __graft_entry__.build()")
    lib = ctypes.CDLL(LIB_PATH)
    P, I32, F32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_float
    sig = {
        "rp_status_string": (ctypes.c_char_p, [ctypes.c_int]),
        "rp_last_error": (ctypes.c_char_p, []),
        "rp_kv_append": (ctypes.c_int, [P, P, P, P, P]),
        "rp_group_decode_attn_workspace_size": (ctypes.c_int, [P, P, ctypes.POINTER(ctypes.c_size_t)]),
        "rp_group_decode_attn": (ctypes.c_int, [P, P, P, F32, P, P, P, ctypes.c_size_t, P]),
        "rp_group_decode_attn_noalloc": (ctypes.c_int, [P, P, P, F32, P, P, P]),
        "rp_lse_combine": (ctypes.c_int, [P, P, P, I32, I32, P, P, P]),
        "rp_plan": (ctypes.c_int, [P, P, P, ctypes.c_size_t, P]),
        "rp_attn_parts": (ctypes.c_int, [P, P, P, F32, P, ctypes.c_size_t, P]),
        "rp_combine_parts": (ctypes.c_int, [P, P, P, P, P, ctypes.c_size_t, P]),
        "rp_plan_layout": (ctypes.c_int, [P, P, P]),
        "rp_validate_layout": (ctypes.c_int, [P, P, P]),
        "rp_prefill_kv_write": (ctypes.c_int, [P, P, P, P, P]),
        "rp_prefill_attn": (ctypes.c_int, [P, P, P, P, P, F32, P, P, P]),
        "rp_prefill": (ctypes.c_int, [P, P, P, P, P, F32, P, P, P]),
        "rp_decode_qk_prep": (ctypes.c_int, [P, P, P, P, P, P, P, ctypes.c_double, ctypes.c_double, P, P, P]),
        "rp_decode_qk_prep_plan": (ctypes.c_int, [P, P, P, P, P, P, P, ctypes.c_double, ctypes.c_double, P, P, P,
                                                   ctypes.c_size_t, P]),
        "rp_sched_simulate": (ctypes.c_int, [P, P, P, P, P, P, P, P, P, P]),
        "rp_grpo_advantage": (ctypes.c_int, [P, I32, I32, ctypes.c_double, I32, P, P, P, P]),
        "rp_selftest_mfma": (ctypes.c_int, [I32, P, P, P, P]),
        "rp_group_tree_attn_workspace_size": (ctypes.c_int, [P, P, P, ctypes.POINTER(ctypes.c_size_t)]),
        "rp_group_tree_attn": (ctypes.c_int, [P, P, P, P, P, P, F32, P, P, P, ctypes.c_size_t, P]),
        "rp_kv_write_slots": (ctypes.c_int, [P, P, I32, P, P, P, I32, P]),
        "rp_page_tables_resize": (ctypes.c_int, [P, P, P, P, P, P, I32, P]),
        "rp_stream_read": (ctypes.c_int, [P, ctypes.c_uint64, P, I32, P]),
    }
    for name, (res, args) in sig.items():
        f = getattr(lib, name)
        f.restype, f.argtypes = res, args
    _lib = lib
    return lib


def status_string(status: int) -> str:
    return load().rp_status_string(int(status)).decode()


def last_error() -> str:
    return load().rp_last_error().decode()


def _check(status: int, func: str) -> None:
    if status != RP_OK:
        raise RpError(status, func, last_error())


def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _stream(stream) -> Optional[int]:
    if stream is None:
        # The raw handle of torch's current stream: a Stream object costs 2.7 us, more than a launch.
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device()) \
            if torch.cuda.is_initialized() or torch.cuda.is_available() else None
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _holding(descriptor, *tensors):
    """The descriptor, with the tensors behind its addresses alive for as long as it is."""
    descriptor.tensors = tuple(t for t in tensors if isinstance(t, torch.Tensor))
    return descriptor


def paged_kv(k_pages, v_pages, k_scale=None, v_scale=None, *, num_pages=None, num_kv_heads=None,
             page_size=16, head_dim=None, kv_dtype=None) -> RpPagedKV:
    """Describe a pool of tensors shaped [num_pages][Hkv][page_size][head_dim]."""
    shape = tuple(k_pages.shape) if hasattr(k_pages, "shape") else None
    if kv_dtype is None:
        kv_dtype = RP_KV_FP8_E4M3 if k_scale is not None else RP_KV_BF16
    kv = RpPagedKV(_ptr(k_pages), _ptr(v_pages), _ptr(k_scale), _ptr(v_scale),
                   num_pages if num_pages is not None else shape[0],
                   num_kv_heads if num_kv_heads is not None else shape[1],
                   page_size, head_dim if head_dim is not None else shape[3], kv_dtype)
    return _holding(kv, k_pages, v_pages, k_scale, v_scale)


def group_layout(seq_to_group, prefix_lens, prefix_block_table, resp_lens, resp_block_table, *,
                 num_q_heads, num_seqs=None, num_groups=None, max_prefix_pages=None,
                 max_resp_pages=None) -> RpGroupLayout:
    layout = RpGroupLayout(
        num_seqs if num_seqs is not None else seq_to_group.shape[0],
        num_groups if num_groups is not None else prefix_lens.shape[0],
        num_q_heads, _ptr(seq_to_group), _ptr(prefix_lens), _ptr(prefix_block_table),
        max_prefix_pages if max_prefix_pages is not None else prefix_block_table.shape[1],
        _ptr(resp_lens), _ptr(resp_block_table),
        max_resp_pages if max_resp_pages is not None else resp_block_table.shape[1])
    return _holding(layout, seq_to_group, prefix_lens, prefix_block_table, resp_lens, resp_block_table)


def kv_append(kv: RpPagedKV, layout: RpGroupLayout, k_new, v_new, stream=None) -> None:
    _check(load().rp_kv_append(ctypes.byref(kv), ctypes.byref(layout), _ptr(k_new), _ptr(v_new),
                               _stream(stream)), "rp_kv_append")


def decode_qk_prep(kv, layout, q_in, k_in, v_in, q_norm_w, k_norm_w, q_out, k_out=None, *,
                   rms_eps=1e-6, rope_theta=1e6, stream=None) -> None:
    _check(load().rp_decode_qk_prep(ctypes.byref(kv), ctypes.byref(layout), _ptr(q_in), _ptr(k_in), _ptr(v_in),
                                    _ptr(q_norm_w), _ptr(k_norm_w), float(rms_eps), float(rope_theta),
                                    _ptr(q_out), _ptr(k_out), _stream(stream)),
           "rp_decode_qk_prep")


def decode_qk_prep_plan(kv, layout, q_in, k_in, v_in, q_norm_w, k_norm_w, q_out, k_out, workspace, *,
                        rms_eps=1e-6, rope_theta=1e6, stream=None) -> None:
    """q/k prep with the append (``layout``: pre-append lengths) and the plan of the attention over the
    advanced lengths, in ``workspace``."""
    _check(load().rp_decode_qk_prep_plan(ctypes.byref(kv), ctypes.byref(layout), _ptr(q_in), _ptr(k_in),
                                         _ptr(v_in), _ptr(q_norm_w), _ptr(k_norm_w), float(rms_eps),
                                         float(rope_theta), _ptr(q_out), _ptr(k_out), _ptr(workspace),
                                         _ws_bytes(workspace), _stream(stream)),
           "rp_decode_qk_prep_plan")


def grpo_advantage(rewards, advantages, group_mean=None, group_std=None, *, eps_std=1e-6, ddof=1,
                   stream=None) -> None:
    """rewards, advantages: fp32 device tensors [R][K]; group_mean, group_std: [R] or None."""
    R, K = int(rewards.shape[0]), int(rewards.shape[1])
    _check(load().rp_grpo_advantage(_ptr(rewards), R, K, float(eps_std), int(ddof), _ptr(advantages),
                                    _ptr(group_mean), _ptr(group_std), _stream(stream)), "rp_grpo_advantage")


def group_decode_attn_workspace_size(kv: RpPagedKV, layout: RpGroupLayout) -> int:
    n = ctypes.c_size_t(0)
    _check(load().rp_group_decode_attn_workspace_size(ctypes.byref(kv), ctypes.byref(layout),
                                                      ctypes.byref(n)),
           "rp_group_decode_attn_workspace_size")
    return int(n.value)


def _ws_bytes(workspace) -> int:
    if workspace is None:
        return 0
    return workspace.numel() * workspace.element_size()


def group_decode_attn(kv, layout, q, softmax_scale, out, lse, workspace, stream=None) -> None:
    _check(load().rp_group_decode_attn(ctypes.byref(kv), ctypes.byref(layout), _ptr(q),
                                       float(softmax_scale), _ptr(out), _ptr(lse), _ptr(workspace),
                                       _ws_bytes(workspace), _stream(stream)),
           "rp_group_decode_attn")


def group_decode_attn_noalloc(kv, layout, q, softmax_scale, out, lse, stream=None) -> None:
    """rp_group_decode_attn on the library's static scratch (no workspace, nothing allocated)."""
    _check(load().rp_group_decode_attn_noalloc(ctypes.byref(kv), ctypes.byref(layout), _ptr(q),
                                               float(softmax_scale), _ptr(out), _ptr(lse), _stream(stream)),
           "rp_group_decode_attn_noalloc")


def plan(kv, layout, workspace, stream=None) -> None:
    _check(load().rp_plan(ctypes.byref(kv), ctypes.byref(layout), _ptr(workspace),
                          _ws_bytes(workspace), _stream(stream)), "rp_plan")


def attn_parts(kv, layout, q, softmax_scale, workspace, stream=None) -> None:
    _check(load().rp_attn_parts(ctypes.byref(kv), ctypes.byref(layout), _ptr(q), float(softmax_scale),
                                _ptr(workspace), _ws_bytes(workspace), _stream(stream)),
           "rp_attn_parts")


def combine_parts(kv, layout, out, lse, workspace, stream=None) -> None:
    _check(load().rp_combine_parts(ctypes.byref(kv), ctypes.byref(layout), _ptr(out), _ptr(lse),
                                   _ptr(workspace), _ws_bytes(workspace), _stream(stream)),
           "rp_combine_parts")


def selftest_mfma(shape, a, b, c, stream=None) -> None:
    """One MFMA in the kernels' lane layouts: c (fp32 [M][N]) = a (bf16 [M][K]) b (bf16 [K][N]).

    shape: a key of RP_SELFTEST_SHAPES or its integer code."""
    code = RP_SELFTEST_SHAPES[shape][0] if isinstance(shape, str) else int(shape)
    _check(load().rp_selftest_mfma(code, _ptr(a), _ptr(b), _ptr(c), _stream(stream)), "rp_selftest_mfma")


def stream_read(src, nbytes, sink, nontemporal=False, stream=None) -> None:
    """Read nbytes of device tensor src once (16-byte loads); sink: int32/uint32 [RP_STREAM_READ_SINK_WORDS]."""
    _check(load().rp_stream_read(_ptr(src), int(nbytes), _ptr(sink), int(bool(nontemporal)), _stream(stream)),
           "rp_stream_read")


def lse_combine(o_parts, lse_parts, row_part_offsets, num_rows, head_dim, out, lse_out,
                stream=None) -> None:
    _check(load().rp_lse_combine(_ptr(o_parts), _ptr(lse_parts), _ptr(row_part_offsets),
                                 int(num_rows), int(head_dim), _ptr(out), _ptr(lse_out),
                                 _stream(stream)), "rp_lse_combine")


def plan_layout(kv, layout) -> RpPlanInfo:
    info = RpPlanInfo()
    _check(load().rp_plan_layout(ctypes.byref(kv), ctypes.byref(layout), ctypes.byref(info)), "rp_plan_layout")
    return info


def validate_layout(kv, layout, stream=None) -> None:
    _check(load().rp_validate_layout(ctypes.byref(kv), ctypes.byref(layout), _stream(stream)),
           "rp_validate_layout")


def _tensors(*specs) -> None:
    """Refuse tensors that the library would read as others: (name, tensor, dtype, shape), with None for what may
    be any. Raw addresses (int) and None pass; every tensor is on the current device."""
    device = None
    for name, t, dtype, shape in specs:
        if t is None or isinstance(t, int):
            continue
        if dtype is not None and t.dtype is not dtype:
            raise ValueError(f"{name}: dtype {t.dtype}, not {dtype}")
        if shape is not None and t.shape != shape and (t.dim() != len(shape) or any(w not in (None, g) for g, w in zip(t.shape, shape))):
            raise ValueError(f"{name}: shape {tuple(t.shape)}, not {shape}")
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous (strides {t.stride()})")
        if device is None and t.is_cuda:
            device = torch.cuda.current_device()
        if not t.is_cuda or t.get_device() != device:
            raise ValueError(f"{name} is on {t.device}, not on the current GPU")


def draft_tree(draft_offs, masks, *, max_drafts, num_drafts=None) -> RpDraftTree:
    """Describe packed trees: sequence s has the drafts draft_offs[s] .. draft_offs[s+1]-1 (int32 [S + 1]),
    masks (int64 or uint64 [T]) say which drafts of its sequence each one sees, bit u for the u-th. Offsets of more
    sequences than a layout's may be used with it."""
    _tensors(("draft_offs", draft_offs, torch.int32, (None,)),
             ("masks", masks, torch.uint64 if getattr(masks, "dtype", None) is torch.uint64 else torch.int64, (None,)))
    T = int(masks.shape[0]) if num_drafts is None else int(num_drafts)
    if not isinstance(masks, int) and T > masks.shape[0]:
        raise ValueError(f"num_drafts {T}, but masks has {masks.shape[0]} entries")
    tree = _holding(RpDraftTree(T, int(max_drafts), _ptr(draft_offs), _ptr(masks)), draft_offs, masks)
    tree.offsets = None if isinstance(draft_offs, int) else int(draft_offs.shape[0])
    return tree


def _fits(layout, tree) -> None:
    """Refuse offsets of fewer sequences than the layout's: the kernels read layout.num_seqs + 1 of them."""
    n = getattr(tree, "offsets", None)
    if n is not None and n < layout.num_seqs + 1:
        raise ValueError(f"draft_offs has {n} entries, {layout.num_seqs} sequences need {layout.num_seqs + 1}")


def group_tree_attn_workspace_size(kv, layout, tree) -> int:
    _fits(layout, tree)
    n = ctypes.c_size_t(0)
    _check(load().rp_group_tree_attn_workspace_size(ctypes.byref(kv), ctypes.byref(layout), ctypes.byref(tree),
                                                    ctypes.byref(n)), "rp_group_tree_attn_workspace_size")
    return int(n.value)


def group_tree_attn(kv, layout, tree, q, k_draft, v_draft, softmax_scale, out, lse, workspace, stream=None) -> None:
    """Attention of every drafted token over the cache and its tree: q, out bf16 [T][Hq][d], k_draft, v_draft
    bf16 [T][Hkv][d], lse fp32 [T][Hq] or None, workspace uint8 (None where its size is 0)."""
    _fits(layout, tree)
    T, hq, hkv, d = tree.num_drafts, layout.num_q_heads, kv.num_kv_heads, kv.head_dim
    bf16 = torch.bfloat16
    _tensors(("q", q, bf16, (T, hq, d)), ("k_draft", k_draft, bf16, (T, hkv, d)), ("v_draft", v_draft, bf16, (T, hkv, d)),
             ("out", out, bf16, (T, hq, d)), ("lse", lse, torch.float32, (T, hq)), ("workspace", workspace, None, None))
    _check(load().rp_group_tree_attn(ctypes.byref(kv), ctypes.byref(layout), ctypes.byref(tree), _ptr(q),
                                     _ptr(k_draft), _ptr(v_draft), float(softmax_scale), _ptr(out), _ptr(lse),
                                     _ptr(workspace), _ws_bytes(workspace), _stream(stream)), "rp_group_tree_attn")


def page_tables(block_table, free_pages, free_count) -> RpPageTables:
    """Describe block tables (int32 [S][max_pages]) and their stack of free pages (int32 [num_pages], and its
    count, int32 [1])."""
    _tensors(("block_table", block_table, torch.int32, (None, None)), ("free_pages", free_pages, torch.int32, (None,)),
             ("free_count", free_count, torch.int32, (1,)))
    tables = RpPageTables(int(block_table.shape[0]), int(block_table.shape[1]), 16, int(free_pages.shape[0]),
                          _ptr(block_table), _ptr(free_pages), _ptr(free_count))
    return _holding(tables, block_table, free_pages, free_count)


def page_tables_resize(tables, old_lens, new_lens, status, slot_offs=None, slot_map=None, stream=None) -> None:
    """Grow and shrink sequences: int32 [S] lengths before and after; status int32 [4] on the device gets
    {RP_TABLES_*, pages taken, pages given back, new tokens}; slot_offs int32 [S + 1]; slot_map int32 [max_slots]."""
    S, i32 = tables.num_seqs, torch.int32
    _tensors(("old_lens", old_lens, i32, (S,)), ("new_lens", new_lens, i32, (S,)), ("status", status, i32, (4,)),
             ("slot_offs", slot_offs, i32, (S + 1,)), ("slot_map", slot_map, i32, (None,)))
    if slot_map is not None and slot_offs is None:
        raise RpError(RP_ERR_INVALID_ARG, "rp_page_tables_resize", "slot_map needs slot_offs")
    slots = 0 if slot_map is None else int(slot_map.shape[0])
    # An empty tensor has no address; the library then only counts against its size.
    where = (_ptr(slot_map) or _ptr(slot_offs)) if slot_map is not None else None
    _check(load().rp_page_tables_resize(ctypes.byref(tables), _ptr(old_lens), _ptr(new_lens), _ptr(status),
                                        _ptr(slot_offs), where, slots, _stream(stream)), "rp_page_tables_resize")


def kv_write_slots(kv, slot_map, k_new, v_new, src_rows=None, stream=None) -> None:
    """Write rows of k_new and v_new (bf16 [num_src][Hkv][d]) into the slots of slot_map (int32 [T]): row
    src_rows[i] (int32 [T]; row i where None) into slot_map[i]; negative slots are skipped. fp8: the entries of a
    page follow each other, fewer than 64 places apart, with rising slots."""
    T, rows = int(slot_map.shape[0]), int(k_new.shape[0])
    row = (rows, kv.num_kv_heads, kv.head_dim)
    _tensors(("slot_map", slot_map, torch.int32, (T,)), ("k_new", k_new, torch.bfloat16, row),
             ("v_new", v_new, torch.bfloat16, row), ("src_rows", src_rows, torch.int32, (T,)))
    _check(load().rp_kv_write_slots(ctypes.byref(kv), _ptr(slot_map), T, _ptr(k_new), _ptr(v_new), _ptr(src_rows),
                                    rows, _stream(stream)), "rp_kv_write_slots")


def prefill_layout(prompt_offs, prefix_block_table, *, num_q_heads, num_tokens) -> RpPrefillLayout:
    """Describe packed prompts: group g owns rows prompt_offs[g] .. prompt_offs[g+1]-1."""
    layout = RpPrefillLayout(int(prompt_offs.shape[0]) - 1, int(num_q_heads), int(num_tokens), _ptr(prompt_offs),
                             _ptr(prefix_block_table), int(prefix_block_table.shape[1]))
    return _holding(layout, prompt_offs, prefix_block_table)


def prefill_kv_write(kv, layout, k, v, stream=None) -> None:
    _check(load().rp_prefill_kv_write(ctypes.byref(kv), ctypes.byref(layout), _ptr(k), _ptr(v), _stream(stream)),
           "rp_prefill_kv_write")


def prefill_attn(kv, layout, q, k, v, softmax_scale, out, lse, stream=None) -> None:
    _check(load().rp_prefill_attn(ctypes.byref(kv), ctypes.byref(layout), _ptr(q), _ptr(k), _ptr(v),
                                  float(softmax_scale), _ptr(out), _ptr(lse), _stream(stream)), "rp_prefill_attn")


def prefill(kv, layout, q, k, v, softmax_scale, out, lse, stream=None) -> None:
    _check(load().rp_prefill(ctypes.byref(kv), ctypes.byref(layout), _ptr(q), _ptr(k), _ptr(v),
                             float(softmax_scale), _ptr(out), _ptr(lse), _stream(stream)), "rp_prefill")


def sched_simulate(*, mode, group_size, update_groups, prompt_lens, resp_lens, max_running, frontier_width=0,
                   step_base=0.0, step_per_seq=0.0, step_per_ctx_token=0.0, prefill_per_token=0.0,
                   mat_base=0.0, mat_per_token=0.0, train_base=0.0, train_per_token=0.0, opt_step=0.0) -> dict:
    """Run rp_sched_simulate on host arrays; returns the summary and the per-group timelines."""
    import numpy as np
    prompt = np.ascontiguousarray(prompt_lens, dtype=np.int32)
    resp = np.ascontiguousarray(resp_lens, dtype=np.int32)
    R = int(prompt.shape[0])
    U = max(int(update_groups), 1)
    cfg = RpSchedConfig(RP_SCHED_MODES[mode], R, int(group_size), int(update_groups), int(frontier_width),
                        int(max_running), step_base, step_per_seq, step_per_ctx_token, prefill_per_token,
                        mat_base, mat_per_token, train_base, train_per_token, opt_step)
    summ = RpSchedSummary()
    f64 = [np.zeros(R, np.float64) for _ in range(3)]
    fifo = np.zeros(R, np.int32)
    upd = [np.zeros(max(R // U, 1), np.float64) for _ in range(2)]
    dp = lambda a: a.ctypes.data_as(ctypes.c_void_p)
    _check(load().rp_sched_simulate(ctypes.byref(cfg), dp(prompt), dp(resp), ctypes.byref(summ), dp(f64[0]),
                                    dp(f64[1]), dp(f64[2]), dp(fifo), dp(upd[0]), dp(upd[1])),
           "rp_sched_simulate")
    out = {n: getattr(summ, n) for n, _ in RpSchedSummary._fields_}
    out.update(serve_done=f64[0].tolist(), frontier_enter=f64[1].tolist(), trainable=f64[2].tolist(),
               fifo=fifo.tolist(), update_start=upd[0][:R // U].tolist(), update_end=upd[1][:R // U].tolist())
    return out
