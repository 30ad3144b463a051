"""Thin ctypes binding of liblvspec.so: argument marshalling only.

Every step of the verify path runs inside the library's HIP kernels; torch supplies device
memory, the current stream and nothing else.  There is no CPU fallback: if the shared library
is missing, importing this module raises.
"""
from __future__ import annotations

import ctypes as C
import functools
import os
from typing import NamedTuple, Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "liblvspec.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(
        f"{LIB_PATH} not found: build it with `python -m paper_2604_05650_amd.build` "
        "(there is no fallback path)")

_lib = C.CDLL(LIB_PATH)

OK, EINVAL, EUNSUPPORTED, EWORKSPACE, EHIP, ESCRATCH = 0, -1, -2, -3, -4, -5
STATIC_SCRATCH_BYTES = 16 << 20
REJECT, EXACT, LOOSE, SHIFT, GATED = 0, 1, 2, 3, 4
RULE_VISUAL, RULE_ENTROPY_GATE, RULE_ENTROPY_WINDOW = 0, 1, 2
MAX_GAMMA, MAX_TOPK, MAX_TOPN = 16, 16, 1024
PAGE_TOKENS, TAIL_ROWS = 64, 128          # of the paged caches
SLOT_NONE, SLOT_TAIL = -1, -2
BF16, F16, F32 = 0, 1, 2                  # types of rotary rows
SCALING_NONE, SCALING_LINEAR, SCALING_NTK, SCALING_YARN = 0, 1, 2, 3


class AttnArgs(C.Structure):
    _fields_ = [
        ("B", C.c_int32), ("gamma", C.c_int32), ("Hq", C.c_int32), ("Hkv", C.c_int32),
        ("D", C.c_int32),
        ("q", C.c_void_p), ("q_sb", C.c_int64), ("q_sg", C.c_int64), ("q_sh", C.c_int64),
        ("k", C.c_void_p), ("v", C.c_void_p),
        ("kv_sb", C.c_int64), ("kv_sh", C.c_int64), ("kv_sl", C.c_int64),
        ("cap", C.c_int64),
        ("kv_len", C.c_void_p), ("kv_len_host", C.POINTER(C.c_int32)), ("max_kv_len", C.c_int64),
        ("vis_begin", C.c_void_p), ("vis_end", C.c_void_p),
        ("draft_mask", C.POINTER(C.c_uint32)),
        ("scale", C.c_float),
        ("out", C.c_void_p), ("o_sb", C.c_int64), ("o_sg", C.c_int64), ("o_sh", C.c_int64),
        ("lse", C.c_void_p), ("vis_mass", C.c_void_p),
        ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t),
    ]


class RelArgs(C.Structure):
    _fields_ = [
        ("B", C.c_int32), ("gamma", C.c_int32), ("d", C.c_int32), ("top_n", C.c_int32),
        ("h_d", C.c_void_p), ("hd_sb", C.c_int64), ("hd_sg", C.c_int64),
        ("h_v", C.c_void_p), ("hv_sb", C.c_int64), ("hv_sl", C.c_int64),
        ("lv_max", C.c_int64),
        ("l_v", C.c_void_p),
        ("hv_inv_norm", C.c_void_p),
        ("relevance", C.c_void_p),
        ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t),
    ]


class HvArgs(C.Structure):
    _fields_ = [
        ("B", C.c_int32), ("d", C.c_int32),
        ("h_v", C.c_void_p), ("hv_sb", C.c_int64), ("hv_sl", C.c_int64),
        ("lv_max", C.c_int64),
        ("hv_inv_norm", C.c_void_p),
    ]


class AcceptArgs(C.Structure):
    _fields_ = [
        ("B", C.c_int32), ("gamma", C.c_int32), ("d", C.c_int32), ("V", C.c_int32),
        ("topk", C.c_int32),
        ("h_d", C.c_void_p), ("hd_sb", C.c_int64), ("hd_sg", C.c_int64),
        ("lm_head", C.c_void_p), ("w_sv", C.c_int64),
        ("draft_ids", C.c_void_p), ("relevance", C.c_void_p),
        ("n_loose", C.c_int32), ("pst_window", C.c_int32), ("loose_topk_gate", C.c_int32),
        ("n_branches", C.c_int32),
        ("bonus_row", C.c_int32),
        ("rule", C.c_int32), ("entropy_threshold", C.c_float), ("defer_window", C.c_int32),
        ("target_ids", C.c_void_p), ("topk_ids", C.c_void_p), ("topk_probs", C.c_void_p),
        ("verdict", C.c_void_p), ("accept_len", C.c_void_p), ("bonus_id", C.c_void_p),
        ("best_branch", C.c_void_p),
        ("logits", C.c_void_p), ("entropy", C.c_void_p),
        ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t),
    ]


class CommitArgs(C.Structure):
    _fields_ = [
        ("B", C.c_int32), ("Hkv", C.c_int32), ("D", C.c_int32), ("n_layers", C.c_int32),
        ("n_branches", C.c_int32), ("chain_len", C.c_int32),
        ("k", C.c_void_p), ("v", C.c_void_p),
        ("kv_slayer", C.c_int64), ("kv_sb", C.c_int64), ("kv_sh", C.c_int64), ("kv_sl", C.c_int64),
        ("cap", C.c_int64),
        ("kv_len", C.c_void_p), ("accept_len", C.c_void_p), ("best_branch", C.c_void_p),
        ("new_len", C.c_void_p),
    ]


class PagedCacheStruct(C.Structure):
    _fields_ = [
        ("B", C.c_int32), ("Hkv", C.c_int32), ("D", C.c_int32), ("n_blocks", C.c_int32),
        ("k_pool", C.c_void_p), ("v_pool", C.c_void_p),
        ("k_scale", C.c_void_p), ("v_scale", C.c_void_p),
        ("k_tail", C.c_void_p), ("v_tail", C.c_void_p),
    ]


class PagedPlanArgs(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("B", "table_cols", "n_blocks", "max_rows", "reserve", "draft")] + [
        (n, C.c_void_p) for n in ("kv_len", "n_new", "held", "state", "queue", "table", "granted", "new_held",
                                  "new_state", "cu_rows", "slots", "row_seq", "row_pos")]


class PagedAppendArgs(C.Structure):
    _fields_ = [
        ("cache", PagedCacheStruct), ("n_rows", C.c_int32),
        ("k", C.c_void_p), ("v", C.c_void_p),
        ("k_sr", C.c_int64), ("k_sh", C.c_int64), ("v_sr", C.c_int64), ("v_sh", C.c_int64),
        ("slots", C.c_void_p), ("row_seq", C.c_void_p), ("row_pos", C.c_void_p), ("cu_rows", C.c_void_p),
    ]


class PagedAttnArgs(C.Structure):
    _fields_ = [
        ("cache", PagedCacheStruct), ("gamma", C.c_int32), ("Hq", C.c_int32),
        ("q", C.c_void_p), ("q_sb", C.c_int64), ("q_sg", C.c_int64), ("q_sh", C.c_int64),
        ("table", C.c_void_p), ("table_cols", C.c_int32), ("kv_len", C.c_void_p),
        ("vis_begin", C.c_void_p), ("vis_end", C.c_void_p),
        ("draft_mask", C.POINTER(C.c_uint32)),
        ("scale", C.c_float),
        ("out", C.c_void_p), ("o_sb", C.c_int64), ("o_sg", C.c_int64), ("o_sh", C.c_int64),
        ("lse", C.c_void_p), ("vis_mass", C.c_void_p),
        ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t),
    ]


class PagedCommitArgs(C.Structure):
    _fields_ = [
        ("cache", PagedCacheStruct), ("n_layers", C.c_int32),
        ("n_branches", C.c_int32), ("chain_len", C.c_int32),
        ("table", C.c_void_p), ("table_cols", C.c_int32),
        ("kv_len", C.c_void_p), ("accept_len", C.c_void_p), ("best_branch", C.c_void_p),
        ("new_len", C.c_void_p),
        ("granted", C.c_void_p), ("held", C.c_void_p), ("cu_rows", C.c_void_p),
    ]


class Rotation(C.Structure):
    _fields_ = [
        ("dim", C.c_int32), ("interleaved", C.c_int32), ("transpose", C.c_int32), ("n_axes", C.c_int32),
        ("inv_freq", C.c_void_p), ("axis", C.c_void_p), ("pos", C.c_void_p), ("pos_sa", C.c_int64),
        ("factor", C.c_float),
    ]


class RotaryArgs(C.Structure):
    _fields_ = [
        ("rot", Rotation),
        ("n_rows", C.c_int32), ("Hq", C.c_int32), ("Hkv", C.c_int32), ("D", C.c_int32), ("dtype", C.c_int32),
        ("q", C.c_void_p), ("q_sr", C.c_int64), ("q_sh", C.c_int64),
        ("q_out", C.c_void_p), ("qo_sr", C.c_int64), ("qo_sh", C.c_int64),
        ("k", C.c_void_p), ("k_sr", C.c_int64), ("k_sh", C.c_int64),
        ("k_out", C.c_void_p), ("ko_sr", C.c_int64), ("ko_sh", C.c_int64),
    ]


class RotaryFreqArgs(C.Structure):
    _fields_ = [("dim", C.c_int32), ("scaling", C.c_int32)] + [
        (n, C.c_double) for n in ("base", "scale", "original_len", "beta_fast", "beta_slow")]


_ROTATED_QUERIES = [
    ("rot", Rotation), ("Hq", C.c_int32),
    ("q", C.c_void_p), ("q_sr", C.c_int64), ("q_sh", C.c_int64),
    ("q_out", C.c_void_p), ("qo_sr", C.c_int64), ("qo_sh", C.c_int64),
]


class PagedAppendRotaryArgs(C.Structure):
    _fields_ = [("rows", PagedAppendArgs)] + _ROTATED_QUERIES


class PagedMxCacheStruct(C.Structure):
    _fields_ = PagedCacheStruct._fields_


class PagedMxAppendArgs(C.Structure):
    _fields_ = [("cache", PagedMxCacheStruct)] + PagedAppendArgs._fields_[1:] + _ROTATED_QUERIES


class PagedMxReadArgs(C.Structure):
    _fields_ = [
        ("cache", PagedMxCacheStruct), ("n_rows", C.c_int32), ("slots", C.c_void_p),
        ("k", C.c_void_p), ("v", C.c_void_p),
        ("k_sr", C.c_int64), ("k_sh", C.c_int64), ("v_sr", C.c_int64), ("v_sh", C.c_int64),
    ]


class PagedMxAttnArgs(C.Structure):
    _fields_ = [("cache", PagedMxCacheStruct)] + PagedAttnArgs._fields_[1:]


class PagedMxCommitArgs(C.Structure):
    _fields_ = [("cache", PagedMxCacheStruct)] + PagedCommitArgs._fields_[1:]


class PlanInfo(C.Structure):
    _fields_ = [(n, C.c_int32) for n in (
        "attn_rows_padded", "attn_row_chunks", "attn_splits", "rel_splits", "rel_stage_bytes",
        "rel_slices", "rel_slice_rows", "acc_rows_per_task", "acc_chains_per_pass", "acc_passes")]


_lib.lvspec_status_string.restype = C.c_char_p
_lib.lvspec_status_string.argtypes = [C.c_int]
_lib.lvspec_version.restype = C.c_int
_lib.lvspec_last_hip_error.restype = C.c_int
_lib.lvspec_n_loose.restype = C.c_int
_lib.lvspec_n_loose.argtypes = [C.c_float, C.c_int]
_lib.lvspec_describe_plan.restype = C.c_int
_lib.lvspec_describe_plan.argtypes = [C.POINTER(AttnArgs), C.POINTER(RelArgs),
                                      C.POINTER(AcceptArgs), C.POINTER(PlanInfo)]
_lib.lvspec_kv_commit.restype = C.c_int
_lib.lvspec_kv_commit.argtypes = [C.POINTER(CommitArgs), C.c_void_p]
for _name, _t in (("verify_attn", AttnArgs), ("visual_relevance", RelArgs),
                  ("loose_accept", AcceptArgs)):
    getattr(_lib, f"lvspec_{_name}_workspace").restype = C.c_size_t
    getattr(_lib, f"lvspec_{_name}_workspace").argtypes = [C.POINTER(_t)]
    getattr(_lib, f"lvspec_{_name}").restype = C.c_int
    getattr(_lib, f"lvspec_{_name}").argtypes = [C.POINTER(_t), C.c_void_p]

_lib.lvspec_hv_prepare.restype = C.c_int
_lib.lvspec_hv_prepare.argtypes = [C.POINTER(HvArgs), C.c_void_p]
_lib.lvspec_verify_attn_static.restype = C.c_int
_lib.lvspec_verify_attn_static.argtypes = [C.POINTER(AttnArgs), C.c_void_p]

for _name, _t in (("paged_plan", PagedPlanArgs), ("paged_append", PagedAppendArgs),
                  ("verify_attn_paged", PagedAttnArgs), ("paged_commit", PagedCommitArgs)):
    getattr(_lib, f"lvspec_{_name}").restype = C.c_int
    getattr(_lib, f"lvspec_{_name}").argtypes = [C.POINTER(_t), C.c_void_p]
_lib.lvspec_verify_attn_paged_workspace.restype = C.c_size_t
_lib.lvspec_verify_attn_paged_workspace.argtypes = [C.POINTER(PagedAttnArgs)]

for _name, _t in (("rotary", RotaryArgs), ("paged_append_rotary", PagedAppendRotaryArgs),
                  ("paged_mx_append", PagedMxAppendArgs), ("paged_mx_read", PagedMxReadArgs),
                  ("verify_attn_paged_mx", PagedMxAttnArgs), ("paged_mx_commit", PagedMxCommitArgs)):
    getattr(_lib, f"lvspec_{_name}").restype = C.c_int
    getattr(_lib, f"lvspec_{_name}").argtypes = [C.POINTER(_t), C.c_void_p]
_lib.lvspec_verify_attn_paged_mx_workspace.restype = C.c_size_t
_lib.lvspec_verify_attn_paged_mx_workspace.argtypes = [C.POINTER(PagedMxAttnArgs)]
_lib.lvspec_rotary_frequencies.restype = C.c_int
_lib.lvspec_rotary_frequencies.argtypes = [C.POINTER(RotaryFreqArgs), C.POINTER(C.c_float), C.POINTER(C.c_float)]

EXPORTS = ["lvspec_hv_prepare", "lvspec_verify_attn_static", "lvspec_status_string", "lvspec_version", "lvspec_last_hip_error", "lvspec_n_loose",
           "lvspec_verify_attn_workspace", "lvspec_verify_attn",
           "lvspec_visual_relevance_workspace", "lvspec_visual_relevance",
           "lvspec_loose_accept_workspace", "lvspec_loose_accept", "lvspec_kv_commit",
           "lvspec_describe_plan", "lvspec_paged_plan", "lvspec_paged_append",
           "lvspec_verify_attn_paged_workspace", "lvspec_verify_attn_paged", "lvspec_paged_commit",
           "lvspec_rotary", "lvspec_rotary_frequencies", "lvspec_paged_append_rotary",
           "lvspec_paged_mx_append", "lvspec_paged_mx_read", "lvspec_verify_attn_paged_mx_workspace",
           "lvspec_verify_attn_paged_mx", "lvspec_paged_mx_commit"]


class LvspecError(RuntimeError):
    def __init__(self, status: int):
        self.status = status
        msg = _lib.lvspec_status_string(status).decode()
        if status == EHIP:
            msg += f" (hipError_t {_lib.lvspec_last_hip_error()})"
        super().__init__(f"lvspec status {status}: {msg}")


def raw():
    """The ctypes library handle (tests of the C ABI call it directly)."""
    return _lib


def version() -> int:
    return int(_lib.lvspec_version())


def status_string(status: int) -> str:
    return _lib.lvspec_status_string(status).decode()


def n_loose(lam: float, gamma: int) -> int:
    return int(_lib.lvspec_n_loose(float(lam), int(gamma)))


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _stream(stream) -> Optional[int]:
    if stream is None:
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _check(status: int):
    if status != OK:
        raise LvspecError(status)


def _tensors(x):
    """The tensors among arguments or results (tuples, dicts)."""
    if isinstance(x, torch.Tensor):
        yield x
    elif isinstance(x, (tuple, dict)):
        for y in (x.values() if isinstance(x, dict) else x):
            yield from _tensors(y)


def _allocates_on_stream(call):
    """For calls that allocate outputs or a workspace and take `stream`: they come from that stream's memory.
    Memory of the caller's stream may still be read by work before the call, and a workspace could be
    given out again, to a launch on a third stream, as soon as the call returns.  Results may be used (behind a
    wait) and dropped on the caller's stream."""
    @functools.wraps(call)
    def on_stream(*args, stream=None, **kwargs):
        if stream is None:
            return call(*args, **kwargs)
        device = next((t.device for t in _tensors((args, kwargs)) if t.is_cuda), None)
        if device is None:                     # (refused by the call)
            return call(*args, **kwargs)
        caller = torch.cuda.current_stream(device)
        handle = _stream(stream)
        if handle == caller.cuda_stream and device.index == torch.cuda.current_device():
            return call(*args, **kwargs)
        if handle in (0, 1):                   # (the default stream's two names)
            stream = torch.cuda.default_stream(device)
        elif not isinstance(stream, torch.cuda.Stream):
            stream = torch.cuda.ExternalStream(handle, device=device)
        with torch.cuda.stream(stream):
            result = call(*args, **kwargs)
        for t in _tensors(result):
            t.record_stream(caller)
        return result
    return on_stream


# What a call costs in the interpreter: new_empty of an input takes 3.6 us where torch.empty takes
# 4.5 (outputs and workspaces of the three verify calls), one stride() 0.4 us where one per dimension
# takes 1.5 (verify_attn_args), and an array assigned to a pointer field 0.7 us where ctypes.cast takes
# 6.4.  A smallest step of three calls from Python: 72 -> 67 us.  The other argument functions read
# a stride at a time, and kv_commit allocates with torch.empty.
def _workspace(nbytes: int, like: torch.Tensor, workspace: Optional[torch.Tensor]) -> torch.Tensor:
    if workspace is not None:
        return workspace
    return like.new_empty((max(int(nbytes), 256),), dtype=torch.uint8)


def verify_attn_args(q, k, v, kv_len, *, out, vis_begin=None, vis_end=None, draft_mask=None,
                     scale=0.0, lse=None, vis_mass=None, max_kv_len=0,
                     kv_len_host=None) -> AttnArgs:
    """Fill the C struct from torch tensors: q [B,gamma,Hq,D], k/v [B,Hkv,cap,D] (bf16, last dim
    contiguous), kv_len / vis_begin / vis_end int32 [B] on the device; kv_len_host an optional
    host sequence with the same lengths."""
    B, gamma, Hq, D = q.shape
    a = AttnArgs()
    k_shape = k.shape
    a.B, a.gamma, a.Hq, a.Hkv, a.D = B, gamma, Hq, k_shape[1], D
    a.q, (a.q_sb, a.q_sg, a.q_sh) = q.data_ptr(), q.stride()[:3]
    a.k, a.v = k.data_ptr(), v.data_ptr()
    a.kv_sb, a.kv_sh, a.kv_sl = k.stride()[:3]
    a.cap = k_shape[2]
    a.kv_len, a.max_kv_len = _ptr(kv_len), int(max_kv_len)
    if kv_len_host is not None:
        lens = (C.c_int32 * B)(*[int(x) for x in kv_len_host])
        a._keep_len = a.kv_len_host = lens
    a.vis_begin, a.vis_end = _ptr(vis_begin), _ptr(vis_end)
    if draft_mask is not None:
        arr = (C.c_uint32 * gamma)(*[int(m) for m in draft_mask])
        a._keep = a.draft_mask = arr
    a.scale = float(scale)
    a.out, (a.o_sb, a.o_sg, a.o_sh) = out.data_ptr(), out.stride()[:3]
    a.lse, a.vis_mass = _ptr(lse), _ptr(vis_mass)
    return a


@_allocates_on_stream
def verify_attn(q, k, v, kv_len, *, vis_begin=None, vis_end=None, draft_mask=None, scale=0.0,
                out=None, return_lse=False, return_vis_mass=False, workspace=None,
                max_kv_len=0, kv_len_host=None, stream=None):
    """lvspec_verify_attn.  Returns out, or (out, lse, vis_mass) when either extra is asked for
    (the one not asked for is None)."""
    assert q.dtype == torch.bfloat16 and k.dtype == torch.bfloat16 and v.dtype == torch.bfloat16
    assert q.stride(-1) == 1 and k.stride(-1) == 1 and v.stride(-1) == 1
    assert k.stride() == v.stride() and k.shape == v.shape
    B, gamma, Hq, D = q.shape
    if out is None:
        out = q.new_empty((B, gamma, Hq, D))
    lse = q.new_empty((B, Hq, gamma), dtype=torch.float32) if return_lse else None
    vm = q.new_empty((B, Hq, gamma), dtype=torch.float32) if return_vis_mass else None
    a = verify_attn_args(q, k, v, kv_len, out=out, vis_begin=vis_begin, vis_end=vis_end,
                         draft_mask=draft_mask, scale=scale, lse=lse, vis_mass=vm,
                         max_kv_len=max_kv_len, kv_len_host=kv_len_host)
    need = _lib.lvspec_verify_attn_workspace(C.byref(a))
    ws = _workspace(need, q, workspace)
    a.workspace, a.workspace_bytes = ws.data_ptr(), ws.numel() * ws.element_size()
    _check(_lib.lvspec_verify_attn(C.byref(a), _stream(stream)))
    if return_lse or return_vis_mass:
        return out, lse, vm
    return out


def verify_attn_static(q, k, v, kv_len, *, out, vis_begin=None, vis_end=None, draft_mask=None,
                       scale=0.0, lse=None, vis_mass=None, max_kv_len=0, kv_len_host=None,
                       stream=None):
    """lvspec_verify_attn_static: the same attention with the library's static scratch; every
    output tensor is the caller's, nothing is allocated here."""
    a = verify_attn_args(q, k, v, kv_len, out=out, vis_begin=vis_begin, vis_end=vis_end,
                         draft_mask=draft_mask, scale=scale, lse=lse, vis_mass=vis_mass,
                         max_kv_len=max_kv_len, kv_len_host=kv_len_host)
    _check(_lib.lvspec_verify_attn_static(C.byref(a), _stream(stream)))
    return out


@_allocates_on_stream
def hv_prepare(h_v, *, hv_inv_norm=None, stream=None):
    """lvspec_hv_prepare: h_v [B,lv_max,d] bf16 -> fp32 [B,lv_max] inverse row norms (once, at
    prefill), to be handed to visual_relevance at every step."""
    assert h_v.dtype == torch.bfloat16 and h_v.stride(-1) == 1
    B, lv_max, d = h_v.shape
    if hv_inv_norm is None:
        hv_inv_norm = h_v.new_empty((B, lv_max), dtype=torch.float32)
    assert hv_inv_norm.is_contiguous() and hv_inv_norm.shape == (B, lv_max)
    a = HvArgs()
    a.B, a.d = B, d
    a.h_v, a.hv_sb, a.hv_sl = h_v.data_ptr(), h_v.stride(0), h_v.stride(1)
    a.lv_max = lv_max
    a.hv_inv_norm = hv_inv_norm.data_ptr()
    _check(_lib.lvspec_hv_prepare(C.byref(a), _stream(stream)))
    return hv_inv_norm


def visual_relevance_args(h_d, h_v, l_v, top_n, *, relevance, hv_inv_norm=None) -> RelArgs:
    B, gamma, d = h_d.shape
    a = RelArgs()
    a.B, a.gamma, a.d, a.top_n = B, gamma, d, int(top_n)
    a.h_d, a.hd_sb, a.hd_sg = h_d.data_ptr(), h_d.stride(0), h_d.stride(1)
    a.h_v, a.hv_sb, a.hv_sl = h_v.data_ptr(), h_v.stride(0), h_v.stride(1)
    a.lv_max = h_v.shape[1]
    a.l_v = l_v.data_ptr()
    if hv_inv_norm is not None:
        assert hv_inv_norm.dtype == torch.float32 and hv_inv_norm.is_contiguous()
        assert hv_inv_norm.shape == (B, h_v.shape[1])
        a.hv_inv_norm = hv_inv_norm.data_ptr()
    a.relevance = relevance.data_ptr()
    return a


@_allocates_on_stream
def visual_relevance(h_d, h_v, l_v, top_n=10, *, relevance=None, workspace=None, stream=None,
                     hv_inv_norm=None):
    """lvspec_visual_relevance.  h_d [B,gamma,d], h_v [B,lv_max,d] bf16; l_v int32 [B] (device);
    hv_inv_norm optional fp32 [B,lv_max] from hv_prepare.  Returns fp32 [B,gamma]."""
    assert h_d.dtype == torch.bfloat16 and h_v.dtype == torch.bfloat16
    assert h_d.stride(-1) == 1 and h_v.stride(-1) == 1
    B, gamma, d = h_d.shape
    if relevance is None:
        relevance = h_d.new_empty((B, gamma), dtype=torch.float32)
    a = visual_relevance_args(h_d, h_v, l_v, top_n, relevance=relevance, hv_inv_norm=hv_inv_norm)
    need = _lib.lvspec_visual_relevance_workspace(C.byref(a))
    ws = _workspace(need, h_d, workspace)
    a.workspace, a.workspace_bytes = ws.data_ptr(), ws.numel() * ws.element_size()
    _check(_lib.lvspec_visual_relevance(C.byref(a), _stream(stream)))
    return relevance


def loose_accept_args(h_d, lm_head, draft_ids, relevance, n_loose_, pst_window, *, topk,
                      loose_topk_gate, outs, n_branches=1, bonus_row=False, rule=RULE_VISUAL,
                      entropy_threshold=0.0, defer_window=0) -> AcceptArgs:
    B, rows, d = h_d.shape
    gamma = rows - 1 if bonus_row else rows
    a = AcceptArgs()
    a.B, a.gamma, a.d, a.V, a.topk = B, gamma, d, lm_head.shape[0], int(topk)
    a.h_d, a.hd_sb, a.hd_sg = h_d.data_ptr(), h_d.stride(0), h_d.stride(1)
    a.lm_head, a.w_sv = lm_head.data_ptr(), lm_head.stride(0)
    a.draft_ids, a.relevance = draft_ids.data_ptr(), _ptr(relevance)
    a.rule, a.entropy_threshold, a.defer_window = int(rule), float(entropy_threshold), int(defer_window)
    a.n_loose, a.pst_window, a.loose_topk_gate = int(n_loose_), int(pst_window), int(loose_topk_gate)
    a.target_ids = outs["target_ids"].data_ptr()
    a.topk_ids, a.topk_probs = _ptr(outs.get("topk_ids")), _ptr(outs.get("topk_probs"))
    a.verdict = outs["verdict"].data_ptr()
    a.accept_len = outs["accept_len"].data_ptr()
    a.bonus_id = outs["bonus_id"].data_ptr()
    a.n_branches = int(n_branches)
    a.bonus_row = 1 if bonus_row else 0
    a.best_branch = _ptr(outs.get("best_branch"))
    a.logits = _ptr(outs.get("logits"))
    a.entropy = _ptr(outs.get("entropy"))
    return a


def alloc_accept_outputs(B, gamma, V, topk, device, return_logits=False, return_topk=True,
                         n_branches=1, return_entropy=False, bonus_row=False):
    return _accept_outputs(torch.empty((0,), dtype=torch.int32, device=device), B, gamma, V, topk,
                           return_logits, return_topk, n_branches, return_entropy, bonus_row)


def _accept_outputs(like, B, gamma, V, topk, return_logits, return_topk, n_branches,
                    return_entropy, bonus_row):
    """The outputs of loose_accept on the device of `like`."""
    rows = gamma + (1 if bonus_row else 0)   # hidden rows per chain
    new = like.new_empty
    outs = dict(
        target_ids=new((B, rows), dtype=torch.int32),
        verdict=new((B, gamma), dtype=torch.uint8),
        accept_len=new((B,), dtype=torch.int32),
        bonus_id=new((B,), dtype=torch.int32))
    if return_topk:
        outs["topk_ids"] = new((B, rows, topk), dtype=torch.int32)
        outs["topk_probs"] = new((B, rows, topk), dtype=torch.float32)
    if return_logits:
        outs["logits"] = new((B, rows, V), dtype=torch.float32)
    if n_branches > 1:
        outs["best_branch"] = new((B // n_branches,), dtype=torch.int32)
    if return_entropy:
        outs["entropy"] = new((B, rows), dtype=torch.float32)
    return outs


@_allocates_on_stream
def loose_accept(h_d, lm_head, draft_ids, relevance, n_loose_, pst_window, *, topk=1,
                 loose_topk_gate=0, return_logits=False, outs=None, workspace=None, stream=None,
                 n_branches=1, return_entropy=False, bonus_row=False, rule=RULE_VISUAL,
                 entropy_threshold=0.0, defer_window=0):
    """lvspec_loose_accept.  h_d [B,gamma,d] bf16 ([B,gamma+1,d] with bonus_row), lm_head [V,d]
    bf16, draft_ids int32 [B,gamma], relevance fp32 [B,gamma] (all on the device); B counts
    chains, n_branches of them per sequence.  Returns a dict of device tensors: target_ids,
    topk_ids, topk_probs, verdict, accept_len, bonus_id (+ logits, + best_branch when
    n_branches > 1, + entropy)."""
    assert h_d.dtype == torch.bfloat16 and lm_head.dtype == torch.bfloat16
    assert draft_ids.dtype == torch.int32
    assert relevance is None or relevance.dtype == torch.float32
    assert h_d.stride(-1) == 1 and lm_head.stride(-1) == 1
    assert draft_ids.is_contiguous() and (relevance is None or relevance.is_contiguous())
    B, rows, d = h_d.shape
    gamma = rows - 1 if bonus_row else rows
    assert draft_ids.shape == (B, gamma) and (relevance is None or relevance.shape == (B, gamma))
    if outs is None:
        outs = _accept_outputs(h_d, B, gamma, lm_head.shape[0], topk, return_logits, True,
                               n_branches, return_entropy, bonus_row)
    a = loose_accept_args(h_d, lm_head, draft_ids, relevance, n_loose_, pst_window, topk=topk,
                          loose_topk_gate=loose_topk_gate, outs=outs, n_branches=n_branches,
                          bonus_row=bonus_row, rule=rule, entropy_threshold=entropy_threshold,
                          defer_window=defer_window)
    need = _lib.lvspec_loose_accept_workspace(C.byref(a))
    ws = _workspace(need, h_d, workspace)
    a.workspace, a.workspace_bytes = ws.data_ptr(), ws.numel() * ws.element_size()
    _check(_lib.lvspec_loose_accept(C.byref(a), _stream(stream)))
    return outs


@_allocates_on_stream
def kv_commit(k, v, kv_len, accept_len, chain_len, *, best_branch=None, n_branches=1, new_len=None,
              stream=None):
    """lvspec_kv_commit.  k, v bf16 [B,Hkv,cap,D] or [layers,B,Hkv,cap,D] (changed in place),
    kv_len int32 [B], accept_len int32 [B*n_branches], best_branch int32 [B] (trees).
    Returns new_len int32 [B]."""
    assert k.dtype == torch.bfloat16 and v.dtype == torch.bfloat16 and k.shape == v.shape
    assert k.stride() == v.stride() and k.stride(-1) == 1
    if k.dim() == 4:
        k, v = k.unsqueeze(0), v.unsqueeze(0)
    layers, B, Hkv, cap, D = k.shape
    assert kv_len.dtype == torch.int32 and accept_len.dtype == torch.int32
    if new_len is None:
        new_len = torch.empty((B,), dtype=torch.int32, device=k.device)
    a = CommitArgs()
    a.B, a.Hkv, a.D, a.n_layers = B, Hkv, D, layers
    a.n_branches, a.chain_len = int(n_branches), int(chain_len)
    a.k, a.v = k.data_ptr(), v.data_ptr()
    a.kv_slayer, a.kv_sb, a.kv_sh, a.kv_sl = k.stride(0), k.stride(1), k.stride(2), k.stride(3)
    a.cap = cap
    a.kv_len, a.accept_len = kv_len.data_ptr(), accept_len.data_ptr()
    a.best_branch = _ptr(best_branch)
    a.new_len = new_len.data_ptr()
    _check(_lib.lvspec_kv_commit(C.byref(a), _stream(stream)))
    return new_len


def describe_plan(attn: Optional[AttnArgs] = None, rel: Optional[RelArgs] = None,
                  accept: Optional[AcceptArgs] = None) -> dict:
    """lvspec_describe_plan: the launch planning for the given argument structures (shape fields and
    the attention's workspace_bytes are read).  Returns the fields of the structures that were given."""
    info = PlanInfo()
    _check(_lib.lvspec_describe_plan(C.byref(attn) if attn is not None else None,
                                     C.byref(rel) if rel is not None else None,
                                     C.byref(accept) if accept is not None else None,
                                     C.byref(info)))
    out = {}
    for name, _ in PlanInfo._fields_:
        if ((name.startswith("attn_") and attn is not None) or
                (name.startswith("rel_") and rel is not None) or
                (name.startswith("acc_") and accept is not None)):
            out[name] = int(getattr(info, name))
    return out


# ------------------------------------------------------------------ paged cache in 8 bits
class PagedCache(NamedTuple):
    """The arrays of one layer, or of several with a leading dimension (include/lvspec.h says what
    they hold).  Pools: float8_e4m3fn or uint8."""
    k_pool: torch.Tensor      # [n_blocks, Hkv, 64, 128]
    v_pool: torch.Tensor      # [n_blocks, Hkv, 128, 64]
    k_scale: torch.Tensor     # fp32 [n_blocks, Hkv]
    v_scale: torch.Tensor
    k_tail: torch.Tensor      # bf16 [B, Hkv, 128, 128]
    v_tail: torch.Tensor

    def layer(self, i: int) -> "PagedCache":
        return PagedCache(*[x[i] for x in self])


def alloc_paged_cache(B, Hkv, n_blocks, device, layers: Optional[int] = None) -> PagedCache:
    lead = () if layers is None else (layers,)

    def new(shape, dtype):
        return torch.zeros(lead + shape, dtype=dtype, device=device)

    return PagedCache(
        new((n_blocks, Hkv, PAGE_TOKENS, 128), torch.float8_e4m3fn),
        new((n_blocks, Hkv, 128, PAGE_TOKENS), torch.float8_e4m3fn),
        new((n_blocks, Hkv), torch.float32), new((n_blocks, Hkv), torch.float32),
        new((B, Hkv, TAIL_ROWS, 128), torch.bfloat16), new((B, Hkv, TAIL_ROWS, 128), torch.bfloat16))


def alloc_paged_state(B, n_blocks, table_cols, device) -> dict:
    """What the plan of a batch starts from: every block free, nobody holds one."""
    def new(*shape):
        return torch.zeros(shape, dtype=torch.int32, device=device)

    state = new(2)
    state[1] = n_blocks
    return dict(held=new(B), state=state, queue=torch.arange(n_blocks, dtype=torch.int32, device=device),
                table=new(B, table_cols) - 1)


def alloc_paged_plan(B, max_rows, device) -> dict:
    """The outputs of paged_plan."""
    shapes = dict(granted=B, new_held=B, new_state=2, cu_rows=B + 1, slots=max_rows, row_seq=max_rows,
                  row_pos=max_rows)
    return {k: torch.empty((n,), dtype=torch.int32, device=device) for k, n in shapes.items()}


def _dense(t, dtype, shape, *also):
    assert t.is_cuda and t.dtype in (dtype, *also) and t.is_contiguous() and tuple(t.shape) == tuple(shape), (
        t.device, t.dtype, tuple(t.shape))
    return t.data_ptr()


def _one_device(*tensors):
    """The kernels of a call read all of its tensors from one device."""
    devices = {t.device for t in tensors if t is not None}
    assert len(devices) == 1, devices


def _call_on(device, fn, a, stream):
    """The call with the tensors' device current, which need not be the caller's."""
    if device.index == torch.cuda.current_device():
        _check(fn(C.byref(a), _stream(stream)))
    else:
        with torch.cuda.device(device):
            _check(fn(C.byref(a), _stream(stream)))


def _strides(t):
    """Strides of all but the last dimension.  torch gives any stride to a dimension of one: a row's."""
    return [s if n > 1 else 128 for n, s in zip(t.shape[:-1], t.stride())]


def _strides(t):
    """Strides of all but the last dimension.  torch gives any stride to a dimension of one: a row's."""
    return [s if n > 1 else 128 for n, s in zip(t.shape[:-1], t.stride())]


def _cache_struct(cache: PagedCache, lead=()) -> PagedCacheStruct:
    n = len(lead)
    n_blocks, Hkv = cache.k_pool.shape[n:n + 2]
    B = cache.k_tail.shape[n]
    f8, bf = torch.float8_e4m3fn, torch.bfloat16
    s = PagedCacheStruct()
    s.B, s.Hkv, s.D, s.n_blocks = B, Hkv, 128, n_blocks
    s.k_pool = _dense(cache.k_pool, f8, (*lead, n_blocks, Hkv, PAGE_TOKENS, 128), torch.uint8)
    s.v_pool = _dense(cache.v_pool, f8, (*lead, n_blocks, Hkv, 128, PAGE_TOKENS), torch.uint8)
    s.k_scale = _dense(cache.k_scale, torch.float32, (*lead, n_blocks, Hkv))
    s.v_scale = _dense(cache.v_scale, torch.float32, (*lead, n_blocks, Hkv))
    s.k_tail = _dense(cache.k_tail, bf, (*lead, B, Hkv, TAIL_ROWS, 128))
    s.v_tail = _dense(cache.v_tail, bf, (*lead, B, Hkv, TAIL_ROWS, 128))
    return s


def paged_plan_args(kv_len, n_new, held, queue, state, table, *, outs, max_rows, reserve=0,
                    draft=False) -> PagedPlanArgs:
    i32 = torch.int32
    B, cols = table.shape
    _one_device(kv_len, n_new, held, queue, state, table, *outs.values())
    a = PagedPlanArgs()
    a.B, a.table_cols, a.n_blocks = B, cols, queue.numel()
    a.max_rows, a.reserve, a.draft = int(max_rows), int(reserve), 1 if draft else 0
    a.kv_len, a.n_new, a.held = (_dense(x, i32, (B,)) for x in (kv_len, n_new, held))
    a.state, a.queue, a.table = _dense(state, i32, (2,)), _dense(queue, i32, queue.shape), _dense(table, i32, (B, cols))
    sizes = dict(granted=B, new_held=B, new_state=2, cu_rows=B + 1, slots=max_rows, row_seq=max_rows, row_pos=max_rows)
    for name, n in sizes.items():
        setattr(a, name, _dense(outs[name], i32, (n,)))
    return a


@_allocates_on_stream
def paged_plan(kv_len, n_new, held, queue, state, table, *, max_rows, reserve=0, draft=False, outs=None,
               stream=None) -> dict:
    """lvspec_paged_plan.  kv_len, n_new, held int32 [B]; queue int32 [n_blocks], state int32 [2], table
    int32 [B, cols] (queue and table are changed); kv_len 0 and n_new -1 where a request has finished or
    there is none.  Returns granted, new_held, new_state, cu_rows, slots, row_seq, row_pos; new_held and
    new_state are held and state of the next call."""
    if outs is None:
        outs = alloc_paged_plan(table.shape[0], max_rows, table.device)
    a = paged_plan_args(kv_len, n_new, held, queue, state, table, outs=outs, max_rows=max_rows, reserve=reserve,
                        draft=draft)
    _call_on(table.device, _lib.lvspec_paged_plan, a, stream)
    return outs


def _fill_append(a, cache, k, v, plan):
    """The packed rows of an append, a.cache set."""
    i32 = torch.int32
    _one_device(*cache, k, v, plan["slots"], plan["row_seq"], plan["row_pos"], plan["cu_rows"])
    n = k.shape[0]
    assert k.is_cuda and v.is_cuda and k.dtype == torch.bfloat16 and v.dtype == torch.bfloat16 and k.shape == v.shape
    assert k.shape[1:] == (a.cache.Hkv, 128) and k.stride(-1) == 1 and v.stride(-1) == 1
    a.n_rows, a.k, a.v = n, k.data_ptr(), v.data_ptr()
    (a.k_sr, a.k_sh), (a.v_sr, a.v_sh) = _strides(k), _strides(v)
    a.slots, a.row_seq, a.row_pos = (_dense(plan[x], i32, (n,)) for x in ("slots", "row_seq", "row_pos"))
    a.cu_rows = _dense(plan["cu_rows"], i32, (a.cache.B + 1,))
    return a


def paged_append_args(cache: PagedCache, k, v, plan) -> PagedAppendArgs:
    a = PagedAppendArgs()
    a.cache = _cache_struct(cache)
    return _fill_append(a, cache, k, v, plan)


def paged_append(cache: PagedCache, k, v, plan, *, stream=None) -> None:
    """lvspec_paged_append.  k, v bf16 [n_rows, Hkv, 128], a packed row for every entry of the plan's
    maps (plan: what paged_plan returned, with max_rows = n_rows)."""
    a = paged_append_args(cache, k, v, plan)
    _call_on(k.device, _lib.lvspec_paged_append, a, stream)


def verify_attn_paged_args(q, cache: PagedCache, table, kv_len, *, out, vis_begin=None, vis_end=None,
                           draft_mask=None, scale=0.0, lse=None, vis_mass=None) -> PagedAttnArgs:
    a = PagedAttnArgs()
    a.cache = _cache_struct(cache)
    return _fill_attn(a, q, cache, table, kv_len, out, vis_begin, vis_end, draft_mask, scale, lse, vis_mass)


def _fill_attn(a, q, cache, table, kv_len, out, vis_begin, vis_end, draft_mask, scale, lse, vis_mass):
    """The other fields of an attention over a paged cache, a.cache set."""
    i32 = torch.int32
    _one_device(*cache, q, table, kv_len, out, vis_begin, vis_end, lse, vis_mass)
    B, gamma, Hq, D = q.shape
    assert q.is_cuda and out.is_cuda and q.dtype == torch.bfloat16 and out.dtype == torch.bfloat16
    assert out.shape == q.shape
    assert B == a.cache.B and D == 128 and q.stride(-1) == 1 and out.stride(-1) == 1
    a.gamma, a.Hq = gamma, Hq
    a.q, (a.q_sb, a.q_sg, a.q_sh) = q.data_ptr(), _strides(q)
    a.table, a.table_cols = _dense(table, i32, (B, table.shape[1])), table.shape[1]
    a.kv_len = _dense(kv_len, i32, (B,))
    for name, t in (("vis_begin", vis_begin), ("vis_end", vis_end)):
        setattr(a, name, None if t is None else _dense(t, i32, (B,)))
    if draft_mask is not None:
        assert len(draft_mask) == gamma
        a._keep = a.draft_mask = (C.c_uint32 * gamma)(*[int(m) for m in draft_mask])
    a.scale = float(scale)
    a.out, (a.o_sb, a.o_sg, a.o_sh) = out.data_ptr(), _strides(out)
    for name, t in (("lse", lse), ("vis_mass", vis_mass)):
        setattr(a, name, None if t is None else _dense(t, torch.float32, (B, Hq, gamma)))
    return a


@_allocates_on_stream
def verify_attn_paged(q, cache: PagedCache, table, kv_len, *, vis_begin=None, vis_end=None, draft_mask=None,
                      scale=0.0, out=None, return_lse=False, return_vis_mass=False, workspace=None,
                      stream=None):
    """lvspec_verify_attn_paged.  q bf16 [B,gamma,Hq,128], one layer's cache, table int32 [B,cols], kv_len
    int32 [B].  Returns out, or (out, lse, vis_mass) when either extra is asked for."""
    return _attn(verify_attn_paged_args, "verify_attn_paged", q, cache, table, kv_len, vis_begin, vis_end, draft_mask,
                 scale, out, return_lse, return_vis_mass, workspace, stream)


def _attn(make, name, q, cache, table, kv_len, vis_begin, vis_end, draft_mask, scale, out, return_lse, return_vis_mass,
          workspace, stream):
    B, gamma, Hq, _ = q.shape
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    lse = q.new_empty((B, Hq, gamma), dtype=torch.float32) if return_lse else None
    vm = q.new_empty((B, Hq, gamma), dtype=torch.float32) if return_vis_mass else None
    a = make(q, cache, table, kv_len, out=out, vis_begin=vis_begin, vis_end=vis_end, draft_mask=draft_mask, scale=scale,
             lse=lse, vis_mass=vm)
    ws = _workspace(getattr(_lib, f"lvspec_{name}_workspace")(C.byref(a)), q, workspace)
    a.workspace, a.workspace_bytes = ws.data_ptr(), ws.numel() * ws.element_size()
    _call_on(q.device, getattr(_lib, f"lvspec_{name}"), a, stream)
    if return_lse or return_vis_mass:
        return out, lse, vm
    return out


def paged_commit_args(cache: PagedCache, table, kv_len, accept_len, chain_len, *, best_branch=None, n_branches=1,
                      new_len, plan=None) -> PagedCommitArgs:
    a = PagedCommitArgs()
    layers = cache.k_pool.shape[0] if cache.k_pool.dim() == 5 else 1
    a.cache = _cache_struct(cache, (layers,) if cache.k_pool.dim() == 5 else ())
    return _fill_commit(a, layers, cache, table, kv_len, accept_len, chain_len, best_branch, n_branches, new_len, plan)


def _fill_commit(a, layers, cache, table, kv_len, accept_len, chain_len, best_branch, n_branches, new_len, plan):
    """The other fields of a commit to a paged cache, a.cache set."""
    i32 = torch.int32
    given = () if plan is None else (plan["granted"], plan["new_held"], plan["cu_rows"])
    _one_device(*cache, table, kv_len, accept_len, best_branch, new_len, *given)
    B = a.cache.B
    a.n_layers, a.n_branches, a.chain_len = layers, int(n_branches), int(chain_len)
    a.table, a.table_cols = _dense(table, i32, (B, table.shape[1])), table.shape[1]
    a.kv_len, a.new_len = _dense(kv_len, i32, (B,)), _dense(new_len, i32, (B,))
    a.accept_len = _dense(accept_len, i32, (B * max(1, int(n_branches)),))
    a.best_branch = None if best_branch is None else _dense(best_branch, i32, (B,))
    if plan is not None:
        a.granted, a.held, a.cu_rows = (_dense(x, i32, (n,)) for x, n in zip(given, (B, B, B + 1)))
    return a


@_allocates_on_stream
def paged_commit(cache: PagedCache, table, kv_len, accept_len, chain_len, *, best_branch=None, n_branches=1,
                 new_len=None, plan=None, stream=None):
    """lvspec_paged_commit.  cache of one layer, or of all with a leading dimension; accept_len int32
    [B*n_branches], best_branch int32 [B] (trees); plan: what the step's paged_plan returned, by which
    refused sequences are left as they are (None: the caller answers for all having been granted).
    Returns new_len int32 [B]."""
    if new_len is None:
        new_len = torch.empty_like(kv_len)
    a = paged_commit_args(cache, table, kv_len, accept_len, chain_len, best_branch=best_branch,
                          n_branches=n_branches, new_len=new_len, plan=plan)
    _call_on(table.device, _lib.lvspec_paged_commit, a, stream)
    return new_len


# ------------------------------------------------------------------ rotary positions
class Rotary(NamedTuple):
    """How rows are turned: frequencies and factor as rotary_frequencies gives them."""
    inv_freq: torch.Tensor                  # fp32 [dim / 2] on the device
    factor: float = 1.0
    interleaved: bool = False
    axis: Optional[torch.Tensor] = None     # uint8 [dim / 2]: which of a token's positions a frequency goes by


def rotary_frequencies(dim, base=10000.0, *, scaling=SCALING_NONE, scale=1.0, original_len=0, beta_fast=0.0, beta_slow=0.0,
                       device=None):
    """lvspec_rotary_frequencies: (inv_freq fp32 [dim / 2] on `device`, factor)."""
    if not 0 < dim <= 512:                     # (before 32 bits are taken of it)
        raise LvspecError(EINVAL)
    a = RotaryFreqArgs(int(dim), int(scaling), float(base), float(scale), float(original_len), float(beta_fast),
                       float(beta_slow))
    out, factor = (C.c_float * max(1, int(dim) // 2))(), C.c_float()
    _check(_lib.lvspec_rotary_frequencies(C.byref(a), out, C.byref(factor)))
    return torch.tensor(list(out), dtype=torch.float32, device=device), float(factor.value)


_ROTARY_TYPES = {torch.bfloat16: BF16, torch.float16: F16, torch.float32: F32}


def _fill_rotation(r: Rotation, rot: Rotary, pos, n_rows, transpose=False):
    inv = rot.inv_freq
    half = inv.numel()
    assert half > 0
    r.dim, r.interleaved, r.transpose = 2 * half, 1 if rot.interleaved else 0, 1 if transpose else 0
    r.inv_freq = _dense(inv, torch.float32, (half,))
    r.axis = None if rot.axis is None else _dense(rot.axis, torch.uint8, (half,))
    r.factor = float(rot.factor)
    r.n_axes = 1
    if pos is not None:
        n_axes = 1 if pos.dim() == 1 else pos.shape[0]
        assert pos.is_cuda and pos.dtype == torch.int32 and pos.shape[-1] == n_rows and pos.dim() <= 2
        assert pos.stride(-1) == 1 or n_rows <= 1
        r.n_axes, r.pos, r.pos_sa = n_axes, pos.data_ptr(), pos.stride(0) if pos.dim() == 2 and n_axes > 1 else 0
    assert rot.axis is not None or r.n_axes == 1


def _rows_of(x, dtype, n_rows):
    """[n_rows, H, D] with rows of contiguous channels: (data, row and head strides, in 16 bytes where there is one)."""
    n, H, D = x.shape
    assert x.is_cuda and x.dtype == dtype and n == n_rows and (x.stride(-1) == 1 or D == 1)
    most = -(-D // 8) * 8
    return x.data_ptr(), x.stride(0) if n > 1 else max(most, H * most), x.stride(1) if H > 1 else most


def _new_rows(x):
    """Uninitialised rows of x's shape as _rows_of wants them: every head from one 16-byte border to the next."""
    n, H, D = x.shape
    per = 16 // x.element_size()
    if D % per == 0:
        return torch.empty_like(x, memory_format=torch.contiguous_format)
    return torch.empty((n, H, -(-D // per) * per), dtype=x.dtype, device=x.device)[..., :D]


def _fill_queries(a, q, q_out, n_rows):
    a.Hq = 0
    if q is not None:
        assert q_out is not None and q_out.shape == q.shape and q.shape[2] == 128
        a.Hq = q.shape[1]
        a.q, a.q_sr, a.q_sh = _rows_of(q, torch.bfloat16, n_rows)
        a.q_out, a.qo_sr, a.qo_sh = _rows_of(q_out, torch.bfloat16, n_rows)


def rotary_args(q, pos, rot: Rotary, *, out, k=None, k_out=None, transpose=False) -> RotaryArgs:
    a = RotaryArgs()
    n, Hq, D = q.shape
    assert n < 1 << 31, f"{n} rows"            # (the field would take 32 bits of it)
    _one_device(q, pos, out, k, k_out, rot.inv_freq, rot.axis)
    _fill_rotation(a.rot, rot, pos, n, transpose)
    a.n_rows, a.Hq, a.Hkv, a.D, a.dtype = n, Hq, 0, D, _ROTARY_TYPES[q.dtype]
    assert out.shape == q.shape
    a.q, a.q_sr, a.q_sh = _rows_of(q, q.dtype, n)
    a.q_out, a.qo_sr, a.qo_sh = _rows_of(out, q.dtype, n)
    if k is not None:
        assert k.shape[2] == D and k_out is not None and k_out.shape == k.shape
        a.Hkv = k.shape[1]
        a.k, a.k_sr, a.k_sh = _rows_of(k, q.dtype, n)
        a.k_out, a.ko_sr, a.ko_sh = _rows_of(k_out, q.dtype, n)
    return a


@_allocates_on_stream
def rotary(q, pos, rot: Rotary, *, k=None, out=None, k_out=None, transpose=False, stream=None):
    """lvspec_rotary.  q [n_rows,Hq,D] and k [n_rows,Hkv,D] (optional) bf16, fp16 or fp32; pos int32 [n_rows], or
    [n_axes,n_rows] with rot.axis.  out and k_out may be q and k.  transpose: turned back, the gradient of q (and k)
    from that of out.  Returns out, or (out, k_out).  Rows and heads start on 16-byte borders, so heads of other sizes are
    slices of wider ones; what is allocated here is, and contiguous where heads are whole multiples of 16 bytes."""
    if out is None:
        out = _new_rows(q)
    if k is not None and k_out is None:
        k_out = _new_rows(k)
    a = rotary_args(q, pos, rot, out=out, k=k, k_out=k_out, transpose=transpose)
    _call_on(q.device, _lib.lvspec_rotary, a, stream)
    return out if k is None else (out, k_out)


def paged_append_rotary_args(cache: PagedCache, k, v, plan, rot: Rotary, *, pos=None, q=None, q_out=None) -> PagedAppendRotaryArgs:
    a = PagedAppendRotaryArgs()
    _one_device(k, pos, q, q_out, rot.inv_freq, rot.axis)
    a.rows = paged_append_args(cache, k, v, plan)
    _fill_rotation(a.rot, rot, pos, k.shape[0])
    _fill_queries(a, q, q_out, k.shape[0])
    return a


@_allocates_on_stream
def paged_append_rotary(cache: PagedCache, k, v, plan, rot: Rotary, *, pos=None, q=None, q_out=None, stream=None):
    """lvspec_paged_append_rotary: paged_append of k as rot turns it.  pos int32 [n_rows] or [n_axes,n_rows] (None: the
    rows' places in the cache); q bf16 [n_rows,Hq,128] is turned in the same launch.  Returns q_out (None without q).
    A q_out that is allocated here holds zeros where there is no row."""
    if q is not None and q_out is None:
        q_out = torch.zeros_like(q, memory_format=torch.contiguous_format)
    a = paged_append_rotary_args(cache, k, v, plan, rot, pos=pos, q=q, q_out=q_out)
    _call_on(k.device, _lib.lvspec_paged_append_rotary, a, stream)
    return q_out


# ------------------------------------------------------------------ paged cache in 4 bits
class PagedMxCache(NamedTuple):
    """The arrays of one layer, or of several with a leading dimension (include/lvspec.h says what
    they hold).  Plans, tables and slots are those of the cache in 8 bits."""
    k_pool: torch.Tensor      # uint8 [n_blocks, Hkv, 2, 64, 32]
    v_pool: torch.Tensor      # uint8 [n_blocks, Hkv, 128, 32]
    k_scale: torch.Tensor     # uint8 [n_blocks, Hkv, 2, 32, 4]
    v_scale: torch.Tensor
    k_tail: torch.Tensor      # bf16 [B, Hkv, 128, 128]
    v_tail: torch.Tensor

    def layer(self, i: int) -> "PagedMxCache":
        return PagedMxCache(*[x[i] for x in self])


def _paged_mx_shapes(B, Hkv, n_blocks):
    pool = (n_blocks, Hkv)
    return [((*pool, 2, PAGE_TOKENS, 32), torch.uint8), ((*pool, 128, 32), torch.uint8),
            ((*pool, 2, 32, 4), torch.uint8), ((*pool, 2, 32, 4), torch.uint8),
            ((B, Hkv, TAIL_ROWS, 128), torch.bfloat16), ((B, Hkv, TAIL_ROWS, 128), torch.bfloat16)]


def alloc_paged_mx_cache(B, Hkv, n_blocks, device, layers: Optional[int] = None) -> PagedMxCache:
    lead = () if layers is None else (layers,)
    return PagedMxCache(*[torch.zeros(lead + s, dtype=t, device=device) for s, t in _paged_mx_shapes(B, Hkv, n_blocks)])


def _cache4_struct(cache: PagedMxCache, lead=()) -> PagedMxCacheStruct:
    n_blocks, Hkv = cache.k_pool.shape[len(lead):len(lead) + 2]
    s = PagedMxCacheStruct()
    s.B, s.Hkv, s.D, s.n_blocks = cache.k_tail.shape[len(lead)], Hkv, 128, n_blocks
    for name, x, (shape, dtype) in zip(PagedMxCache._fields, cache, _paged_mx_shapes(s.B, Hkv, n_blocks)):
        setattr(s, name, _dense(x, dtype, (*lead, *shape)))
    return s


def paged_mx_append_args(cache: PagedMxCache, k, v, plan, *, rot: Optional[Rotary] = None, pos=None, q=None,
                       q_out=None) -> PagedMxAppendArgs:
    a = PagedMxAppendArgs()
    a.cache = _cache4_struct(cache)
    _fill_append(a, cache, k, v, plan)
    if rot is None:
        assert pos is None and q is None
        return a
    _one_device(k, pos, q, q_out, rot.inv_freq, rot.axis)
    _fill_rotation(a.rot, rot, pos, k.shape[0])
    _fill_queries(a, q, q_out, k.shape[0])
    return a


@_allocates_on_stream
def paged_mx_append(cache: PagedMxCache, k, v, plan, *, rot: Optional[Rotary] = None, pos=None, q=None, q_out=None,
                  stream=None):
    """lvspec_paged_mx_append: as paged_append or, with rot, as paged_append_rotary."""
    if q is not None and q_out is None:
        q_out = torch.zeros_like(q, memory_format=torch.contiguous_format)
    a = paged_mx_append_args(cache, k, v, plan, rot=rot, pos=pos, q=q, q_out=q_out)
    _call_on(k.device, _lib.lvspec_paged_mx_append, a, stream)
    return q_out


def paged_mx_read_args(cache: PagedMxCache, slots, *, k, v) -> PagedMxReadArgs:
    a = PagedMxReadArgs()
    _one_device(*cache, slots, k, v)
    a.cache = _cache4_struct(cache)
    n = slots.shape[0]
    a.n_rows, a.slots = n, _dense(slots, torch.int32, (n,))
    assert k.shape == v.shape == (n, a.cache.Hkv, 128)
    a.k, a.k_sr, a.k_sh = _rows_of(k, torch.bfloat16, n)
    a.v, a.v_sr, a.v_sh = _rows_of(v, torch.bfloat16, n)
    return a


@_allocates_on_stream
def paged_mx_read(cache: PagedMxCache, slots, *, k=None, v=None, stream=None):
    """lvspec_paged_mx_read: the rows at slots int32 [n_rows] (a plan's, say), bf16 [n_rows,Hkv,128].  Returns (k, v);
    what is allocated here holds zeros where a slot names no row."""
    shape = (slots.shape[0], cache.k_tail.shape[1], 128)
    k, v = (torch.zeros(shape, dtype=torch.bfloat16, device=slots.device) if x is None else x for x in (k, v))
    a = paged_mx_read_args(cache, slots, k=k, v=v)
    _call_on(slots.device, _lib.lvspec_paged_mx_read, a, stream)
    return k, v


def verify_attn_paged_mx_args(q, cache: PagedMxCache, table, kv_len, *, out, vis_begin=None, vis_end=None,
                            draft_mask=None, scale=0.0, lse=None, vis_mass=None) -> PagedMxAttnArgs:
    a = PagedMxAttnArgs()
    a.cache = _cache4_struct(cache)
    return _fill_attn(a, q, cache, table, kv_len, out, vis_begin, vis_end, draft_mask, scale, lse, vis_mass)


@_allocates_on_stream
def verify_attn_paged_mx(q, cache: PagedMxCache, table, kv_len, *, vis_begin=None, vis_end=None, draft_mask=None,
                       scale=0.0, out=None, return_lse=False, return_vis_mass=False, workspace=None,
                       stream=None):
    """lvspec_verify_attn_paged_mx: as verify_attn_paged."""
    return _attn(verify_attn_paged_mx_args, "verify_attn_paged_mx", q, cache, table, kv_len, vis_begin, vis_end, draft_mask,
                 scale, out, return_lse, return_vis_mass, workspace, stream)


def paged_mx_commit_args(cache: PagedMxCache, table, kv_len, accept_len, chain_len, *, best_branch=None, n_branches=1,
                       new_len, plan=None) -> PagedMxCommitArgs:
    a = PagedMxCommitArgs()
    layers = cache.k_pool.shape[0] if cache.k_pool.dim() == 6 else 1
    a.cache = _cache4_struct(cache, (layers,) if cache.k_pool.dim() == 6 else ())
    return _fill_commit(a, layers, cache, table, kv_len, accept_len, chain_len, best_branch, n_branches, new_len, plan)


@_allocates_on_stream
def paged_mx_commit(cache: PagedMxCache, table, kv_len, accept_len, chain_len, *, best_branch=None, n_branches=1,
                  new_len=None, plan=None, stream=None):
    """lvspec_paged_mx_commit: as paged_commit."""
    if new_len is None:
        new_len = torch.empty_like(kv_len)
    a = paged_mx_commit_args(cache, table, kv_len, accept_len, chain_len, best_branch=best_branch,
                           n_branches=n_branches, new_len=new_len, plan=plan)
    _call_on(table.device, _lib.lvspec_paged_mx_commit, a, stream)
    return new_len
