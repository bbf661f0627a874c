"""ctypes binding of libtreetrain.so.  Argument marshalling only.

Streams: a call queues its work on the current stream, or on the torch.cuda.Stream that it is given as `stream`.  The inputs have to be
ready on that stream and to stay until it is through with them; outputs are used on another stream behind an event or a wait of it, as
for any work on a stream of one's own.
"""
from __future__ import annotations

import ctypes
import functools
import os
from dataclasses import dataclass
from typing import NamedTuple, Optional

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
KTILE = 64
DTYPE_BF16, DTYPE_FP32 = 0, 1
FLAG_REFERENCE_KERNELS = 1

_c_i32p = ctypes.POINTER(ctypes.c_int32)
_c_u8p = ctypes.POINTER(ctypes.c_uint8)
_c_f32p = ctypes.POINTER(ctypes.c_float)
_vp = ctypes.c_void_p


class TreeTrainError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"libtreetrain status {status}: {message}")
        self.status = status


class _MetaSizes(ctypes.Structure):
    _fields_ = [("n_nodes", ctypes.c_int32), ("n_tokens", ctypes.c_int32), ("n_leaves", ctypes.c_int32),
                ("n_roots", ctypes.c_int32), ("n_ktiles", ctypes.c_int32)]


class _PartitionSizes(ctypes.Structure):
    _fields_ = [("n_parts", ctypes.c_int32), ("n_tokens", ctypes.c_int32), ("max_part_tokens", ctypes.c_int32),
                ("max_prefix", ctypes.c_int32), ("sum_prefix", ctypes.c_int64), ("sum_ktiles", ctypes.c_int64)]


class _PartitionPlan(ctypes.Structure):
    _fields_ = [("n_parts", ctypes.c_int32), ("n_tokens", ctypes.c_int32),
                ("part_tok_off", _vp), ("part_prefix_off", _vp), ("part_ktile_off", _vp),
                ("part_own_start", _vp), ("part_prefix_start", _vp),
                ("own_tok", _vp), ("prefix_tok", _vp), ("kend", _vp), ("kt_min", _vp), ("kt_max", _vp)]


class _AttnDesc(ctypes.Structure):
    _fields_ = [("n_q", ctypes.c_int32), ("n_prefix", ctypes.c_int32), ("hq", ctypes.c_int32),
                ("hkv", ctypes.c_int32), ("d", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("scale", ctypes.c_float), ("flags", ctypes.c_int32),
                ("q_stride_tok", ctypes.c_int64), ("k_stride_tok", ctypes.c_int64),
                ("v_stride_tok", ctypes.c_int64)]


def lib_path() -> str:
    return os.path.join(HERE, "libtreetrain.so")


_LIB = None


def _lib() -> ctypes.CDLL:
    global _LIB
    if _LIB is None:
        path = lib_path()
        if not os.path.exists(path):
            raise ImportError(
                f"{path} is missing: build it with `python -m paper_2511_00413_amd.build` "
                "(there is no fallback implementation)")
        # The library and PyTorch must share one HIP runtime.  PyTorch ships its own copy under the same soname, so
        # whichever is loaded first serves both; with the system's copy loaded first, device calls made after
        # `import torch` have failed with "no ROCm-capable device".  Load PyTorch's first when it is there.
        try:
            import torch  # noqa: F401
        except ImportError:
            pass
        lib = ctypes.CDLL(path)
        lib.tt_last_error.restype = ctypes.c_char_p
        lib.tt_version.restype = ctypes.c_int32
        lib.tt_tree_attn_workspace.restype = ctypes.c_size_t
        lib.tt_tree_attn_workspace.argtypes = [ctypes.POINTER(_AttnDesc), ctypes.c_int32]
        lib.tt_tree_meta_sizes.restype = ctypes.c_int32
        lib.tt_tree_meta_sizes.argtypes = [ctypes.c_int32, _vp, _vp, ctypes.c_int32, ctypes.POINTER(_MetaSizes)]
        lib.tt_tree_build_meta.restype = ctypes.c_int32
        lib.tt_tree_build_meta.argtypes = [ctypes.c_int32, _vp, _vp, _vp, _vp, _vp, ctypes.c_int32,
                                           ctypes.c_int32, _vp] + [_vp] * 13
        lib.tt_tree_attn_fwd.restype = ctypes.c_int32
        lib.tt_tree_attn_fwd.argtypes = [ctypes.POINTER(_AttnDesc)] + [_vp] * 10 + [_vp, ctypes.c_size_t, _vp]
        lib.tt_tree_attn_bwd.restype = ctypes.c_int32
        lib.tt_tree_attn_bwd.argtypes = [ctypes.POINTER(_AttnDesc)] + [_vp] * 16 + [_vp, ctypes.c_size_t, _vp]
        lib.tt_tree_weighted_logprob.restype = ctypes.c_int32
        lib.tt_tree_weighted_logprob.argtypes = [ctypes.c_int64, ctypes.c_int32, ctypes.c_int32, _vp,
                                                 ctypes.c_int64, _vp, _vp, _vp, _vp, _vp, _vp]
        lib.tt_tree_weighted_logprob_bwd.restype = ctypes.c_int32
        lib.tt_tree_weighted_logprob_bwd.argtypes = [ctypes.c_int64, ctypes.c_int32, ctypes.c_int32, _vp, ctypes.c_int64,
                                                     _vp, _vp, _vp, ctypes.c_float, _vp, ctypes.c_int64, _vp]
        lib.tt_tree_weighted_logprob_fwd_bwd.restype = ctypes.c_int32
        lib.tt_tree_weighted_logprob_fwd_bwd.argtypes = [ctypes.c_int64, ctypes.c_int32, ctypes.c_int32, _vp, ctypes.c_int64,
                                                         _vp, _vp, ctypes.c_float, _vp, _vp, _vp, _vp, ctypes.c_int64, _vp]
        lib.tt_tree_rope.restype = ctypes.c_int32
        lib.tt_tree_rope.argtypes = [ctypes.c_int64, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, _vp, ctypes.c_int64,
                                     _vp, ctypes.c_float, ctypes.c_int32, _vp, ctypes.c_int64, _vp]
        lib.tt_tree_rope_axes.restype = ctypes.c_int32
        lib.tt_tree_rope_axes.argtypes = [ctypes.c_int64, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, _vp, ctypes.c_int64,
                                          ctypes.c_int32, _vp, ctypes.c_char_p, ctypes.c_float, ctypes.c_int32, _vp, ctypes.c_int64, _vp]
        lib.tt_tree_axis_positions.restype = ctypes.c_int32
        lib.tt_tree_axis_positions.argtypes = [ctypes.c_int32, _vp, _vp, _vp, _vp, _vp]
        lib.tt_tree_logprob_entropy_workspace.restype = ctypes.c_size_t
        lib.tt_tree_logprob_entropy_workspace.argtypes = [ctypes.c_int64, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32]
        lib.tt_tree_logprob_entropy.restype = ctypes.c_int32
        lib.tt_tree_logprob_entropy.argtypes = [ctypes.c_int64, ctypes.c_int32, ctypes.c_int32, _vp, ctypes.c_int64, _vp, ctypes.c_int32,
                                                _vp, _vp, _vp, _vp, _vp, _vp, ctypes.c_size_t, _vp]
        lib.tt_tree_logprob_entropy_bwd.restype = ctypes.c_int32
        lib.tt_tree_logprob_entropy_bwd.argtypes = [ctypes.c_int64, ctypes.c_int32, ctypes.c_int32, _vp, ctypes.c_int64, _vp, _vp, _vp,
                                                    _vp, _vp, _vp, ctypes.c_int64, _vp]
        lib.tt_tree_conv_fwd.restype = ctypes.c_int32
        lib.tt_tree_conv_fwd.argtypes = [ctypes.c_int64, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, _vp,
                                         ctypes.c_int64, _vp, _vp, _vp, _vp, ctypes.c_int64, _vp]
        lib.tt_tree_conv_plan_sizes.restype = ctypes.c_int32
        lib.tt_tree_conv_plan_sizes.argtypes = [ctypes.c_int64, _vp, ctypes.c_int32, _c_i32p, _c_i32p]
        lib.tt_tree_conv_plan.restype = ctypes.c_int32
        lib.tt_tree_conv_plan.argtypes = [ctypes.c_int64, _vp, ctypes.c_int32, _vp, _vp, _vp, _vp]
        lib.tt_tree_conv_bwd_workspace.restype = ctypes.c_size_t
        lib.tt_tree_conv_bwd_workspace.argtypes = [ctypes.c_int64, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32]
        lib.tt_tree_conv_bwd.restype = ctypes.c_int32
        lib.tt_tree_conv_bwd.argtypes = [ctypes.c_int64, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, _vp,
                                         ctypes.c_int64, _vp, _vp, _vp, _vp, ctypes.c_int64, ctypes.c_int32, _vp, _vp, _vp, _vp,
                                         _vp, ctypes.c_int64, _vp, _vp, _vp, ctypes.c_size_t, _vp]
        lib.tt_tree_conv_bwd_static.restype = ctypes.c_int32
        lib.tt_tree_conv_bwd_static.argtypes = [ctypes.c_int64, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, _vp,
                                                ctypes.c_int64, _vp, _vp, _vp, _vp, ctypes.c_int64, ctypes.c_int32, _vp, _vp, _vp,
                                                _vp, _vp, ctypes.c_int64, _vp, _vp, _vp]
        lib.tt_tree_gdn_plan_sizes.restype = ctypes.c_int32
        lib.tt_tree_gdn_plan_sizes.argtypes = [ctypes.c_int32, _vp, _vp, _c_i32p, _c_i32p]
        lib.tt_tree_gdn_plan.restype = ctypes.c_int32
        lib.tt_tree_gdn_plan.argtypes = [ctypes.c_int32, _vp, _vp, ctypes.c_int32, _vp, _vp, _vp, _vp, _vp, _vp]
        lib.tt_tree_gdn_workspace.restype = ctypes.c_size_t
        lib.tt_tree_gdn_workspace.argtypes = [ctypes.c_int32, ctypes.c_int32, ctypes.c_int32]
        lib.tt_tree_gdn_fwd.restype = ctypes.c_int32
        lib.tt_tree_gdn_fwd.argtypes = [ctypes.c_int64, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_float,
                                        _vp, _vp, _vp, _vp, _vp, ctypes.c_int32, _vp, _vp, _vp, _vp, ctypes.c_int32, _vp, _vp, _vp, _vp,
                                        _vp, _vp, ctypes.c_size_t, _vp]
        lib.tt_tree_gdn_schedule_sizes.restype = ctypes.c_int32
        lib.tt_tree_gdn_schedule_sizes.argtypes = [ctypes.c_int32, _vp, _vp, ctypes.c_int32, _c_i32p, _c_i32p, _c_i32p]
        lib.tt_tree_gdn_schedule.restype = ctypes.c_int32
        lib.tt_tree_gdn_schedule.argtypes = [ctypes.c_int32, _vp, _vp, ctypes.c_int32, _vp, _vp, _vp, _vp, _vp]
        lib.tt_tree_gdn_bwd_workspace.restype = ctypes.c_size_t
        lib.tt_tree_gdn_bwd_workspace.argtypes = [ctypes.c_int64, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32]
        lib.tt_tree_gdn_bwd_workspace_min.restype = ctypes.c_size_t
        lib.tt_tree_gdn_bwd_workspace_min.argtypes = lib.tt_tree_gdn_bwd_workspace.argtypes
        lib.tt_tree_gdn_bwd.restype = ctypes.c_int32
        lib.tt_tree_gdn_bwd.argtypes = [ctypes.c_int64, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_float,
                                        _vp, _vp, _vp, _vp, _vp, _vp, ctypes.c_int32, _vp, _vp, _vp, _vp, ctypes.c_int32, _vp, _vp, _vp, _vp,
                                        _vp, _vp, _vp, _vp, _vp, _vp, _vp, ctypes.c_size_t, _vp]
        desc, chunks = ctypes.POINTER(_ScanDesc), ctypes.POINTER(_ScanChunks)
        lib.tt_tree_scan_program.restype = ctypes.c_int32
        lib.tt_tree_scan_program.argtypes = [ctypes.c_int32] + [_vp] * 5 + [ctypes.c_int32, ctypes.c_int32, _c_i32p] + [_vp] * 5
        for name in ("tt_tree_scan_fwd_workspace", "tt_tree_scan_bwd_workspace"):
            getattr(lib, name).restype = ctypes.c_size_t
            getattr(lib, name).argtypes = [desc, ctypes.c_int32, ctypes.c_int32]
        lib.tt_tree_scan_fwd.restype = ctypes.c_int32
        lib.tt_tree_scan_fwd.argtypes = [desc, chunks] + [_vp] * 12 + [ctypes.c_size_t, _vp]
        lib.tt_tree_scan_bwd.restype = ctypes.c_int32
        lib.tt_tree_scan_bwd.argtypes = [desc, chunks] + [_vp] * 21 + [ctypes.c_size_t, _vp]
        lib.tt_tree_scan_step.restype = ctypes.c_int32
        lib.tt_tree_scan_step.argtypes = [desc] + [_vp] * 8 + [ctypes.c_int32] + [_vp] * 5
        lib.tt_tree_conv_step.restype = ctypes.c_int32
        lib.tt_tree_conv_step.argtypes = [ctypes.c_int64, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, _vp, ctypes.c_int64,
                                          _vp, _vp, ctypes.c_int32, _vp, _vp, _vp, _vp, ctypes.c_int64, _vp]
        lib.tt_tree_path_weights.restype = ctypes.c_int32
        lib.tt_tree_path_weights.argtypes = [ctypes.c_int32, _vp, _vp, _vp, ctypes.c_int32, _vp, _vp, _vp, _vp]
        lib.tt_tree_partition_sizes.restype = ctypes.c_int32
        lib.tt_tree_partition_sizes.argtypes = [ctypes.c_int32, _vp, _vp, ctypes.c_int32, ctypes.POINTER(_PartitionSizes)]
        lib.tt_tree_partition_plan.restype = ctypes.c_int32
        lib.tt_tree_partition_plan.argtypes = [ctypes.c_int32, _vp, _vp, ctypes.c_int32] + [_vp] * 17
        lib.tt_tree_attn_partitioned_workspace.restype = ctypes.c_size_t
        lib.tt_tree_attn_partitioned_workspace.argtypes = [ctypes.POINTER(_AttnDesc), ctypes.POINTER(_PartitionPlan), ctypes.c_int32]
        lib.tt_tree_attn_partitioned_fwd.restype = ctypes.c_int32
        lib.tt_tree_attn_partitioned_fwd.argtypes = [ctypes.POINTER(_AttnDesc), ctypes.POINTER(_PartitionPlan)] + [_vp] * 5 + [_vp, ctypes.c_size_t, _vp]
        lib.tt_tree_attn_partitioned_bwd.restype = ctypes.c_int32
        lib.tt_tree_attn_partitioned_bwd.argtypes = [ctypes.POINTER(_AttnDesc), ctypes.POINTER(_PartitionPlan)] + [_vp] * 9 + [_vp, ctypes.c_size_t, _vp]
        lib.tt_kernel_timing_enable.restype = ctypes.c_int32
        lib.tt_kernel_timing_enable.argtypes = [ctypes.c_int32]
        lib.tt_kernel_timing_read.restype = ctypes.c_int32
        lib.tt_kernel_timing_read.argtypes = [ctypes.POINTER(_KernelTimes)]
        _LIB = lib
    return _LIB


KERNEL_NAMES = ("attn_fwd", "loss_fused", "attn_dkdv", "attn_dq", "loss_rows", "loss_sum", "ref_fwd", "ref_bwd",
                "attn_plan", "attn_reduce", "loss_bwd", "rope", "part_gather", "part_scatter", "conv_fwd", "conv_bwd", "conv_fix", "gdn_prepare", "gdn_scan",
                "gdn_bwd_fscan", "gdn_bwd_rscan", "gdn_bwd_finish", "rope_axes", "entropy_rows", "entropy_join", "entropy_bwd",
                "scan_carry", "scan_states", "scan_out", "scan_grads", "scan_sums", "scan_step", "conv_step")


class _KernelTimes(ctypes.Structure):
    _fields_ = [("ms", ctypes.c_double * len(KERNEL_NAMES)), ("launches", ctypes.c_int64 * len(KERNEL_NAMES))]


def kernel_timing_enable(on: bool) -> None:
    """Bracket every kernel launch with HIP events on its stream (resets the totals)."""
    _check(_lib().tt_kernel_timing_enable(1 if on else 0))


def kernel_timing_read() -> dict:
    """Blocks until the recorded events completed; {kernel: (total_ms, launches)} since enable."""
    out = _KernelTimes()
    _check(_lib().tt_kernel_timing_read(ctypes.byref(out)))
    return {n: (float(out.ms[i]), int(out.launches[i])) for i, n in enumerate(KERNEL_NAMES)}


def last_error() -> str:
    return _lib().tt_last_error().decode()


def version() -> int:
    return int(_lib().tt_version())


def _check(status: int) -> None:
    if status != 0:
        raise TreeTrainError(status, last_error())


def _np(a, dtype):
    return None if a is None else np.ascontiguousarray(a, dtype=dtype)


def _hp(a: Optional[np.ndarray]):
    return None if a is None else a.ctypes.data_as(_vp)


@dataclass
class TreeMeta:
    n_nodes: int
    n_tokens: int
    n_leaves: int
    n_roots: int
    n_prefix: int
    n_ktiles: int
    dfs_order: np.ndarray
    node_start: np.ndarray
    node_end: np.ndarray
    subtree_end: np.ndarray
    node_parent: np.ndarray
    node_g: np.ndarray
    tok_node: np.ndarray
    tok_pos: np.ndarray
    tok_pred: np.ndarray
    tok_weight: np.ndarray
    kend: np.ndarray
    ktile_kend_min: np.ndarray
    ktile_kend_max: np.ndarray


def tree_meta_sizes(parent, seg_len, n_prefix: int = 0) -> dict:
    parent, seg_len = _np(parent, np.int32), _np(seg_len, np.int32)
    out = _MetaSizes()
    _check(_lib().tt_tree_meta_sizes(len(parent), _hp(parent), _hp(seg_len), n_prefix, ctypes.byref(out)))
    return {k: getattr(out, k) for k, _ in _MetaSizes._fields_}


def tree_build_meta(parent, seg_len, trained=None, root_pos_offset=None, g_override=None,
                    K_override: int = 0, n_prefix: int = 0, prefix_visible=None) -> TreeMeta:
    parent, seg_len = _np(parent, np.int32), _np(seg_len, np.int32)
    if parent.shape != seg_len.shape or parent.ndim != 1:
        raise ValueError("parent and seg_len must be 1-D arrays of equal length")
    trained = _np(trained, np.uint8)
    root_pos_offset = _np(root_pos_offset, np.int32)
    g_override = _np(g_override, np.int32)
    prefix_visible = _np(prefix_visible, np.uint8)
    for name, arr, n in (("trained", trained, len(parent)), ("g_override", g_override, len(parent)),
                         ("prefix_visible", prefix_visible, n_prefix)):
        if arr is not None and arr.shape != (n,):
            raise ValueError(f"{name} must have shape ({n},)")
    sz = tree_meta_sizes(parent, seg_len, n_prefix)
    if root_pos_offset is not None and root_pos_offset.shape != (sz["n_roots"],):
        raise ValueError(f"root_pos_offset must have one entry per root ({sz['n_roots']})")
    nn, nt, nk = sz["n_nodes"], sz["n_tokens"], sz["n_ktiles"]
    i32 = lambda n: np.zeros(n, dtype=np.int32)
    m = TreeMeta(nn, nt, sz["n_leaves"], sz["n_roots"], n_prefix, nk,
                 i32(nn), i32(nn), i32(nn), i32(nn), i32(nn), i32(nn), i32(nt), i32(nt), i32(nt),
                 np.zeros(nt, dtype=np.float32), i32(n_prefix + nt), i32(nk), i32(nk))
    _check(_lib().tt_tree_build_meta(
        nn, _hp(parent), _hp(seg_len), _hp(trained), _hp(root_pos_offset), _hp(g_override), K_override,
        n_prefix, _hp(prefix_visible),
        _hp(m.dfs_order), _hp(m.node_start), _hp(m.node_end), _hp(m.subtree_end), _hp(m.node_parent),
        _hp(m.node_g), _hp(m.tok_node), _hp(m.tok_pos), _hp(m.tok_pred), _hp(m.tok_weight),
        _hp(m.kend), _hp(m.ktile_kend_min), _hp(m.ktile_kend_max)))
    return m


WEIGHT_PATH_SUM, WEIGHT_UNIFORM, WEIGHT_PATH_TOKEN_MEAN = 0, 1, 2


@dataclass
class ConvPlan:
    """Host output of tt_tree_conv_plan: tokens with successors that do not directly follow them."""
    kernel_size: int
    fix_tok: np.ndarray
    fix_off: np.ndarray
    fix_t: np.ndarray
    fix_r: np.ndarray
    device: Optional[dict] = None

    def to_device(self, device="cuda"):
        torch = _torch()
        self.device = {n: torch.from_numpy(getattr(self, n)).to(device) for n in ("fix_tok", "fix_off", "fix_t", "fix_r")}
        return self


GDN_CHUNK = 64


class _ScanDesc(ctypes.Structure):
    _fields_ = [("n_tokens", ctypes.c_int64), ("channels", ctypes.c_int32), ("n_state", ctypes.c_int32), ("groups", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("softplus", ctypes.c_int32)] + \
               [(f"{name}_stride_tok", ctypes.c_int64) for name in ("x", "dt", "z", "b", "c", "y")]


class _ScanChunks(ctypes.Structure):
    _fields_ = [("n_chunks", ctypes.c_int32), ("n_slots", ctypes.c_int32)] + \
               [(name, _vp) for name in ("chunk_tok0", "chunk_len", "chunk_src", "chunk_dst", "chunk_cap", "chunk_order")] + \
               [("n_capture", ctypes.c_int32)]


class _GdnSchedule(ctypes.Structure):
    _fields_ = [("n_segments", ctypes.c_int32), ("n_levels", ctypes.c_int32), ("level_off", ctypes.c_void_p),
                ("seg_chunk0", ctypes.c_void_p), ("seg_chunk1", ctypes.c_void_p), ("slot_cons_off", ctypes.c_void_p),
                ("slot_cons", ctypes.c_void_p)]


def _sched_ref(plan):
    sc = plan._schedule()
    return None if sc is None else ctypes.byref(sc)


@dataclass
class GdnPlan:
    """Host output of tt_tree_gdn_plan: the chunk program of the gated delta rule and of the selective scan.  The device calls read copies of it
    that belong to the plan: a graph that holds such a call needs the plan as long as it is replayed."""
    n_chunks: int
    n_slots: int
    chunk_tok0: np.ndarray
    chunk_len: np.ndarray
    chunk_src: np.ndarray
    chunk_dst: np.ndarray
    chunk_cap: np.ndarray
    n_capture: int = 0
    device: Optional[dict] = None
    # tt_tree_gdn_schedule: segments of the chunk program by dependency level (sibling subtrees side by side)
    seg_chunk0: Optional[np.ndarray] = None
    seg_chunk1: Optional[np.ndarray] = None
    level_off: Optional[np.ndarray] = None
    slot_cons_off: Optional[np.ndarray] = None
    slot_cons: Optional[np.ndarray] = None
    parallel: bool = True          # False: the device calls walk all chunks in sequence order (for cross-checks)
    scan_programs = None           # (no field) the scan's programs, by channels and direction, on the host and on devices; a copy has its own

    def __getstate__(self):
        return {**self.__dict__, "scan_programs": None}

    @property
    def n_segments(self) -> int:
        return 0 if self.seg_chunk0 is None else len(self.seg_chunk0)

    @property
    def n_levels(self) -> int:
        return 0 if self.level_off is None else len(self.level_off) - 1

    def to_device(self, device="cuda"):
        torch = _torch()
        names = ["chunk_tok0", "chunk_len", "chunk_src", "chunk_dst", "chunk_cap"]
        if self.seg_chunk0 is not None:
            names += ["seg_chunk0", "seg_chunk1", "slot_cons_off", "slot_cons"]
        self.device = {n: torch.from_numpy(getattr(self, n)).to(device) for n in names}
        return self

    def _scan_program(self, channels: int, backward: bool):
        """tt_tree_scan_program for the scan with this many channels, [5, pieces] int32.  Laid out once per number of channels."""
        if self.scan_programs is None:
            self.scan_programs = {}
        prog = self.scan_programs.get((channels, backward))
        if prog is None:
            f, n = _lib().tt_tree_scan_program, ctypes.c_int32(0)
            given = [_hp(a) for a in (self.chunk_tok0, self.chunk_len, self.chunk_src, self.chunk_dst, self.chunk_cap)]
            _check(f(self.n_chunks, *given, channels, int(backward), ctypes.byref(n), *[None] * 5))
            prog = np.zeros((5, n.value), np.int32)
            _check(f(self.n_chunks, *given, channels, int(backward), ctypes.byref(n), *(_hp(a) for a in prog)))
            self.scan_programs[(channels, backward)] = prog
        return prog

    def _scan_chunks(self, channels: int, backward: bool, device, captured: bool):
        """ctypes tt_scan_chunks of that program on `device`, for a call on the current stream."""
        prog = self._scan_program(channels, backward)
        key = (channels, backward, device)
        on_device = self.scan_programs.get(key)
        if on_device is None:
            if _torch().cuda.is_current_stream_capturing():
                raise RuntimeError("the first scan call of a plan with this many channels copies its program: make it before the capture")
            longest_first = np.argsort(-prog[1], kind="stable").astype(np.int32)      # (the last to end are short)
            packed = _torch().from_numpy(np.concatenate([prog, longest_first[None]])).to(device)
            rows, n = [packed[i].data_ptr() for i in range(6)], prog.shape[1]
            on_device = self.scan_programs[key] = (packed, _ScanChunks(n, self.n_slots, *rows[:4], None, rows[5]),
                                                   _ScanChunks(n, self.n_slots, *rows, self.n_capture), _stream_ptr(None))
        if _stream_ptr(None) != on_device[3]:        # not reused, once the plan is dropped, before this stream is through with it
            on_device[0].record_stream(_torch().cuda.current_stream())
        return on_device[2 if captured else 1]

    def _schedule(self):
        """ctypes tt_gdn_schedule for the device calls, or None (sequential walk)."""
        if not self.parallel or self.seg_chunk0 is None or self.device is None or "seg_chunk0" not in self.device:
            return None
        d = self.device
        return _GdnSchedule(self.n_segments, self.n_levels, _hp(self.level_off), ctypes.c_void_p(d["seg_chunk0"].data_ptr()),
                            ctypes.c_void_p(d["seg_chunk1"].data_ptr()), ctypes.c_void_p(d["slot_cons_off"].data_ptr()),
                            ctypes.c_void_p(d["slot_cons"].data_ptr()) if len(self.slot_cons) else None)


def tree_gdn_plan(parent, seg_len, capture_nodes=()) -> GdnPlan:
    parent, seg_len = _np(parent, np.int32), _np(seg_len, np.int32)
    if len(parent) != len(seg_len):
        raise ValueError("parent and seg_len differ in length")
    nc, ns = ctypes.c_int32(0), ctypes.c_int32(0)
    _check(_lib().tt_tree_gdn_plan_sizes(len(parent), _hp(parent), _hp(seg_len), ctypes.byref(nc), ctypes.byref(ns)))
    arrs = [np.zeros(nc.value, np.int32) for _ in range(5)]
    cap = _np(list(capture_nodes), np.int32)
    _check(_lib().tt_tree_gdn_plan(len(parent), _hp(parent), _hp(seg_len), len(cap), _hp(cap), *(_hp(a) for a in arrs)))
    plan = GdnPlan(nc.value, ns.value, *arrs, n_capture=len(cap))
    nseg, nlev, ncons = ctypes.c_int32(0), ctypes.c_int32(0), ctypes.c_int32(0)
    _check(_lib().tt_tree_gdn_schedule_sizes(plan.n_chunks, _hp(plan.chunk_src), _hp(plan.chunk_dst), plan.n_slots,
                                             ctypes.byref(nseg), ctypes.byref(nlev), ctypes.byref(ncons)))
    plan.seg_chunk0, plan.seg_chunk1 = np.zeros(nseg.value, np.int32), np.zeros(nseg.value, np.int32)
    plan.level_off = np.zeros(nlev.value + 1, np.int32)
    plan.slot_cons_off, plan.slot_cons = np.zeros(plan.n_slots + 1, np.int32), np.zeros(ncons.value, np.int32)
    _check(_lib().tt_tree_gdn_schedule(plan.n_chunks, _hp(plan.chunk_src), _hp(plan.chunk_dst), plan.n_slots, _hp(plan.seg_chunk0),
                                       _hp(plan.seg_chunk1), _hp(plan.level_off), _hp(plan.slot_cons_off), _hp(plan.slot_cons)))
    return plan


def tree_conv_plan(tok_pred, kernel_size: int) -> ConvPlan:
    tok_pred = _np(tok_pred, np.int32)
    nf, npairs = ctypes.c_int32(0), ctypes.c_int32(0)
    _check(_lib().tt_tree_conv_plan_sizes(len(tok_pred), _hp(tok_pred), int(kernel_size), ctypes.byref(nf), ctypes.byref(npairs)))
    fix_tok, fix_off = np.zeros(nf.value, np.int32), np.zeros(nf.value + 1, np.int32)
    fix_t, fix_r = np.zeros(npairs.value, np.int32), np.zeros(npairs.value, np.int32)
    _check(_lib().tt_tree_conv_plan(len(tok_pred), _hp(tok_pred), int(kernel_size), _hp(fix_tok), _hp(fix_off), _hp(fix_t), _hp(fix_r)))
    return ConvPlan(int(kernel_size), fix_tok, fix_off, fix_t, fix_r)


def tree_path_weights(parent, seg_len, trained=None, *, scheme: int = WEIGHT_PATH_SUM, path_weight=None, advantage=None):
    """General loss weights lambda_t = sum of path weights over the paths through t (host).
    Returns (tok_weight [n_tokens] fp32, leaf_node [n_leaves] int32: the leaf of path k)."""
    parent, seg_len = _np(parent, np.int32), _np(seg_len, np.int32)
    if len(parent) != len(seg_len):
        raise ValueError("parent and seg_len differ in length")
    trained = _np(trained, np.uint8)
    sz = tree_meta_sizes(parent, seg_len)
    path_weight, advantage = _np(path_weight, np.float32), _np(advantage, np.float32)
    if path_weight is not None and len(path_weight) != sz["n_leaves"]:
        raise ValueError(f"path_weight has {len(path_weight)} entries for {sz['n_leaves']} paths")
    if advantage is not None and len(advantage) != sz["n_tokens"]:
        raise ValueError("advantage must have one entry per token")
    w = np.zeros(sz["n_tokens"], np.float32)
    leaf = np.zeros(sz["n_leaves"], np.int32)
    _check(_lib().tt_tree_path_weights(len(parent), _hp(parent), _hp(seg_len), _hp(trained), int(scheme), _hp(path_weight),
                                       _hp(advantage), _hp(w), _hp(leaf)))
    return w, leaf


@dataclass
class PartitionPlan:
    """Outputs of tt_tree_partition_plan (numpy, host).  `device` holds torch copies of the five arrays the
    device driver reads, once to_device() was called."""
    n_parts: int
    n_tokens: int
    capacity: int
    max_part_tokens: int
    max_prefix: int
    part_of_node: np.ndarray
    part_node_off: np.ndarray
    part_nodes: np.ndarray
    part_parent: np.ndarray
    part_cut_node: np.ndarray
    part_pos_offset: np.ndarray
    part_tok_off: np.ndarray
    own_tok: np.ndarray
    part_prefix_off: np.ndarray
    prefix_tok: np.ndarray
    prefix_visible: np.ndarray
    kend: np.ndarray
    part_ktile_off: np.ndarray
    kt_min: np.ndarray
    kt_max: np.ndarray
    part_own_start: np.ndarray
    part_prefix_start: np.ndarray
    device: Optional[dict] = None
    in_place: bool = True          # False: the driver gathers every partition (for cross-checks)

    def to_device(self, device="cuda"):
        torch = _torch()
        self.device = {name: torch.from_numpy(getattr(self, name)).to(device)
                       for name in ("own_tok", "prefix_tok", "kend", "kt_min", "kt_max")}
        return self

    def _c(self) -> _PartitionPlan:
        if self.device is None:
            raise ValueError("call to_device() on the plan first")
        d = self.device
        return _PartitionPlan(self.n_parts, self.n_tokens, _hp(self.part_tok_off), _hp(self.part_prefix_off),
                              _hp(self.part_ktile_off), _hp(self.part_own_start) if self.in_place else None,
                              _hp(self.part_prefix_start) if self.in_place else None, *(ctypes.c_void_p(d[n].data_ptr()) for n in
                                                         ("own_tok", "prefix_tok", "kend", "kt_min", "kt_max")))


def tree_partition_sizes(parent, seg_len, capacity: int) -> dict:
    parent, seg_len = _np(parent, np.int32), _np(seg_len, np.int32)
    out = _PartitionSizes()
    _check(_lib().tt_tree_partition_sizes(len(parent), _hp(parent), _hp(seg_len), int(capacity), ctypes.byref(out)))
    return {f: int(getattr(out, f)) for f, _ in _PartitionSizes._fields_}


def tree_partition_plan(parent, seg_len, capacity: int) -> PartitionPlan:
    """Cuts the tree into partitions of at most `capacity` tokens and lays out everything the partitioned
    attention calls need (host only)."""
    parent, seg_len = _np(parent, np.int32), _np(seg_len, np.int32)
    if len(parent) != len(seg_len):
        raise ValueError("parent and seg_len differ in length")
    sz = tree_partition_sizes(parent, seg_len, capacity)
    n, npart, ntok = len(parent), sz["n_parts"], sz["n_tokens"]
    arr = dict(
        part_of_node=np.zeros(n, np.int32), part_node_off=np.zeros(npart + 1, np.int32), part_nodes=np.zeros(n, np.int32),
        part_parent=np.zeros(npart, np.int32), part_cut_node=np.zeros(npart, np.int32),
        part_pos_offset=np.zeros(npart, np.int32), part_tok_off=np.zeros(npart + 1, np.int32),
        own_tok=np.zeros(ntok, np.int32), part_prefix_off=np.zeros(npart + 1, np.int64),
        prefix_tok=np.zeros(sz["sum_prefix"], np.int32), prefix_visible=np.zeros(sz["sum_prefix"], np.uint8),
        kend=np.zeros(sz["sum_prefix"] + ntok, np.int32), part_ktile_off=np.zeros(npart + 1, np.int64),
        kt_min=np.zeros(sz["sum_ktiles"], np.int32), kt_max=np.zeros(sz["sum_ktiles"], np.int32),
        part_own_start=np.zeros(npart, np.int32), part_prefix_start=np.zeros(npart, np.int32))
    _check(_lib().tt_tree_partition_plan(n, _hp(parent), _hp(seg_len), int(capacity), *(_hp(a) for a in arr.values())))
    return PartitionPlan(n_parts=npart, n_tokens=ntok, capacity=int(capacity), max_part_tokens=sz["max_part_tokens"],
                         max_prefix=sz["max_prefix"], **arr)


# ---- device calls -----------------------------------------------------------------------------

# The small calls are bound by the time the host takes to make them (a forward over 256 tokens ran 13 us on the GPU and
# 19 us here), so what every call does is kept short: pointers and streams are passed as plain integers, the current stream
# is asked for without building a Stream object, shapes and strides are fetched once per tensor.
_TORCH = None


def _torch():
    global _TORCH
    if _TORCH is None:
        import torch
        _TORCH = torch
    return _TORCH


def _dp(t):
    return None if t is None else t.data_ptr()


def _current_device() -> int:
    torch = _torch()
    device = getattr(torch._C, "_cuda_getDevice", None)                 # private names, here and below: not every version has to
    return torch.cuda.current_device() if device is None else device()  # have them (what torch.cuda does around them costs 0.6 us)


def _stream_ptr(stream):
    if stream is not None:
        return stream.cuda_stream
    torch = _torch()
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return torch.cuda.current_stream().cuda_stream if raw is None else raw(_current_device())


def _desc(q, k, v, n_prefix: int, scale, reference_kernels: bool) -> _AttnDesc:
    torch = _torch()
    qs, ks, vs = q.shape, k.shape, v.shape
    if len(qs) != 3 or len(ks) != 3 or len(vs) != 3:
        raise ValueError("q, k, v must be [tokens, heads, d]")
    dtype = q.dtype
    if dtype not in (torch.bfloat16, torch.float32) or k.dtype != dtype or v.dtype != dtype:
        raise ValueError("q, k, v must share dtype bf16 or fp32")
    row = []
    for t, (n, heads, dim) in ((q, qs), (k, ks), (v, vs)):
        st = t.stride()
        if n and heads and dim and (st[2] != 1 or st[1] != dim):
            raise ValueError("heads and d must be contiguous (only the token stride is free)")
        row.append(st[0] if n > 1 else heads * dim)
    n_q, hq, d = qs
    if ks[0] != n_q or vs != ks or ks[2] != d:
        raise ValueError("k, v must be [n_q, hkv, d]")
    return _AttnDesc(n_q, n_prefix, hq, ks[1], d, DTYPE_BF16 if dtype == torch.bfloat16 else DTYPE_FP32,
                     float(d) ** -0.5 if scale is None else float(scale),
                     FLAG_REFERENCE_KERNELS if reference_kernels else 0, *row)


def tree_attn_workspace(q, k, v, n_prefix: int = 0, backward: bool = False, scale=None,
                        reference_kernels: bool = False) -> int:
    d = _desc(q, k, v, n_prefix, scale, reference_kernels)
    return int(_lib().tt_tree_attn_workspace(ctypes.byref(d), 1 if backward else 0))


def _workspace(desc, backward, workspace, device):
    torch = _torch()
    need = int(_lib().tt_tree_attn_workspace(ctypes.byref(desc), 1 if backward else 0))
    if workspace is None:
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=device)
    return workspace, workspace.numel() * workspace.element_size()


I32_MAX = 2 ** 31 - 1        # what the library's sizes hold (ctypes would pass the lower bits of a larger one)


def _check_tensor(t, name, shape, dtype):
    """A contiguous tensor of exactly this shape and dtype."""
    if t.shape != shape or t.dtype is not dtype or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {shape}")


def _check_rows(t, name, shape, dtypes):
    """Rows of contiguous elements with a free stride between them (one of the dtypes); returns that stride in elements."""
    if t.shape != shape or t.dtype not in dtypes:
        raise ValueError(f"{name} must be {shape} of {' / '.join(str(d) for d in dtypes)}")
    width = shape[1] if len(shape) == 2 else shape[1] * shape[2]
    if width > I32_MAX:
        raise ValueError(f"the rows of {name} hold at most {I32_MAX} elements, not {width}")
    if t.is_contiguous():
        return width
    step = t.stride()
    row = 1
    for i in range(len(shape) - 1, 0, -1):
        if shape[i] > 1 and step[i] != row:
            raise ValueError(f"the rows of {name} must be contiguous (only the stride between them is free)")
        row *= shape[i]
    if shape[0] <= 1:
        return width
    if step[0] < width:
        raise ValueError(f"the rows of {name} overlap")
    return step[0]


def _enter_device(*tensors):
    """Makes the tensors' device, which must be one and the same GPU, the current one.  Returns what _leave_device wants."""
    dev = tensors[0].get_device()
    for t in tensors:
        if t is not None and t.get_device() != dev:
            raise ValueError(f"tensors on {tensors[0].device} and {t.device} in one call")
    if dev < 0:
        raise ValueError("the tensors must be on the GPU")
    before = _current_device()
    if before == dev:
        return None
    _torch().cuda.set_device(dev)
    return before


def _new(like, shape, dtype=None):
    """An empty tensor on the device of `like` (and of its dtype)."""
    if dtype is not None:
        return like.new_empty(shape, dtype=dtype)
    if like.shape == shape and like.is_contiguous():
        return _TORCH.empty_like(like)                    # the quickest of the three
    return like.new_empty(shape)


def _on_stream(stream, call, arguments):
    """call(**arguments) with the `stream` among them as the current one, so that what the call allocates is that stream's memory.  (Memory
    of the stream that is current now may just have been dropped by work that is still queued there, and nothing orders the call behind
    that work.)  What is returned is not handed out again, once dropped, before the stream that is current now is through with it."""
    torch = _torch()
    del arguments["stream"]
    for t in arguments.values():
        if isinstance(t, torch.Tensor) and t.get_device() != stream.device_index:
            raise ValueError(f"a tensor on {t.device} in a call on a stream of cuda:{stream.device_index}")
    here = torch.cuda.current_stream(stream.device_index)
    with torch.cuda.stream(stream):
        out = call(**arguments)
    for t in out if isinstance(out, tuple) else (out,):
        if t is not None:
            t.record_stream(here)
    return out


def _leave_device(before):
    if before is not None:
        _torch().cuda.set_device(before)


def tree_attn_fwd(q, k, v, kend, kt_min, kt_max, *, k_prefix=None, v_prefix=None, scale=None,
                  o=None, lse=None, workspace=None, stream=None, reference_kernels: bool = False):
    """q [N,hq,d]; k, v [N,hkv,d]; kend/kt_min/kt_max: int32 device tensors from tree_build_meta.
    Returns (o [N,hq,d], lse [hq,N] fp32)."""
    if stream is not None:
        return _on_stream(stream, tree_attn_fwd, locals())
    torch = _torch()
    n_prefix = 0 if k_prefix is None else k_prefix.shape[0]
    desc = _desc(q, k, v, n_prefix, scale, reference_kernels)
    if k_prefix is not None:
        k_prefix, v_prefix = k_prefix.contiguous(), v_prefix.contiguous()
    if o is None:
        o = torch.empty((desc.n_q, desc.hq, desc.d), dtype=q.dtype, device=q.device)
    if lse is None:
        lse = torch.empty((desc.hq, desc.n_q), dtype=torch.float32, device=q.device)
    workspace, ws_bytes = _workspace(desc, False, workspace, q.device)
    _check(_lib().tt_tree_attn_fwd(ctypes.byref(desc), _dp(q), _dp(k), _dp(v), _dp(k_prefix), _dp(v_prefix),
                                   _dp(kend), _dp(kt_min), _dp(kt_max), _dp(o), _dp(lse),
                                   _dp(workspace), ws_bytes, _stream_ptr(None)))
    return o, lse


def tree_attn_bwd(q, k, v, kend, kt_min, kt_max, o, d_o, lse, *, k_prefix=None, v_prefix=None,
                  dk_prefix_acc=None, dv_prefix_acc=None, scale=None, dq=None, dk=None, dv=None,
                  workspace=None, stream=None, reference_kernels: bool = False):
    """Returns (dq [N,hq,d], dk [N,hkv,d], dv [N,hkv,d]); prefix gradients are added into the fp32
    accumulators dk_prefix_acc / dv_prefix_acc [P,hkv,d]."""
    if stream is not None:
        return _on_stream(stream, tree_attn_bwd, locals())
    torch = _torch()
    n_prefix = 0 if k_prefix is None else k_prefix.shape[0]
    desc = _desc(q, k, v, n_prefix, scale, reference_kernels)
    if k_prefix is not None:
        k_prefix, v_prefix = k_prefix.contiguous(), v_prefix.contiguous()
    if not (o.is_contiguous() and d_o.is_contiguous() and lse.is_contiguous()):
        raise ValueError("o, d_o, lse must be contiguous")
    if dq is None:
        dq = torch.empty((desc.n_q, desc.hq, desc.d), dtype=q.dtype, device=q.device)
    if dk is None:
        dk = torch.empty((desc.n_q, desc.hkv, desc.d), dtype=q.dtype, device=q.device)
    if dv is None:
        dv = torch.empty((desc.n_q, desc.hkv, desc.d), dtype=q.dtype, device=q.device)
    workspace, ws_bytes = _workspace(desc, True, workspace, q.device)
    _check(_lib().tt_tree_attn_bwd(ctypes.byref(desc), _dp(q), _dp(k), _dp(v), _dp(k_prefix), _dp(v_prefix),
                                   _dp(kend), _dp(kt_min), _dp(kt_max), _dp(o), _dp(d_o), _dp(lse),
                                   _dp(dq), _dp(dk), _dp(dv), _dp(dk_prefix_acc), _dp(dv_prefix_acc),
                                   _dp(workspace), ws_bytes, _stream_ptr(None)))
    return dq, dk, dv


def tree_weighted_logprob(logits, target, weight=None, *, loss_acc=None, logp=None, lse=None,
                          want_lse: bool = True, stream=None):
    """logits [n, V] bf16/fp32 (row stride free), target [n] int32, weight [n] fp32 or None.
    Returns (logp [n], lse [n] or None, loss_acc [1]); loss_acc is added to (zeroed if created here)."""
    if stream is not None:
        return _on_stream(stream, tree_weighted_logprob, locals())
    torch = _torch()
    if logits.dim() != 2 or logits.stride(1) != 1:
        raise ValueError("logits must be [rows, vocab] with contiguous vocab")
    if logits.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("logits must be bf16 or fp32")
    n, vocab = logits.shape
    if logp is None:
        logp = torch.empty(n, dtype=torch.float32, device=logits.device)
    if lse is None and want_lse:
        lse = torch.empty(n, dtype=torch.float32, device=logits.device)
    if loss_acc is None:
        loss_acc = torch.zeros(1, dtype=torch.float32, device=logits.device)
    _check(_lib().tt_tree_weighted_logprob(
        n, vocab, DTYPE_BF16 if logits.dtype == torch.bfloat16 else DTYPE_FP32, _dp(logits),
        logits.stride(0) if n > 1 else vocab, _dp(target), _dp(weight), _dp(logp), _dp(lse), _dp(loss_acc),
        _stream_ptr(None)))
    return logp, lse, loss_acc


def tree_rope(x, tok_pos, *, theta_base: float = 1.0e6, inverse: bool = False, out=None, stream=None):
    """Rotary embedding of x [n, heads, d] (bf16/fp32, heads and d contiguous, free token stride) with the
    tree position ids tok_pos [n] int32; `inverse` undoes it / is its backward.  `out` may be x (in place)."""
    if stream is not None:
        return _on_stream(stream, tree_rope, locals())
    torch = _torch()
    if x.dim() != 3 or x.stride(2) != 1 or (x.shape[1] > 1 and x.stride(1) != x.shape[2]):
        raise ValueError("x must be [tokens, heads, d] with heads and d contiguous")
    if x.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("x must be bf16 or fp32")
    n, h, d = x.shape
    if out is None:
        out = torch.empty((n, h, d), dtype=x.dtype, device=x.device)
    if out.shape != x.shape or out.dtype != x.dtype or out.stride(2) != 1 or (h > 1 and out.stride(1) != d):
        raise ValueError("out must match x in shape and dtype, heads and d contiguous")
    _check(_lib().tt_tree_rope(n, h, d, DTYPE_BF16 if x.dtype == torch.bfloat16 else DTYPE_FP32, _dp(x),
                               x.stride(0) if n > 1 else h * d, _dp(tok_pos), float(theta_base), 1 if inverse else 0,
                               _dp(out), out.stride(0) if n > 1 else h * d, _stream_ptr(None)))
    return out


@functools.lru_cache(maxsize=64)
def _pair_axis(sections: tuple, n_axes: int, half: int, interleaved: bool) -> bytes:
    if len(sections) != n_axes or min(sections) < 0 or sum(sections) != half:
        raise ValueError(f"sections must hold one non-negative count per axis ({n_axes}), {half} pairs together")
    if not interleaved:
        return bytes(a for a, s in enumerate(sections) for _ in range(s))
    return bytes(i % n_axes if i // n_axes < sections[i % n_axes] else 0 for i in range(half))


def tree_rope_axes(x, axis_pos, sections, *, interleaved: bool = False, theta_base: float = 1.0e6, inverse: bool = False, out=None,
                   stream=None):
    """tree_rope with a position per axis (time, height, width): x [n, heads, d] bf16/fp32 (heads and d contiguous, free token
    stride), axis_pos [n_axes, n] int32, 1 to 4 axes.  sections: pairs of every axis, d/2 together; the first axis has the first
    pairs and so on or, interleaved, pair i belongs to axis i % n_axes while that axis has had fewer pairs than its section, and
    to the first axis otherwise.  `inverse` undoes the rotation / is its backward; `out` may be x (in place)."""
    if stream is not None:
        return _on_stream(stream, tree_rope_axes, locals())
    torch = _torch()
    if x.dim() != 3 or axis_pos.dim() != 2:
        raise ValueError("x must be [tokens, heads, d], axis_pos [axes, tokens]")
    n, h, d = x.shape
    stride = _check_rows(x, "x", (n, h, d), (torch.bfloat16, torch.float32))
    n_axes = axis_pos.shape[0]
    _check_tensor(axis_pos, "axis_pos", (n_axes, n), torch.int32)
    if not 1 <= n_axes <= 4:
        raise ValueError("axis_pos must have 1 to 4 axes")
    if d % 2:
        raise ValueError("d must be even")
    pair_axis = _pair_axis(tuple(sections), n_axes, d // 2, bool(interleaved))
    out_stride = h * d
    if out is not None:
        out_stride = _check_rows(out, "out", (n, h, d), (x.dtype,))
    before = _enter_device(x, axis_pos, out)
    try:
        if out is None:
            out = _new(x, (n, h, d))
        _check(_lib().tt_tree_rope_axes(n, h, d, DTYPE_BF16 if x.dtype == torch.bfloat16 else DTYPE_FP32, _dp(x), stride, n_axes,
                                        _dp(axis_pos), pair_axis, float(theta_base), 1 if inverse else 0, _dp(out), out_stride,
                                        _stream_ptr(None)))
    finally:
        _leave_device(before)
    return out


def tree_axis_positions(parent, seg_len, grid=None, root_pos_offset=None) -> np.ndarray:
    """Positions [3, n_tokens] (time, height, width) in DFS order of a tree of text and image nodes (host).  grid [n_nodes, 3]:
    T, H, W of the nodes that hold images (T * H * W tokens, row by row inside a frame), zeros for text; a node starts behind the
    largest position of its parent.  root_pos_offset: one entry per root, in ascending id."""
    parent, seg_len = _np(parent, np.int32), _np(seg_len, np.int32)
    if parent.shape != seg_len.shape or parent.ndim != 1:
        raise ValueError("parent and seg_len must be 1-D arrays of equal length")
    grid, root_pos_offset = _np(grid, np.int32), _np(root_pos_offset, np.int32)
    if grid is not None and grid.shape != (len(parent), 3):
        raise ValueError(f"grid must have shape ({len(parent)}, 3)")
    sz = tree_meta_sizes(parent, seg_len)
    if root_pos_offset is not None and root_pos_offset.shape != (sz["n_roots"],):
        raise ValueError(f"root_pos_offset must have one entry per root ({sz['n_roots']})")
    pos = np.zeros((3, sz["n_tokens"]), np.int32)
    _check(_lib().tt_tree_axis_positions(len(parent), _hp(parent), _hp(seg_len), _hp(grid), _hp(root_pos_offset), _hp(pos)))
    return pos


LOGPROB_TOP_MAX = 64


def _logits_dtype(logits) -> int:
    torch = _torch()
    if logits.dim() != 2:
        raise ValueError("logits must be [rows, vocab]")
    if logits.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("logits must be bf16 or fp32")
    return DTYPE_BF16 if logits.dtype == torch.bfloat16 else DTYPE_FP32


def tree_logprob_entropy_workspace(logits, top_k: int = 0) -> int:
    """Bytes of workspace of tree_logprob_entropy for these logits."""
    code, (n, vocab) = _logits_dtype(logits), logits.shape
    return _logprob_entropy_workspace(n, vocab, code, top_k)


def _logprob_entropy_workspace(n, vocab, code, top_k) -> int:
    small = 0 <= top_k <= LOGPROB_TOP_MAX and vocab <= I32_MAX
    need = _lib().tt_tree_logprob_entropy_workspace(n, vocab, code, int(top_k)) if small else 0
    if need == 0:
        raise ValueError(f"top_k={top_k} must lie in [0, min({LOGPROB_TOP_MAX}, vocab={vocab})], and the vocabulary in [1, 2^30]")
    return need


def tree_logprob_entropy(logits, target, *, top_k: int = 0, logp=None, entropy=None, lse=None, top_index=None, top_logp=None,
                         workspace=None, stream=None):
    """Per row of the logits [n, V] (bf16/fp32, row stride free), in one pass: the log-prob of target [n] int32, the entropy of
    the row's distribution, its log-sum-exp, and the top_k (at most 64) most probable entries.  Returns (logp [n], entropy [n],
    lse [n] fp32, top_index [n, top_k] int32, top_logp [n, top_k] fp32), the last two None when top_k is 0: indices by falling
    log-prob, the lowest index first among equals.  A row whose target lies outside [0, V) is ignored: logp and entropy are 0."""
    if stream is not None:
        return _on_stream(stream, tree_logprob_entropy, locals())
    torch = _torch()
    code, (n, vocab) = _logits_dtype(logits), logits.shape
    stride = _check_rows(logits, "logits", (n, vocab), (torch.bfloat16, torch.float32))
    _check_tensor(target, "target", (n,), torch.int32)
    top_k = int(top_k)
    need = _logprob_entropy_workspace(n, vocab, code, top_k)
    for name, t in (("logp", logp), ("entropy", entropy), ("lse", lse)):
        if t is not None:
            _check_tensor(t, name, (n,), torch.float32)
    if top_k == 0 and (top_index is not None or top_logp is not None):
        raise ValueError("top_index and top_logp need top_k > 0")
    if top_index is not None:
        _check_tensor(top_index, "top_index", (n, top_k), torch.int32)
    if top_logp is not None:
        _check_tensor(top_logp, "top_logp", (n, top_k), torch.float32)
    before = _enter_device(logits, target, logp, entropy, lse, top_index, top_logp, workspace)
    try:
        logp = _new(logits, (n,), torch.float32) if logp is None else logp
        entropy = _new(logp, (n,)) if entropy is None else entropy
        lse = _new(logp, (n,)) if lse is None else lse
        if top_k:
            top_logp = _new(logp, (n, top_k)) if top_logp is None else top_logp
            top_index = _new(top_logp, (n, top_k), torch.int32) if top_index is None else top_index
        if workspace is None:
            workspace = _new(logits, (need,), torch.uint8)
        _check(_lib().tt_tree_logprob_entropy(n, vocab, code, _dp(logits), stride, _dp(target), top_k, _dp(logp), _dp(entropy),
                                              _dp(lse), _dp(top_index), _dp(top_logp), _dp(workspace),
                                              workspace.numel() * workspace.element_size(), _stream_ptr(None)))
    finally:
        _leave_device(before)
    return logp, entropy, lse, top_index, top_logp


def tree_logprob_entropy_bwd(logits, target, lse, entropy, d_logp=None, d_entropy=None, *, out=None, stream=None):
    """Gradient of sum(d_logp * logp + d_entropy * entropy) with respect to the logits, in their dtype and shape; lse and entropy
    [n] are the ones tree_logprob_entropy returned, d_logp and d_entropy [n] fp32 (None = 0).  Rows whose target lies outside
    [0, V) get zero.  `out` may be the logits tensor itself (in place)."""
    if stream is not None:
        return _on_stream(stream, tree_logprob_entropy_bwd, locals())
    torch = _torch()
    code, (n, vocab) = _logits_dtype(logits), logits.shape
    stride = _check_rows(logits, "logits", (n, vocab), (torch.bfloat16, torch.float32))
    _check_tensor(target, "target", (n,), torch.int32)
    for name, t in (("lse", lse), ("entropy", entropy), ("d_logp", d_logp), ("d_entropy", d_entropy)):
        if t is not None:
            _check_tensor(t, name, (n,), torch.float32)
        elif not name.startswith("d_"):
            raise ValueError(f"{name} is required")
    out_stride = vocab
    if out is not None:
        out_stride = _check_rows(out, "out", (n, vocab), (logits.dtype,))
    before = _enter_device(logits, target, lse, entropy, d_logp, d_entropy, out)
    try:
        if out is None:
            out = _new(logits, (n, vocab))
        _check(_lib().tt_tree_logprob_entropy_bwd(n, vocab, code, _dp(logits), stride, _dp(target), _dp(lse), _dp(entropy),
                                                  _dp(d_logp), _dp(d_entropy), _dp(out), out_stride, _stream_ptr(None)))
    finally:
        _leave_device(before)
    return out


def tree_weighted_logprob_bwd(logits, target, weight, lse, *, grad_scale: float = 1.0, out=None, stream=None):
    """dlogits = grad_scale * weight * (softmax(logits) - onehot(target)), same dtype and shape as logits
    (zero rows where target < 0); lse [n] fp32 is the one tree_weighted_logprob returned.  `out` may be
    the logits tensor itself (in place)."""
    if stream is not None:
        return _on_stream(stream, tree_weighted_logprob_bwd, locals())
    torch = _torch()
    if logits.dim() != 2 or logits.stride(1) != 1:
        raise ValueError("logits must be [rows, vocab] with contiguous vocab")
    if logits.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("logits must be bf16 or fp32")
    n, vocab = logits.shape
    if out is None:
        out = torch.empty((n, vocab), dtype=logits.dtype, device=logits.device)
    if out.shape != logits.shape or out.dtype != logits.dtype or out.stride(1) != 1:
        raise ValueError("out must match logits in shape and dtype, with contiguous vocab")
    _check(_lib().tt_tree_weighted_logprob_bwd(
        n, vocab, DTYPE_BF16 if logits.dtype == torch.bfloat16 else DTYPE_FP32, _dp(logits),
        logits.stride(0) if n > 1 else vocab, _dp(target), _dp(weight), _dp(lse), float(grad_scale), _dp(out),
        out.stride(0) if n > 1 else vocab, _stream_ptr(None)))
    return out


def tree_weighted_logprob_fwd_bwd(logits, target, weight=None, *, grad_scale: float = 1.0, loss_acc=None, logp=None,
                                  lse=None, out=None, stream=None):
    """tree_weighted_logprob and tree_weighted_logprob_bwd in one pass over the logits.  Returns (logp [n], lse [n],
    loss_acc [1] (added to; zeroed if created here), dlogits like logits); `out` may be the logits tensor itself."""
    if stream is not None:
        return _on_stream(stream, tree_weighted_logprob_fwd_bwd, locals())
    torch = _torch()
    if logits.dim() != 2 or logits.stride(1) != 1:
        raise ValueError("logits must be [rows, vocab] with contiguous vocab")
    if logits.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("logits must be bf16 or fp32")
    n, vocab = logits.shape
    dev = logits.device
    if logp is None:
        logp = torch.empty(n, dtype=torch.float32, device=dev)
    if lse is None:
        lse = torch.empty(n, dtype=torch.float32, device=dev)
    if loss_acc is None:
        loss_acc = torch.zeros(1, dtype=torch.float32, device=dev)
    if out is None:
        out = torch.empty((n, vocab), dtype=logits.dtype, device=dev)
    if out.shape != logits.shape or out.dtype != logits.dtype or out.stride(1) != 1:
        raise ValueError("out must match logits in shape and dtype, with contiguous vocab")
    _check(_lib().tt_tree_weighted_logprob_fwd_bwd(
        n, vocab, DTYPE_BF16 if logits.dtype == torch.bfloat16 else DTYPE_FP32, _dp(logits),
        logits.stride(0) if n > 1 else vocab, _dp(target), _dp(weight), float(grad_scale), _dp(logp), _dp(lse), _dp(loss_acc),
        _dp(out), out.stride(0) if n > 1 else vocab, _stream_ptr(None)))
    return logp, lse, loss_acc, out


def tree_attn_partitioned_workspace(q, k, v, plan: PartitionPlan, backward: bool = False, scale=None,
                                    reference_kernels: bool = False) -> int:
    d = _desc(q, k, v, 0, scale, reference_kernels)
    c = plan._c()
    return int(_lib().tt_tree_attn_partitioned_workspace(ctypes.byref(d), ctypes.byref(c), 1 if backward else 0))


def _part_workspace(desc, cplan, backward, workspace, device):
    torch = _torch()
    need = int(_lib().tt_tree_attn_partitioned_workspace(ctypes.byref(desc), ctypes.byref(cplan), 1 if backward else 0))
    if need == 0:
        raise TreeTrainError(-2, last_error())
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=device)
    return workspace, workspace.numel() * workspace.element_size()


def tree_attn_partitioned_fwd(q, k, v, plan: PartitionPlan, *, scale=None, o=None, lse=None, workspace=None,
                              stream=None, reference_kernels: bool = False):
    """Whole-tree q [N,hq,d], k, v [N,hkv,d] in whole-tree DFS order; one attention pass per partition of
    `plan`.  Returns (o [N,hq,d], lse [hq,N])."""
    if stream is not None:
        return _on_stream(stream, tree_attn_partitioned_fwd, locals())
    torch = _torch()
    desc = _desc(q, k, v, 0, scale, reference_kernels)
    cplan = plan._c()
    if o is None:
        o = torch.empty((desc.n_q, desc.hq, desc.d), dtype=q.dtype, device=q.device)
    if lse is None:
        lse = torch.empty((desc.hq, desc.n_q), dtype=torch.float32, device=q.device)
    workspace, ws_bytes = _part_workspace(desc, cplan, False, workspace, q.device)
    _check(_lib().tt_tree_attn_partitioned_fwd(ctypes.byref(desc), ctypes.byref(cplan), _dp(q), _dp(k), _dp(v),
                                               _dp(o), _dp(lse), _dp(workspace), ws_bytes, _stream_ptr(None)))
    return o, lse


def tree_attn_partitioned_bwd(q, k, v, plan: PartitionPlan, o, d_o, lse, *, scale=None, dq=None, dk=None, dv=None,
                              workspace=None, stream=None, reference_kernels: bool = False):
    """Returns whole-tree (dq, dk, dv); cached-key gradients of all partitions are summed in fp32 inside."""
    if stream is not None:
        return _on_stream(stream, tree_attn_partitioned_bwd, locals())
    torch = _torch()
    desc = _desc(q, k, v, 0, scale, reference_kernels)
    cplan = plan._c()
    if not (o.is_contiguous() and d_o.is_contiguous() and lse.is_contiguous()):
        raise ValueError("o, d_o, lse must be contiguous")
    if dq is None:
        dq = torch.empty((desc.n_q, desc.hq, desc.d), dtype=q.dtype, device=q.device)
    if dk is None:
        dk = torch.empty((desc.n_q, desc.hkv, desc.d), dtype=q.dtype, device=q.device)
    if dv is None:
        dv = torch.empty((desc.n_q, desc.hkv, desc.d), dtype=q.dtype, device=q.device)
    workspace, ws_bytes = _part_workspace(desc, cplan, True, workspace, q.device)
    _check(_lib().tt_tree_attn_partitioned_bwd(ctypes.byref(desc), ctypes.byref(cplan), _dp(q), _dp(k), _dp(v),
                                               _dp(o), _dp(d_o), _dp(lse), _dp(dq), _dp(dk), _dp(dv),
                                               _dp(workspace), ws_bytes, _stream_ptr(None)))
    return dq, dk, dv


def _conv_check(x, weight, what="x"):
    torch = _torch()
    if x.dim() != 2 or x.stride(1) != 1:
        raise ValueError(f"{what} must be [tokens, channels] with contiguous channels")
    if x.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError(f"{what} must be bf16 or fp32")
    if weight.dim() != 2 or weight.shape[0] != x.shape[1] or weight.dtype != torch.float32 or not weight.is_contiguous():
        raise ValueError("weight must be a contiguous fp32 [channels, K] tensor")
    return x.shape[0], x.shape[1], weight.shape[1], DTYPE_BF16 if x.dtype == torch.bfloat16 else DTYPE_FP32


def _row_stride(t):
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def tree_conv_fwd(x, weight, bias, tok_pred, *, silu: bool = True, out=None, stream=None):
    """Tree-correct depthwise causal conv: x [n, C] bf16/fp32, weight [C, K] fp32, bias [C] fp32 or None,
    tok_pred [n] int32 (from tree_build_meta).  Returns y [n, C]."""
    if stream is not None:
        return _on_stream(stream, tree_conv_fwd, locals())
    torch = _torch()
    n, c, k, dt = _conv_check(x, weight)
    if out is None:
        out = torch.empty((n, c), dtype=x.dtype, device=x.device)
    _check(_lib().tt_tree_conv_fwd(n, c, k, dt, 1 if silu else 0, _dp(x), _row_stride(x), _dp(weight), _dp(bias), _dp(tok_pred),
                                   _dp(out), _row_stride(out), _stream_ptr(None)))
    return out


def tree_conv_bwd(x, weight, bias, tok_pred, dy, plan: ConvPlan, *, silu: bool = True, want_dbias: bool = True,
                  workspace=None, stream=None):
    """Returns (dx [n, C] in x's dtype, dweight [C, K] fp32, dbias [C] fp32 or None)."""
    if stream is not None:
        return _on_stream(stream, tree_conv_bwd, locals())
    torch = _torch()
    n, c, k, dt = _conv_check(x, weight)
    _conv_check(dy, weight, "dy")
    if plan.kernel_size != k:
        raise ValueError(f"the plan was made for kernel size {plan.kernel_size}, weight has {k}")
    if plan.device is None:
        plan.to_device(x.device)
    dx = torch.empty((n, c), dtype=x.dtype, device=x.device)
    dw = torch.empty((c, k), dtype=torch.float32, device=x.device)
    db = torch.empty(c, dtype=torch.float32, device=x.device) if want_dbias else None
    need = int(_lib().tt_tree_conv_bwd_workspace(n, c, k, dt))
    if workspace is None:
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=x.device)
    d = plan.device
    _check(_lib().tt_tree_conv_bwd(n, c, k, dt, 1 if silu else 0, _dp(x), _row_stride(x), _dp(weight), _dp(bias), _dp(tok_pred),
                                   _dp(dy), _row_stride(dy), len(plan.fix_tok), _dp(d["fix_tok"]), _dp(d["fix_off"]),
                                   _dp(d["fix_t"]), _dp(d["fix_r"]), _dp(dx), _row_stride(dx), _dp(dw), _dp(db),
                                   _dp(workspace), workspace.numel(), _stream_ptr(None)))
    return dx, dw, db


CONV_BWD_STATIC_SCRATCH_BYTES = 64 << 20


def tree_conv_bwd_static(x, weight, bias, tok_pred, dy, plan: ConvPlan, dx, dweight, dbias=None, *, silu: bool = True,
                         stream=None) -> None:
    """tree_conv_bwd for callers that may not allocate: every output is passed in (dx [n, C] in x's dtype,
    dweight [C, K] fp32, dbias [C] fp32 or None), the plan must already be on the device, and the scratch is the
    library's static array (shapes whose scratch exceeds CONV_BWD_STATIC_SCRATCH_BYTES are refused)."""
    if stream is not None:
        return _on_stream(stream, tree_conv_bwd_static, locals())
    n, c, k, dt = _conv_check(x, weight)
    _conv_check(dy, weight, "dy")
    if plan.kernel_size != k:
        raise ValueError(f"the plan was made for kernel size {plan.kernel_size}, weight has {k}")
    if plan.device is None:
        raise ValueError("move the plan to the device first (plan.to_device): this call does not allocate")
    if dx.shape != x.shape or dx.dtype != x.dtype or dweight.shape != weight.shape:
        raise ValueError("dx must match x, dweight must match weight")
    d = plan.device
    _check(_lib().tt_tree_conv_bwd_static(n, c, k, dt, 1 if silu else 0, _dp(x), _row_stride(x), _dp(weight), _dp(bias),
                                          _dp(tok_pred), _dp(dy), _row_stride(dy), len(plan.fix_tok), _dp(d["fix_tok"]),
                                          _dp(d["fix_off"]), _dp(d["fix_t"]), _dp(d["fix_r"]), _dp(dx), _row_stride(dx),
                                          _dp(dweight), _dp(dbias), _stream_ptr(None)))


def tree_gdn_fwd(q, k, v, g, beta, plan: GdnPlan, *, scale=None, out=None, workspace=None, stream=None,
                 initial_state=None, return_states: bool = False):
    """Gated delta rule with tree state routing: q, k [n, hk, 128], v [n, hv, 128] bf16 contiguous; g, beta
    [n, hv] fp32 (g = log decay <= 0).  Returns o [n, hv, 128] bf16; with return_states also the end states
    [n_capture, hv, 128, 128] fp32 of the plan's capture nodes.  initial_state [hv, 128, 128] fp32: the state
    every root starts from."""
    if stream is not None:
        return _on_stream(stream, tree_gdn_fwd, locals())
    torch = _torch()
    for t in (q, k, v):
        if t.dim() != 3 or t.dtype != torch.bfloat16 or not t.is_contiguous():
            raise ValueError("q, k, v must be contiguous bf16 [tokens, heads, dim]")
    n, hk, dk = q.shape
    hv, dv = v.shape[1], v.shape[2]
    if k.shape != q.shape or v.shape[0] != n:
        raise ValueError("k must match q, v must have the same token count")
    for t in (g, beta):
        if t.shape != (n, hv) or t.dtype != torch.float32 or not t.is_contiguous():
            raise ValueError("g, beta must be contiguous fp32 [tokens, hv]")
    if plan.device is None:
        plan.to_device(q.device)
    if out is None:
        out = torch.empty((n, hv, dv), dtype=torch.bfloat16, device=q.device)
    need = int(_lib().tt_tree_gdn_workspace(plan.n_chunks, plan.n_slots, hv))
    if workspace is None:
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=q.device)
    d = plan.device
    states = None
    if return_states:
        states = torch.empty((plan.n_capture, hv, dk, dv), dtype=torch.float32, device=q.device)
    if initial_state is not None and (initial_state.shape != (hv, dk, dv) or initial_state.dtype != torch.float32
                                      or not initial_state.is_contiguous()):
        raise ValueError("initial_state must be a contiguous fp32 [hv, dk, dv] tensor")
    _check(_lib().tt_tree_gdn_fwd(n, hk, hv, dk, dv, float(dk) ** -0.5 if scale is None else float(scale), _dp(q), _dp(k), _dp(v),
                                  _dp(g), _dp(beta), plan.n_chunks, _dp(d["chunk_tok0"]), _dp(d["chunk_len"]), _dp(d["chunk_src"]),
                                  _dp(d["chunk_dst"]), plan.n_slots, _dp(d["chunk_cap"]) if return_states and plan.n_capture else None,
                                  _sched_ref(plan), _dp(initial_state), _dp(states) if plan.n_capture else None, _dp(out), _dp(workspace), workspace.numel(),
                                  _stream_ptr(None)))
    return (out, states) if return_states else out


def tree_gdn_bwd_workspace(n_tokens: int, hk: int, hv: int, plan: GdnPlan, smallest: bool = False) -> int:
    """Bytes of workspace with which tree_gdn_bwd takes all heads in one pass, or (smallest) the least it accepts:
    one key head with its value heads per pass.  Anything in between is used for as many key heads per pass as fit."""
    f = _lib().tt_tree_gdn_bwd_workspace_min if smallest else _lib().tt_tree_gdn_bwd_workspace
    return int(f(n_tokens, plan.n_chunks, plan.n_slots, plan.n_segments if plan._schedule() is not None else 0, hk, hv))


def tree_gdn_bwd(q, k, v, g, beta, d_o, plan: GdnPlan, *, scale=None, initial_state=None, d_state_out=None,
                 want_d_initial_state: bool = False, workspace=None, stream=None):
    """Backward of tree_gdn_fwd for upstream d_o [n, hv, 128] bf16.  Returns (dq, dk [n, hk, 128] bf16, dv [n, hv, 128]
    bf16, dg, dbeta [n, hv] fp32), plus d_initial_state [hv, 128, 128] fp32 when asked.  d_state_out
    [n_capture, hv, 128, 128] fp32: upstream gradient of the plan's captured end states.  workspace: a uint8 tensor of
    tree_gdn_bwd_workspace(...) bytes (default: allocated here, full size) or of any size down to its `smallest`."""
    if stream is not None:
        return _on_stream(stream, tree_gdn_bwd, locals())
    torch = _torch()
    for t in (q, k, v, d_o):
        if t.dim() != 3 or t.dtype != torch.bfloat16 or not t.is_contiguous():
            raise ValueError("q, k, v, d_o must be contiguous bf16 [tokens, heads, dim]")
    n, hk, dk = q.shape
    hv, dv = v.shape[1], v.shape[2]
    if k.shape != q.shape or v.shape[0] != n or d_o.shape != v.shape:
        raise ValueError("k must match q, v must have the same token count, d_o must match v")
    for t in (g, beta):
        if t.shape != (n, hv) or t.dtype != torch.float32 or not t.is_contiguous():
            raise ValueError("g, beta must be contiguous fp32 [tokens, hv]")
    for t, shape, name in ((initial_state, (hv, dk, dv), "initial_state"), (d_state_out, (plan.n_capture, hv, dk, dv), "d_state_out")):
        if t is not None and (tuple(t.shape) != shape or t.dtype != torch.float32 or not t.is_contiguous()):
            raise ValueError(f"{name} must be a contiguous fp32 tensor of shape {shape}")
    if plan.device is None:
        plan.to_device(q.device)
    dev = q.device
    dq, dk_ = torch.empty_like(q), torch.empty_like(k)
    dv_ = torch.empty_like(v)
    dg, dbeta = torch.empty_like(g), torch.empty_like(beta)
    d_init = torch.empty((hv, dk, dv), dtype=torch.float32, device=dev) if want_d_initial_state else None
    need = tree_gdn_bwd_workspace(n, hk, hv, plan)
    if workspace is None:
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=dev)
    d = plan.device
    use_cap = d_state_out is not None and plan.n_capture > 0
    _check(_lib().tt_tree_gdn_bwd(n, hk, hv, dk, dv, float(dk) ** -0.5 if scale is None else float(scale), _dp(q), _dp(k), _dp(v),
                                  _dp(g), _dp(beta), _dp(d_o), plan.n_chunks, _dp(d["chunk_tok0"]), _dp(d["chunk_len"]),
                                  _dp(d["chunk_src"]), _dp(d["chunk_dst"]), plan.n_slots, _dp(d["chunk_cap"]) if use_cap else None,
                                  _sched_ref(plan), _dp(initial_state), _dp(d_state_out) if use_cap else None, _dp(dq), _dp(dk_), _dp(dv_), _dp(dg),
                                  _dp(dbeta), _dp(d_init), _dp(workspace), workspace.numel(), _stream_ptr(None)))
    out = (dq, dk_, dv_, dg, dbeta)
    return out + (d_init,) if want_d_initial_state else out


# ---- selective state space scan ----------------------------------------------------------------

class ScanGrads(NamedTuple):
    """Gradients of tree_scan_fwd's inputs; None where the input was not given (or d_initial_state was not asked for)."""
    dx: object
    ddt: object
    dA: object
    dB: object
    dC: object
    dD: object
    dz: object
    ddt_bias: object
    d_initial_state: object


def _scan_desc(x, dt, A, B, C, D, z, dt_bias, softplus) -> _ScanDesc:
    """Checks what the scan and its single-token form share; the stride of y / dy is filled in by the caller."""
    torch = _torch()
    if x.dim() != 2 or A.dim() != 2 or B.dim() != 3:
        raise ValueError("x must be [tokens, channels], A [channels, states], B and C [tokens, groups, states]")
    n, ch = x.shape
    m, groups = A.shape[1], B.shape[1]
    dtype = x.dtype
    xs = _check_rows(x, "x", (n, ch), (torch.bfloat16, torch.float32))
    ds = _check_rows(dt, "dt", (n, ch), (dtype,))
    bs, cs = _check_rows(B, "B", (n, groups, m), (dtype,)), _check_rows(C, "C", (n, groups, m), (dtype,))
    zs = _check_rows(z, "z", (n, ch), (dtype,)) if z is not None else 0
    _check_tensor(A, "A", (ch, m), torch.float32)
    for name, t in (("D", D), ("dt_bias", dt_bias)):
        if t is not None:
            _check_tensor(t, name, (ch,), torch.float32)
    return _ScanDesc(n, ch, m, groups, DTYPE_BF16 if dtype == torch.bfloat16 else DTYPE_FP32, 1 if softplus else 0, xs, ds, zs, bs, cs, 0)


def _check_scan_plan(plan: GdnPlan, n: int) -> None:
    have = int(plan.chunk_tok0[-1]) + int(plan.chunk_len[-1]) if plan.n_chunks else 0
    if have != n:
        raise ValueError(f"the plan is of a tree of {have} tokens, the tensors have {n}")


def tree_scan_fwd(x, dt, A, B, C, plan: GdnPlan, *, D=None, z=None, dt_bias=None, softplus: bool = True, initial_state=None,
                  return_states: bool = False, out=None, workspace=None, stream=None):
    """Selective state space scan with tree state routing: x, dt [n, channels], B, C [n, groups, states] bf16 or fp32 (free token
    strides), A [channels, states] fp32 (negative), D, dt_bias [channels] fp32 or None, z [n, channels] (the gate) or None; the
    chunk program is tree_gdn_plan's, whose first call with these many channels lays it out and copies it to the device (so not one that
    a graph captures; the graph needs the plan afterwards).  Returns y [n, channels]; with return_states also the end states [n_capture, channels, states] fp32 of the plan's
    capture nodes.  initial_state [channels, states] fp32: the state every root starts from."""
    if stream is not None:
        return _on_stream(stream, tree_scan_fwd, locals())
    torch = _torch()
    desc = _scan_desc(x, dt, A, B, C, D, z, dt_bias, softplus)
    n, ch, m = desc.n_tokens, desc.channels, desc.n_state
    _check_scan_plan(plan, n)
    if initial_state is not None:
        _check_tensor(initial_state, "initial_state", (ch, m), torch.float32)
    desc.y_stride_tok = _check_rows(out, "out", (n, ch), (x.dtype,)) if out is not None else ch
    before = _enter_device(x, dt, A, B, C, D, z, dt_bias, initial_state, out, workspace)
    try:
        dev = x.device
        captured = return_states and plan.n_capture > 0
        chunks = plan._scan_chunks(ch, False, dev, captured)
        if out is None:
            out = _new(x, (n, ch))
        states = _new(A, (plan.n_capture, ch, m)) if return_states else None
        need = int(_lib().tt_tree_scan_fwd_workspace(ctypes.byref(desc), chunks.n_chunks, chunks.n_slots))
        if workspace is None:
            workspace = _new(x, (max(need, 256),), torch.uint8)
        _check(_lib().tt_tree_scan_fwd(ctypes.byref(desc), ctypes.byref(chunks), _dp(x), _dp(dt), _dp(A), _dp(B), _dp(C), _dp(D), _dp(z),
                                       _dp(dt_bias), _dp(initial_state), _dp(states) if captured else None, _dp(out), _dp(workspace),
                                       workspace.numel() * workspace.element_size(), _stream_ptr(None)))
    finally:
        _leave_device(before)
    return (out, states) if return_states else out


def tree_scan_workspace(x, A, B, plan: GdnPlan, backward: bool = False) -> int:
    """Bytes of workspace of tree_scan_fwd or tree_scan_bwd for tensors of these shapes."""
    desc = _scan_desc(x, x, A, B, B, None, None, None, True)
    f = _lib().tt_tree_scan_bwd_workspace if backward else _lib().tt_tree_scan_fwd_workspace
    need = int(f(ctypes.byref(desc), plan._scan_program(desc.channels, backward).shape[1], plan.n_slots))
    if need == 0:
        raise ValueError(f"sizes must lie in what the scan is built for: {last_error()}")
    return need


def tree_scan_bwd(x, dt, A, B, C, d_y, plan: GdnPlan, *, D=None, z=None, dt_bias=None, softplus: bool = True, initial_state=None,
                  d_state_out=None, want_d_initial_state: bool = False, workspace=None, stream=None) -> ScanGrads:
    """Backward of tree_scan_fwd for upstream d_y [n, channels] (dtype of x, free token stride).  d_state_out [n_capture, channels,
    states] fp32: upstream gradient of the plan's captured end states.  Returns ScanGrads: dx, ddt, dz like x, dB, dC like B, dA,
    dD, ddt_bias, d_initial_state fp32."""
    if stream is not None:
        return _on_stream(stream, tree_scan_bwd, locals())
    torch = _torch()
    desc = _scan_desc(x, dt, A, B, C, D, z, dt_bias, softplus)
    n, ch, m, groups = desc.n_tokens, desc.channels, desc.n_state, desc.groups
    _check_scan_plan(plan, n)
    if initial_state is not None:
        _check_tensor(initial_state, "initial_state", (ch, m), torch.float32)
    if d_state_out is not None:
        _check_tensor(d_state_out, "d_state_out", (plan.n_capture, ch, m), torch.float32)
    desc.y_stride_tok = _check_rows(d_y, "d_y", (n, ch), (x.dtype,))
    before = _enter_device(x, dt, A, B, C, D, z, dt_bias, initial_state, d_y, d_state_out, workspace)
    try:
        dev = x.device
        captured = d_state_out is not None and plan.n_capture > 0
        chunks = plan._scan_chunks(ch, True, dev, captured)
        like = lambda t: None if t is None else _new(t, t.shape)      # noqa: E731
        grads = ScanGrads(like(x), like(x), like(A), like(B), like(C), like(D), like(z), like(dt_bias), like(A) if want_d_initial_state else None)
        need = int(_lib().tt_tree_scan_bwd_workspace(ctypes.byref(desc), chunks.n_chunks, chunks.n_slots))
        if workspace is None:
            workspace = _new(x, (max(need, 256),), torch.uint8)
        _check(_lib().tt_tree_scan_bwd(ctypes.byref(desc), ctypes.byref(chunks), _dp(x), _dp(dt), _dp(A), _dp(B), _dp(C), _dp(D), _dp(z),
                                       _dp(dt_bias), _dp(initial_state), _dp(d_y), _dp(d_state_out) if captured else None,
                                       *(_dp(g) for g in grads), _dp(workspace), workspace.numel() * workspace.element_size(),
                                       _stream_ptr(None)))
    finally:
        _leave_device(before)
    return grads


def tree_scan_step(x, dt, A, B, C, state, *, index=None, D=None, z=None, dt_bias=None, softplus: bool = True, state_out=None, out=None,
                   stream=None):
    """One token per row: tree_scan_fwd's recurrence from saved states.  x, dt, z [rows, channels], B, C [rows, groups, states]; state
    [slots, channels, states] fp32.  Row r goes on from state index[r] (int32; several rows may share one, an index outside the
    states starts from zero) or, without an index, from state r.  Returns (y [rows, channels], state_out [rows, channels, states]);
    state_out may be state itself (in place) when there is no index."""
    if stream is not None:
        return _on_stream(stream, tree_scan_step, locals())
    torch = _torch()
    desc = _scan_desc(x, dt, A, B, C, D, z, dt_bias, softplus)
    n, ch, m = desc.n_tokens, desc.channels, desc.n_state
    slots = state.shape[0]
    if slots > I32_MAX:
        raise ValueError(f"at most {I32_MAX} slots, not {slots}")
    _check_tensor(state, "state", (slots, ch, m), torch.float32)
    if index is not None:
        _check_tensor(index, "index", (n,), torch.int32)
    if state_out is not None:
        _check_tensor(state_out, "state_out", (slots if state_out is state else n, ch, m), torch.float32)
    desc.y_stride_tok = _check_rows(out, "out", (n, ch), (x.dtype,)) if out is not None else ch
    before = _enter_device(x, dt, A, B, C, D, z, dt_bias, state, index, state_out, out)
    try:
        if out is None:
            out = _new(x, (n, ch))
        if state_out is None:
            state_out = _new(state, (n, ch, m))
        _check(_lib().tt_tree_scan_step(ctypes.byref(desc), _dp(x), _dp(dt), _dp(A), _dp(B), _dp(C), _dp(D), _dp(z), _dp(dt_bias), slots,
                                        _dp(state), _dp(index), _dp(state_out), _dp(out), _stream_ptr(None)))
    finally:
        _leave_device(before)
    return out, state_out


def tree_conv_step(x, state, weight, bias=None, *, index=None, silu: bool = True, state_out=None, out=None, stream=None):
    """One token per row: tree_conv_fwd from saved contexts.  x [rows, C] bf16/fp32 (free row stride), state [slots, K-1, C] like x:
    the inputs before the token, the oldest first; weight [C, K], bias [C] fp32.  index and state_out as in tree_scan_step.
    Returns (y [rows, C], state_out [rows, K-1, C])."""
    if stream is not None:
        return _on_stream(stream, tree_conv_step, locals())
    torch = _torch()
    if x.dim() != 2 or weight.dim() != 2:
        raise ValueError("x must be [rows, channels], weight [channels, taps]")
    n, c = x.shape
    k = weight.shape[1]
    xs = _check_rows(x, "x", (n, c), (torch.bfloat16, torch.float32))
    slots = state.shape[0]
    if slots > I32_MAX or k > I32_MAX:
        raise ValueError(f"at most {I32_MAX} slots, not {slots}, and taps, not {k}")
    _check_tensor(state, "state", (slots, k - 1, c), x.dtype)
    _check_tensor(weight, "weight", (c, k), torch.float32)
    if bias is not None:
        _check_tensor(bias, "bias", (c,), torch.float32)
    if index is not None:
        _check_tensor(index, "index", (n,), torch.int32)
    if state_out is not None:
        _check_tensor(state_out, "state_out", (slots if state_out is state else n, k - 1, c), x.dtype)
    ys = _check_rows(out, "out", (n, c), (x.dtype,)) if out is not None else c
    before = _enter_device(x, state, weight, bias, index, state_out, out)
    try:
        if out is None:
            out = _new(x, (n, c))
        if state_out is None:
            state_out = _new(state, (n, k - 1, c))
        _check(_lib().tt_tree_conv_step(n, c, k, DTYPE_BF16 if x.dtype == torch.bfloat16 else DTYPE_FP32, 1 if silu else 0, _dp(x), xs,
                                        _dp(weight), _dp(bias), slots, _dp(state), _dp(index), _dp(state_out), _dp(out), ys,
                                        _stream_ptr(None)))
    finally:
        _leave_device(before)
    return out, state_out
