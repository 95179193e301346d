"""Python binding of the BLoad C-ABI library (``include/bload.h``).

Argument marshalling only: every function here checks dtypes / devices, takes
``data_ptr()`` of torch tensors (torch is used for device memory and streams,
nothing else) and calls the entry point of the same name in ``libbload.so``.
There is no fallback: importing this module without the built library raises.
"""
from __future__ import annotations

import ctypes
import itertools
import math
import operator
import os
from dataclasses import dataclass

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libbload.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(
        f"{LIB_PATH} is missing: build it with `python -m paper_2310_10879_amd.build` "
        "(there is no CPU fallback)")

_lib = ctypes.CDLL(LIB_PATH)

# status codes (mirror of bload_status)
OK, EINVAL, ELENGTH, EWORKSPACE, EALIGN, EOVERFLOW, EHIP = range(7)
DTYPES = {"u8": 0, "f16": 1, "f32": 2, "i32": 3}
OPS = {"sum": 0, "mean": 1}
ELEM_BYTES = {"u8": 1, "f16": 2, "f32": 4, "i32": 4}
TORCH_DTYPE = {"u8": torch.uint8, "f16": torch.float16, "f32": torch.float32, "i32": torch.int32}
MAX_SEQ = 1 << 27

_vp, _i64, _i32, _u64, _sz = (ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_uint64,
                              ctypes.c_size_t)

_lib.bload_status_string.restype = ctypes.c_char_p
_lib.bload_status_string.argtypes = [ctypes.c_int]
_lib.bload_last_hip_error.restype = ctypes.c_int
_lib.bload_last_hip_error.argtypes = []
_lib.bload_plan_workspace_bytes.restype = _sz
_lib.bload_plan_workspace_bytes.argtypes = [_i64]
_lib.bload_plan.restype = ctypes.c_int
_lib.bload_plan.argtypes = [_vp, _i64, _i32, _u64, _vp, _vp, _vp, _vp,
                            ctypes.POINTER(_i64), ctypes.POINTER(_i64), _vp, _sz, _vp]
_lib.bload_plan_random_fit_workspace_bytes.restype = _sz
_lib.bload_plan_random_fit_workspace_bytes.argtypes = [_i64]
_lib.bload_plan_random_fit.restype = ctypes.c_int
_lib.bload_plan_random_fit.argtypes = list(_lib.bload_plan.argtypes)
_lib.bload_plan_shard.restype = ctypes.c_int
_lib.bload_plan_shard.argtypes = [_vp, _vp, _vp, _i64, _i64, _i32, _i32, _vp, _vp, _vp,
                                  ctypes.POINTER(_i64), ctypes.POINTER(_i64), _vp, _sz, _vp]
_lib.bload_pack_workspace_bytes.restype = _sz
_lib.bload_pack_workspace_bytes.argtypes = [_i64, _i64, _i32, _i64]
_lib.bload_pack_tile_bytes.restype = _i32
_lib.bload_pack_tile_bytes.argtypes = [_i64, _i64, _i32, _i64, _i32]
_lib.bload_pack.restype = ctypes.c_int
_lib.bload_pack.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _i64, _i64, _i32, _i64,
                            _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]
_lib.bload_pack_noalloc.restype = ctypes.c_int
_lib.bload_pack_noalloc.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _i64, _i64, _i32, _i64,
                                    _vp, _vp, _vp, _vp, _vp, _vp]
_lib.bload_pack_check.restype = ctypes.c_int
_lib.bload_pack_check.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, _i64, _i64, _i32, _i64,
                                  ctypes.POINTER(_i64), _vp, _sz, _vp]


class StrategyCounts(ctypes.Structure):
    """bload_strategy_counts_t"""
    _fields_ = [(name, ctypes.c_int64) for name in
                ("total_frames", "longest", "pad_to_longest", "pad_blocks", "chunk_samples",
                 "chunk_deleted")]

    def as_dict(self) -> dict:
        return {name: int(getattr(self, name)) for name, _ in self._fields_}


_lib.bload_strategy_counts.restype = ctypes.c_int
_lib.bload_strategy_counts.argtypes = [_vp, _i64, _i32, _i32, _i64, _i32,
                                       ctypes.POINTER(StrategyCounts), _vp, _sz, _vp]
_lib.bload_segment_scan.restype = ctypes.c_int
_lib.bload_segment_scan.argtypes = [_vp, _vp, _vp, _i64, _i32, _i64, ctypes.c_int, ctypes.c_float, _vp,
                                    _vp, _sz, _vp]
_lib.bload_segment_scan_workspace_bytes.restype = _sz
_lib.bload_segment_scan_workspace_bytes.argtypes = [_i64, _i32, _i64, ctypes.c_int]
_lib.bload_segment_reduce_workspace_bytes.restype = _sz
_lib.bload_segment_reduce_workspace_bytes.argtypes = [_i64, _i32, _i64, ctypes.c_int]
_lib.bload_segment_reduce_layout.restype = _i32
_lib.bload_segment_reduce_layout.argtypes = [_i64, _i32, _i64, ctypes.c_int, _i64, _sz, ctypes.POINTER(_i64)]
_lib.bload_segment_reduce.restype = ctypes.c_int
_lib.bload_segment_reduce.argtypes = [_vp, _vp, _vp, _vp, _i64, _i32, _i64, ctypes.c_int,
                                      ctypes.c_int, _i64, _vp, _vp, _sz, _vp]


class Heads(ctypes.Structure):
    """bload_heads"""
    _fields_ = [("d_data", _vp), ("block_stride", _i64), ("slot_stride", _i64), ("head_stride", _i64)]


_hp, _int, _f32 = ctypes.POINTER(Heads), ctypes.c_int, ctypes.c_float
ATTENTION_MAX_HEAD_DIM = 128
# element types of the operators from bload_segment_attention on, which go by the tensors' own
TYPE_CODE = {torch.float16: 1, torch.float32: 2, torch.bfloat16: 4}
ROTARY_LAYOUTS = {"half": 0, "interleaved": 1}

_lib.bload_segment_mask.restype = _int
_lib.bload_segment_mask.argtypes = [_vp, _vp, _vp, _i64, _i32, _i32, _vp, _i64, _vp, _vp]
_lib.bload_segment_attention.restype = _int
_lib.bload_segment_attention.argtypes = [_hp, _hp, _hp, _vp, _i64, _i32, _i32, _i32, _i32, _int, _f32, _f32, _vp, _hp, _vp, _hp, _vp]
_lib.bload_segment_attention_backward_workspace_bytes.restype = _sz
_lib.bload_segment_attention_backward_workspace_bytes.argtypes = [_i64, _i32, _i32]
_lib.bload_segment_attention_backward.restype = _int
_lib.bload_segment_attention_backward.argtypes = [_hp, _hp, _hp, _hp, _hp, _vp, _hp, _vp, _i64, _i32, _i32, _i32, _i32, _int, _f32,
                                                  _f32, _vp, _hp, _hp, _hp, _vp, _sz, _vp]
_lib.bload_segment_attention_decode_workspace_bytes.restype = _sz
_lib.bload_segment_attention_decode_workspace_bytes.argtypes = [_i64, _i32, _i32, _i32, _i32]
_lib.bload_segment_attention_decode.restype = _int
_lib.bload_segment_attention_decode.argtypes = [_hp, _hp, _hp, _vp, _vp, _vp, _i64, _i64, _i32, _i32, _i32, _i32, _int, _f32, _f32,
                                                _vp, _hp, _vp, _sz, _vp]
_lib.bload_gated_scan_workspace_bytes.restype = _sz
_lib.bload_gated_scan_workspace_bytes.argtypes = [_i64, _i32, _i64, _int]
_lib.bload_gated_scan.restype = _int
_lib.bload_gated_scan.argtypes = [_vp, _vp, _vp, _vp, _i64, _i32, _i64, _int, _vp, _vp, _vp, _vp, _sz, _vp]
_lib.bload_gated_scan_backward.restype = _int
_lib.bload_gated_scan_backward.argtypes = [_vp, _vp, _vp, _vp, _vp, _i64, _i32, _i64, _int, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]
_lib.bload_rotary.restype = _int
_lib.bload_rotary.argtypes = [_hp, _vp, _i64, _i32, _i32, _i32, _int, _vp, _i32, _int, _f32, _i32, _hp, _vp]
_lib.bload_rotary_frequencies.restype = _int
_lib.bload_rotary_frequencies.argtypes = [_i32, ctypes.c_double, ctypes.c_double, _i64, ctypes.c_double, ctypes.c_double, _vp]
_lib.bload_layer_norm.restype = _int
_lib.bload_layer_norm.argtypes = [_hp, _hp, _vp, _i64, _i32, _i32, _i32, _int, _i32, _f32, _vp, _vp, _hp, _hp, _vp, _vp]
_lib.bload_layer_norm_backward_workspace_bytes.restype = _sz
_lib.bload_layer_norm_backward_workspace_bytes.argtypes = [_i64, _i32, _i32, _i32, _int]
_lib.bload_layer_norm_backward.restype = _int
_lib.bload_layer_norm_backward.argtypes = [_hp, _hp, _vp, _vp, _i64, _i32, _i32, _i32, _int, _i32, _vp, _hp, _hp, _vp, _vp, _vp, _sz, _vp]
_lib.bload_segment_conv.restype = _int
_lib.bload_segment_conv.argtypes = [_hp, _vp, _vp, _vp, _vp, _i64, _i32, _i32, _i32, _int, _i32, _vp, _hp, _vp, _vp]
_lib.bload_segment_conv_backward_workspace_bytes.restype = _sz
_lib.bload_segment_conv_backward_workspace_bytes.argtypes = [_i64, _i32, _i32, _i32, _int]
_lib.bload_segment_conv_backward.restype = _int
_lib.bload_segment_conv_backward.argtypes = [_hp, _hp, _vp, _vp, _vp, _vp, _i64, _i32, _i32, _i32, _int, _i32, _vp, _vp, _hp, _vp, _vp, _vp,
                                             _vp, _sz, _vp]


class Selective(ctypes.Structure):
    """bload_selective"""
    _fields_ = [("x", Heads), ("dt", Heads), ("z", Heads), ("b", Heads), ("c", Heads), ("d_rate", _vp), ("d_skip", _vp),
                ("d_dt_bias", _vp), ("d_reset", _vp), ("d_valid", _vp), ("d_state_in", _vp), ("num_blocks", _i64), ("t_blk", _i32),
                ("feat_dim", _i32), ("states", _i32), ("groups", _i32), ("dtype", _int), ("softplus", _i32)]


_sp = ctypes.POINTER(Selective)
SELECTIVE_MAX_STATES = 64
CONV_MAX_TAPS = 8
for _name in ("workspace", "saved", "backward_workspace"):
    _f = getattr(_lib, f"bload_selective_scan_{_name}_bytes")
    _f.restype, _f.argtypes = _sz, [_i64, _i32, _i32, _i32, _i32]
_lib.bload_selective_scan.restype = _int
_lib.bload_selective_scan.argtypes = [_sp, _hp, _vp, _vp, _vp, _sz, _vp]
_lib.bload_selective_scan_backward.restype = _int
_lib.bload_selective_scan_backward.argtypes = [_sp, _hp, _vp, _vp, _hp, _hp, _vp, _hp, _hp, _vp, _hp, _vp, _vp, _vp, _sz, _vp]


class BloadError(RuntimeError):
    def __init__(self, status: int):
        self.status = status
        msg = _lib.bload_status_string(status).decode()
        if status == EHIP:
            msg += f" (hipError {_lib.bload_last_hip_error()})"
        super().__init__(msg)


def status_string(status: int) -> str:
    return _lib.bload_status_string(status).decode()


def _check(status: int) -> None:
    if status != OK:
        raise BloadError(status)


def _ptr(t, dtype=None) -> int:
    if t is None:
        return 0
    if not t.is_cuda:
        raise ValueError("expected a device tensor")
    if not t.is_contiguous():
        raise ValueError("expected a contiguous tensor")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"expected {dtype}, got {t.dtype}")
    return t.data_ptr()


def _room(workspace) -> int:
    return 0 if workspace is None else workspace.numel() * workspace.element_size()


# The current stream's handle without a Stream object around it, where this torch has the call
# (0.4 us instead of 2.9, of 14 that a call on small tensors takes the host in all).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream() -> int:
    if _raw_stream is not None:
        return _raw_stream(torch.cuda.current_device())
    return torch.cuda.current_stream().cuda_stream


def bload_plan_workspace_bytes(n_seq: int) -> int:
    return int(_lib.bload_plan_workspace_bytes(n_seq))


def bload_pack_workspace_bytes(n_seq: int, num_blocks: int, t_blk: int, frame_bytes: int) -> int:
    return int(_lib.bload_pack_workspace_bytes(n_seq, num_blocks, t_blk, frame_bytes))


def bload_segment_reduce_workspace_bytes(num_blocks: int, t_blk: int, feat_dim: int,
                                         dtype: str) -> int:
    return int(_lib.bload_segment_reduce_workspace_bytes(num_blocks, t_blk, feat_dim,
                                                         DTYPES[dtype]))


@dataclass
class Plan:
    """Device-resident result of ``bload_plan``."""
    order: torch.Tensor            # int32[N]
    block_of_seq: torch.Tensor     # int32[N]
    offset_of_seq: torch.Tensor    # int32[N]
    block_first: torch.Tensor      # int32[N+1], entries [0..B] valid
    num_blocks: int
    total_frames: int
    t_blk: int


def _new_plan(n: int, t_blk: int, dev) -> Plan:
    # (one allocation: four take 5.2 us of the some 46 that plan, pack and reduction of a small batch take, this 2.9, or 3.8 where the
    # tables need gaps to begin at multiples of 256 bytes, as device memory of their own would)
    gap = -n % 64
    tables = torch.empty(4 * n + 3 * gap + 1, dtype=torch.int32, device=dev)
    if gap:
        order, _, block_of_seq, _, offset_of_seq, _, block_first = tables.split_with_sizes((n, gap, n, gap, n, gap, n + 1))
    else:
        order, block_of_seq, offset_of_seq, block_first = tables.split_with_sizes((n, n, n, n + 1))
    return Plan(order, block_of_seq, offset_of_seq, block_first, 0, 0, t_blk)


def bload_plan(lengths: torch.Tensor, t_blk: int, seed: int, workspace: torch.Tensor | None = None,
               out: Plan | None = None) -> Plan:
    """lengths: int32[N] on the device.  Synchronises the current stream."""
    n = lengths.shape[0]
    dev = lengths.device
    if out is None:
        out = _new_plan(n, t_blk, dev)
    if workspace is None:
        workspace = torch.empty(max(bload_plan_workspace_bytes(n), 16), dtype=torch.uint8, device=dev)
    nb, tot = _i64(0), _i64(0)
    st = _lib.bload_plan(_ptr(lengths, torch.int32), n, t_blk, seed & (2**64 - 1),
                         _ptr(out.order, torch.int32), _ptr(out.block_of_seq, torch.int32),
                         _ptr(out.offset_of_seq, torch.int32), _ptr(out.block_first, torch.int32),
                         ctypes.byref(nb), ctypes.byref(tot), _ptr(workspace),
                         workspace.numel() * workspace.element_size(), _stream())
    _check(st)
    out.num_blocks, out.total_frames, out.t_blk = int(nb.value), int(tot.value), t_blk
    return out


def bload_plan_random_fit_workspace_bytes(n_seq: int) -> int:
    return int(_lib.bload_plan_random_fit_workspace_bytes(n_seq))


def bload_plan_random_fit(lengths: torch.Tensor, t_blk: int, seed: int,
                          workspace: torch.Tensor | None = None, out: Plan | None = None) -> Plan:
    """The plan built with the paper's sampler (uniform among the remaining sequences that
    still fit the open block).  lengths: int32[N] on the device.  Synchronises the current
    stream."""
    n = lengths.shape[0]
    dev = lengths.device
    if out is None:
        out = _new_plan(n, t_blk, dev)
    if workspace is None:
        workspace = torch.empty(max(bload_plan_random_fit_workspace_bytes(n), 16), dtype=torch.uint8,
                                device=dev)
    nb, tot = _i64(0), _i64(0)
    st = _lib.bload_plan_random_fit(_ptr(lengths, torch.int32), n, t_blk, seed & (2**64 - 1),
                                    _ptr(out.order, torch.int32), _ptr(out.block_of_seq, torch.int32),
                                    _ptr(out.offset_of_seq, torch.int32),
                                    _ptr(out.block_first, torch.int32), ctypes.byref(nb),
                                    ctypes.byref(tot), _ptr(workspace),
                                    workspace.numel() * workspace.element_size(), _stream())
    _check(st)
    out.num_blocks, out.total_frames, out.t_blk = int(nb.value), int(tot.value), t_blk
    return out


def bload_plan_shard(plan: Plan, rank: int, world: int) -> Plan:
    """Worker ``rank``'s share of ``plan`` (blocks rank mod world, plus a padding block for
    the workers that would fall short) as a Plan in the worker's own block numbering.
    Synchronises the current stream."""
    n = plan.order.shape[0]
    dev = plan.order.device
    nb_local = -(-plan.num_blocks // world) if world > 0 else 0     # the library refuses world < 1
    out = Plan(torch.empty(n, dtype=torch.int32, device=dev),
               torch.empty(n, dtype=torch.int32, device=dev), plan.offset_of_seq,
               torch.empty(nb_local + 1, dtype=torch.int32, device=dev), nb_local,
               plan.total_frames, plan.t_blk)
    ws = torch.empty(16, dtype=torch.uint8, device=dev)
    nb, ns = _i64(0), _i64(0)
    st = _lib.bload_plan_shard(_ptr(plan.order, torch.int32), _ptr(plan.block_of_seq, torch.int32),
                               _ptr(plan.block_first, torch.int32), n, plan.num_blocks, rank, world,
                               _ptr(out.order, torch.int32), _ptr(out.block_of_seq, torch.int32),
                               _ptr(out.block_first, torch.int32), ctypes.byref(nb),
                               ctypes.byref(ns), _ptr(ws), 16, _stream())
    _check(st)
    assert nb.value == nb_local
    out.n_local = int(ns.value)
    return out


@dataclass
class Packed:
    """Device-resident result of ``bload_pack``."""
    packed: torch.Tensor      # uint8[B, T, frame_bytes]
    seq_id: torch.Tensor      # int32[B, T]
    frame_idx: torch.Tensor   # int32[B, T]
    reset: torch.Tensor       # uint8[B, T]
    valid: torch.Tensor       # uint8[B, T]


def alloc_packed(num_blocks: int, t_blk: int, frame_bytes: int, device) -> Packed:
    return Packed(torch.empty((num_blocks, t_blk, frame_bytes), dtype=torch.uint8, device=device),
                  torch.empty((num_blocks, t_blk), dtype=torch.int32, device=device),
                  torch.empty((num_blocks, t_blk), dtype=torch.int32, device=device),
                  torch.empty((num_blocks, t_blk), dtype=torch.uint8, device=device),
                  torch.empty((num_blocks, t_blk), dtype=torch.uint8, device=device))


def bload_pack(src: torch.Tensor, src_offsets: torch.Tensor, lengths: torch.Tensor, plan: Plan,
               frame_bytes: int, out: Packed | None = None,
               workspace: torch.Tensor | None = None) -> Packed:
    """src: the ragged source (any dtype, contiguous, ``total_frames * frame_bytes`` bytes);
    src_offsets: int64[N+1].  Asynchronous on the current stream."""
    n = lengths.shape[0]
    if src.numel() * src.element_size() != plan.total_frames * frame_bytes:
        raise ValueError("source size does not match total_frames * frame_bytes")
    if out is None:
        out = alloc_packed(plan.num_blocks, plan.t_blk, frame_bytes, lengths.device)
    if out.packed.numel() != plan.num_blocks * plan.t_blk * frame_bytes or \
            out.seq_id.numel() != plan.num_blocks * plan.t_blk:
        raise ValueError("output buffers do not match num_blocks * t_blk")
    if workspace is None:
        need = bload_pack_workspace_bytes(n, plan.num_blocks, plan.t_blk, frame_bytes)
        workspace = torch.empty(max(need, 32), dtype=torch.uint8, device=lengths.device)
    st = _lib.bload_pack(_ptr(src), _ptr(src_offsets, torch.int64), _ptr(lengths, torch.int32),
                         _ptr(plan.order, torch.int32), _ptr(plan.block_of_seq, torch.int32),
                         _ptr(plan.offset_of_seq, torch.int32), _ptr(plan.block_first, torch.int32),
                         n, plan.num_blocks, plan.t_blk, frame_bytes,
                         _ptr(out.packed, torch.uint8), _ptr(out.seq_id, torch.int32),
                         _ptr(out.frame_idx, torch.int32), _ptr(out.reset, torch.uint8),
                         _ptr(out.valid, torch.uint8), _ptr(workspace),
                         workspace.numel() * workspace.element_size(), _stream())
    _check(st)
    return out


PACK_NOALLOC_MAX_SEQ = 1 << 18
PACK_NOALLOC_MAX_TILES = 1 << 21


def bload_pack_noalloc(src: torch.Tensor, src_offsets: torch.Tensor, lengths: torch.Tensor, plan: Plan,
                       frame_bytes: int, out: Packed) -> Packed:
    """``bload_pack`` with its scratch in the library's fixed device array: nothing is allocated
    here or in the library, so ``out`` must be brought along.  Asynchronous on the current
    stream; calls on one GPU must not overlap."""
    if src.numel() * src.element_size() != plan.total_frames * frame_bytes:
        raise ValueError("source size does not match total_frames * frame_bytes")
    if out.packed.numel() != plan.num_blocks * plan.t_blk * frame_bytes or \
            out.seq_id.numel() != plan.num_blocks * plan.t_blk:
        raise ValueError("output buffers do not match num_blocks * t_blk")
    st = _lib.bload_pack_noalloc(_ptr(src), _ptr(src_offsets, torch.int64), _ptr(lengths, torch.int32),
                                 _ptr(plan.order, torch.int32), _ptr(plan.block_of_seq, torch.int32),
                                 _ptr(plan.offset_of_seq, torch.int32), _ptr(plan.block_first, torch.int32),
                                 lengths.shape[0], plan.num_blocks, plan.t_blk, frame_bytes,
                                 _ptr(out.packed, torch.uint8), _ptr(out.seq_id, torch.int32),
                                 _ptr(out.frame_idx, torch.int32), _ptr(out.reset, torch.uint8),
                                 _ptr(out.valid, torch.uint8), _stream())
    _check(st)
    return out


def bload_pack_check(src_offsets: torch.Tensor, lengths: torch.Tensor, plan: Plan,
                     total_frames: int | None = None) -> int:
    """-1 if the tables are a plan ``bload_pack`` can take, else the smallest shuffled position
    or block at which they are not.  Synchronises the current stream."""
    ws = torch.empty(16, dtype=torch.uint8, device=lengths.device)
    bad = _i64(-1)
    st = _lib.bload_pack_check(_ptr(src_offsets, torch.int64), _ptr(lengths, torch.int32),
                               _ptr(plan.order, torch.int32), _ptr(plan.block_of_seq, torch.int32),
                               _ptr(plan.offset_of_seq, torch.int32), _ptr(plan.block_first, torch.int32),
                               lengths.shape[0], plan.num_blocks, plan.t_blk,
                               plan.total_frames if total_frames is None else total_frames,
                               ctypes.byref(bad), _ptr(ws), 16, _stream())
    if st == EINVAL and bad.value >= 0:
        return int(bad.value)
    _check(st)
    return -1


def bload_segment_reduce(packed: torch.Tensor, seq_id: torch.Tensor, reset: torch.Tensor,
                         valid: torch.Tensor, num_blocks: int, t_blk: int, feat_dim: int,
                         dtype: str, op: str, n_seq: int, out: torch.Tensor | None = None,
                         workspace: torch.Tensor | None = None) -> torch.Tensor:
    """Per-sequence sum / mean over the packed blocks -> [n_seq, feat_dim] (float32, or int64
    for ``i32``).  Rows of sequences that do not occur keep their previous content (zeros when
    this function allocates ``out``).  Asynchronous on the current stream."""
    dev = packed.device
    if out is None:
        out = torch.zeros((n_seq, feat_dim), device=dev,
                          dtype=torch.int64 if dtype == "i32" else torch.float32)
    if workspace is None:
        need = bload_segment_reduce_workspace_bytes(num_blocks, t_blk, feat_dim, dtype)
        workspace = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
    esize = ELEM_BYTES[dtype]
    if packed.numel() * packed.element_size() != num_blocks * t_blk * feat_dim * esize:
        raise ValueError("packed size does not match num_blocks * t_blk * feat_dim")
    st = _lib.bload_segment_reduce(_ptr(packed), _ptr(seq_id, torch.int32),
                                   _ptr(reset, torch.uint8), _ptr(valid, torch.uint8),
                                   num_blocks, t_blk, feat_dim, DTYPES[dtype], OPS[op], n_seq,
                                   _ptr(out), _ptr(workspace), _room(workspace), _stream())
    _check(st)
    return out


def bload_strategy_counts(lengths: torch.Tensor, t_chunk: int, t_max: int = 0, num_blocks: int = 0,
                          t_blk: int = 0, workspace: torch.Tensor | None = None) -> dict:
    """Frames of padding / frames deleted under padding to the longest sequence, chunk sampling
    with pieces of ``t_chunk`` frames, and block packing (``num_blocks`` x ``t_blk``).
    ``t_max`` <= 0 pads to the longest sequence found.  Synchronises the current stream."""
    if workspace is None:
        workspace = torch.empty(64, dtype=torch.uint8, device=lengths.device)
    out = StrategyCounts()
    st = _lib.bload_strategy_counts(_ptr(lengths, torch.int32), lengths.shape[0], t_max, t_chunk,
                                    num_blocks, t_blk, ctypes.byref(out), _ptr(workspace),
                                    workspace.numel() * workspace.element_size(), _stream())
    _check(st)
    return out.as_dict()


def bload_segment_scan_workspace_bytes(num_blocks: int, t_blk: int, feat_dim: int, dtype: str) -> int:
    return int(_lib.bload_segment_scan_workspace_bytes(num_blocks, t_blk, feat_dim, DTYPES[dtype]))


def bload_segment_scan(packed: torch.Tensor, reset: torch.Tensor, valid: torch.Tensor, num_blocks: int,
                       t_blk: int, feat_dim: int, dtype: str, decay: float,
                       out: torch.Tensor | None = None,
                       workspace: torch.Tensor | None = None) -> torch.Tensor:
    """h = x at sequence starts, decay * h_prev + x elsewhere, 0 on padding: float32
    [num_blocks, t_blk, feat_dim].  Asynchronous on the current stream."""
    if out is None:
        out = torch.empty((num_blocks, t_blk, feat_dim), dtype=torch.float32, device=packed.device)
    if workspace is None:
        need = bload_segment_scan_workspace_bytes(num_blocks, t_blk, feat_dim, dtype) if dtype != "i32" else 0
        workspace = torch.empty(need, dtype=torch.uint8, device=packed.device) if need else None
    st = _lib.bload_segment_scan(_ptr(packed), _ptr(reset, torch.uint8), _ptr(valid, torch.uint8),
                                 num_blocks, t_blk, feat_dim, DTYPES[dtype], float(decay),
                                 _ptr(out, torch.float32), _ptr(workspace), _room(workspace), _stream())
    _check(st)
    return out


REDUCE_LAYOUTS = ("none", "wide", "staged", "flat", "narrow")


def bload_segment_reduce_layout(num_blocks: int, t_blk: int, feat_dim: int, dtype: str, n_seq: int,
                                workspace_bytes: int | None = None) -> tuple[str, int]:
    """Which layout ``bload_segment_reduce`` takes for these sizes, and into how many chunks or tiles it
    cuts the blocks, with a workspace of that size (default: what its query answers)."""
    if workspace_bytes is None:
        workspace_bytes = bload_segment_reduce_workspace_bytes(num_blocks, t_blk, feat_dim, dtype)
    chunks = _i64(0)
    layout = _lib.bload_segment_reduce_layout(num_blocks, t_blk, feat_dim, DTYPES[dtype], n_seq, workspace_bytes,
                                              ctypes.byref(chunks))
    return REDUCE_LAYOUTS[layout], int(chunks.value)


def bload_pack_tile_bytes(n_seq: int, num_blocks: int, t_blk: int, frame_bytes: int,
                          src_aligned_16: bool = True) -> int:
    """4096 if ``bload_pack`` cuts the packed tensor into 4 KiB tiles for these sizes
    (pack_wide_kernel, pack_direct_kernel), 0 if into tiles of 1024 slots (pack_narrow_kernel, pack_narrow_direct_kernel)."""
    return int(_lib.bload_pack_tile_bytes(n_seq, num_blocks, t_blk, frame_bytes, int(src_aligned_16)))


# ---- operators on packed blocks whose element type is the tensors' own -------------------------
#
# Their results carry no gradient, whatever requires one: a backward pass is a call of its own (examples/packed_layer.py wraps each
# pair in a torch.autograd.Function).


def _heads(t: torch.Tensor, shape, dtype, name: str) -> Heads:
    """A tensor [B, T, heads, D] (or [n, heads, D]) of any strides with the elements of a head side by side."""
    if not t.is_cuda:
        raise ValueError(f"{name}: expected a device tensor")
    if t.dtype != dtype:
        raise ValueError(f"{name}: expected {dtype}, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name}: expected shape {tuple(shape)}, got {tuple(t.shape)}")
    stride = t.stride()
    if stride[-1] != 1 and shape[-1] > 1:
        raise ValueError(f"{name}: the elements of a head have to lie side by side")
    return Heads(t.data_ptr(), stride[0], stride[1] if len(stride) == 4 else 0, stride[-2])


def _merges(got, shape) -> bool:
    """Whether `got` is `shape` with neighbouring dimensions taken together, or with some of 1 more or less: the same elements
    in the same order, other than a transposed tensor of as many."""
    ends = set(itertools.accumulate(reversed(shape), operator.mul, initial=1))
    return math.prod(got) == math.prod(shape) and ends.issuperset(itertools.accumulate(reversed(got), operator.mul))


def _sized(t: torch.Tensor | None, shape, dtype, name: str) -> int:
    """A contiguous tensor of this shape, dimensions taken together or not; None: no pointer."""
    if t is None:
        return 0
    if t.dtype is dtype and t.shape == shape and t.is_cuda and t.is_contiguous():
        return t.data_ptr()                        # (the checks below at half their price: small calls are all host time)
    if not _merges(t.shape, shape):
        raise ValueError(f"{name}: expected shape {tuple(shape)}, got {tuple(t.shape)}")
    return _ptr(t, dtype)


def _type_code(t: torch.Tensor) -> int:
    code = TYPE_CODE.get(t.dtype)
    if code is None:
        raise ValueError(f"expected float16, bfloat16 or float32, got {t.dtype}")
    return code


def bload_segment_mask(reset: torch.Tensor, valid: torch.Tensor, causal: bool = True, prefix: torch.Tensor | None = None,
                       seq_id: torch.Tensor | None = None, out: torch.Tensor | None = None) -> torch.Tensor:
    """Who sees whom in attention inside the sequences of packed blocks: int32[B, T, 4], per slot the interval of
    keys that its query sees and the interval of queries that see its key.  reset, valid: uint8[B, T].
    causal: a query sees its own frame and those in front of it, and with prefix (int32[n_seq], needs seq_id:
    int32[B, T]) the first prefix[i] frames of its sequence i.  Asynchronous on the current stream."""
    B, T = valid.shape
    if reset.shape != valid.shape or (seq_id is not None and seq_id.shape != valid.shape):
        raise ValueError("reset, valid and seq_id differ in shape")
    if out is None:
        out = torch.empty((B, T, 4), dtype=torch.int32, device=valid.device)
    n = 0 if prefix is None else prefix.shape[0]
    _check(_lib.bload_segment_mask(_ptr(reset, torch.uint8), _ptr(valid, torch.uint8),
                                   0 if prefix is None else _ptr(seq_id, torch.int32), B, T, int(causal), _ptr(prefix, torch.int32),
                                   n, _sized(out, (B, T, 4), torch.int32, "out"), _stream()))
    return out


@dataclass
class Saved:
    """What ``bload_segment_attention`` leaves for its backward pass."""
    lse: torch.Tensor                 # float32[B, heads_q, T]
    rest: torch.Tensor | None         # [B, T, heads_q, D]: what rounding took from the result (None for float32)


def bload_segment_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, mask: torch.Tensor, scale: float | None = None,
                            cap: float = 0.0, slopes: torch.Tensor | None = None, training: bool = False,
                            out: torch.Tensor | None = None):
    """Attention inside the sequences of packed blocks.  q: [B, T, heads_q, D], k and v: [B, T, heads_kv, D] of float16,
    bfloat16 or float32, any strides with the elements of a head side by side; mask from ``bload_segment_mask``;
    scale: 1 / sqrt(D) by default; cap > 0: scores are cap tanh(s / cap); slopes (float32[heads_q]): minus slope times the
    distance in frames.  Returns the result [B, T, heads_q, D], and with ``training`` what
    ``bload_segment_attention_backward`` needs beside it.  Asynchronous on the current stream."""
    B, T, Hq, D = q.shape
    Hkv, dtype = k.shape[2], q.dtype
    code = _type_code(q)
    shape = (B, T, Hkv, D)
    hq, hk, hv = _heads(q, q.shape, dtype, "q"), _heads(k, shape, dtype, "k"), _heads(v, shape, dtype, "v")
    if out is None:
        out = q.new_empty((B, T, Hq, D))
    saved = hr = None
    if training:
        saved = Saved(q.new_empty((B, Hq, T), dtype=torch.float32), None if dtype == torch.float32 else q.new_empty((B, T, Hq, D)))
        hr = None if saved.rest is None else _heads(saved.rest, q.shape, dtype, "rest")
    _check(_lib.bload_segment_attention(hq, hk, hv, _sized(mask, (B, T, 4), torch.int32, "mask"), B, T, Hq, Hkv, D, code,
                                        D ** -0.5 if scale is None else scale, cap, _sized(slopes, (Hq,), torch.float32, "slopes"),
                                        _heads(out, q.shape, dtype, "out"), saved.lse.data_ptr() if training else 0, hr, _stream()))
    return (out, saved) if training else out


def bload_segment_attention_backward_workspace_bytes(num_blocks: int, t_blk: int, heads_q: int) -> int:
    return int(_lib.bload_segment_attention_backward_workspace_bytes(num_blocks, t_blk, heads_q))


def bload_segment_attention_backward(dout: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor,
                                     saved: Saved, mask: torch.Tensor, scale: float | None = None, cap: float = 0.0,
                                     slopes: torch.Tensor | None = None, grads=None, workspace: torch.Tensor | None = None):
    """Gradients (dq, dk, dv) of sum(out * dout); out and saved are the forward call's.  grads: three tensors to
    write into (any strides).  Asynchronous on the current stream."""
    B, T, Hq, D = q.shape
    Hkv, dtype = k.shape[2], q.dtype
    code = _type_code(q)
    shape = (B, T, Hkv, D)
    if grads is None:
        grads = q.new_empty((B, T, Hq, D)), q.new_empty((B, T, Hkv, D)), q.new_empty((B, T, Hkv, D))
    dq, dk, dv = grads
    if workspace is None:
        workspace = torch.empty(max(16, bload_segment_attention_backward_workspace_bytes(B, T, Hq)), dtype=torch.uint8, device=q.device)
    hr = None if saved.rest is None else _heads(saved.rest, q.shape, dtype, "rest")
    _check(_lib.bload_segment_attention_backward(
        _heads(dout, q.shape, dtype, "dout"), _heads(q, q.shape, dtype, "q"), _heads(k, shape, dtype, "k"), _heads(v, shape, dtype, "v"),
        _heads(out, q.shape, dtype, "out"), _sized(saved.lse, (B, Hq, T), torch.float32, "lse"), hr,
        _sized(mask, (B, T, 4), torch.int32, "mask"), B, T, Hq, Hkv, D, code, D ** -0.5 if scale is None else scale, cap,
        _sized(slopes, (Hq,), torch.float32, "slopes"), _heads(dq, q.shape, dtype, "dq"), _heads(dk, shape, dtype, "dk"),
        _heads(dv, shape, dtype, "dv"), _ptr(workspace), _room(workspace), _stream()))
    return dq, dk, dv


def bload_segment_attention_decode_workspace_bytes(n_seq: int, t_blk: int, heads_q: int, heads_kv: int, head_dim: int) -> int:
    return int(_lib.bload_segment_attention_decode_workspace_bytes(n_seq, t_blk, heads_q, heads_kv, head_dim))


def bload_segment_attention_decode(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, block_of_seq: torch.Tensor,
                                   offset_of_seq: torch.Tensor, lengths: torch.Tensor, scale: float | None = None, cap: float = 0.0,
                                   slopes: torch.Tensor | None = None, out: torch.Tensor | None = None,
                                   workspace: torch.Tensor | None = None) -> torch.Tensor:
    """One query per sequence, q: [n_seq, heads_q, D], over the packed blocks k, v: [B, T, heads_kv, D] as a cache: sequence i
    lies in slots [offset_of_seq[i], + lengths[i]) of block block_of_seq[i] (int32[n_seq] each, a plan's tables), and the query
    stands at its last frame.  Returns [n_seq, heads_q, D].  Asynchronous on the current stream."""
    n, Hq, D = q.shape
    B, T, Hkv, _ = k.shape
    dtype = q.dtype
    code = _type_code(q)
    if out is None:
        out = q.new_empty((n, Hq, D))
    if workspace is None:
        need = bload_segment_attention_decode_workspace_bytes(n, T, Hq, Hkv, D)
        workspace = torch.empty(need, dtype=torch.uint8, device=q.device) if need else None
    shape = (B, T, Hkv, D)
    _check(_lib.bload_segment_attention_decode(
        _heads(q, q.shape, dtype, "q"), _heads(k, shape, dtype, "k"), _heads(v, shape, dtype, "v"),
        _sized(block_of_seq, (n,), torch.int32, "block_of_seq"), _sized(offset_of_seq, (n,), torch.int32, "offset_of_seq"),
        _sized(lengths, (n,), torch.int32, "lengths"), n, B, T, Hq, Hkv, D, code, D ** -0.5 if scale is None else scale, cap,
        _sized(slopes, (Hq,), torch.float32, "slopes"), _heads(out, q.shape, dtype, "out"), _ptr(workspace), _room(workspace),
        _stream()))
    return out


def bload_gated_scan_workspace_bytes(num_blocks: int, t_blk: int, feat_dim: int, dtype: torch.dtype) -> int:
    return int(_lib.bload_gated_scan_workspace_bytes(num_blocks, t_blk, feat_dim, TYPE_CODE[dtype]))


def _gated_workspace(workspace, B, T, D, code, device):
    if workspace is None:
        need = _lib.bload_gated_scan_workspace_bytes(B, T, D, code)
        workspace = torch.empty(need, dtype=torch.uint8, device=device) if need else None
    return workspace


def bload_gated_scan(gate: torch.Tensor, x: torch.Tensor, reset: torch.Tensor, valid: torch.Tensor, h0: torch.Tensor | None = None,
                     out: torch.Tensor | None = None, state: torch.Tensor | None = None, workspace: torch.Tensor | None = None):
    """h = gate * h_prev + x inside the sequences of packed blocks, x at their starts, 0 on padding.  gate, x: contiguous
    [B, T, D] of float16, bfloat16 or float32; h0 (float32[B, D]): the state in front of the blocks.  Returns h and
    the state behind the last slots (float32[B, D]), written to `state`, which may be h0 where T <= 8 and is refused where
    it meets h0 in any other way.  Asynchronous on the current stream."""
    B, T, D = x.shape
    dtype, code, shape = x.dtype, _type_code(x), x.shape
    if out is None:
        out = x.new_empty((B, T, D))
    if state is None:
        state = x.new_empty((B, D), dtype=torch.float32)
    workspace = _gated_workspace(workspace, B, T, D, code, x.device)
    _check(_lib.bload_gated_scan(_sized(gate, shape, dtype, "gate"), _ptr(x), _sized(reset, (B, T), torch.uint8, "reset"),
                                 _sized(valid, (B, T), torch.uint8, "valid"), B, T, D, code, _sized(h0, (B, D), torch.float32, "h0"),
                                 _sized(out, shape, dtype, "out"), _sized(state, (B, D), torch.float32, "state"), _ptr(workspace),
                                 _room(workspace), _stream()))
    return out, state


def bload_gated_scan_backward(dout: torch.Tensor, gate: torch.Tensor, out: torch.Tensor, reset: torch.Tensor, valid: torch.Tensor,
                              h0: torch.Tensor | None = None, dstate: torch.Tensor | None = None, grads=None,
                              workspace: torch.Tensor | None = None):
    """Gradients (dgate, dx, dh0) of sum(out * dout) + sum(state * dstate); out is the forward call's result.
    grads: three tensors to write into (dh0 may be dstate or h0 where T <= 8).  Asynchronous on the current stream."""
    B, T, D = dout.shape
    dtype, code, shape = dout.dtype, _type_code(dout), dout.shape
    if grads is None:
        grads = dout.new_empty((B, T, D)), dout.new_empty((B, T, D)), dout.new_empty((B, D), dtype=torch.float32)
    dgate, dx, dh0 = grads
    workspace = _gated_workspace(workspace, B, T, D, code, dout.device)
    _check(_lib.bload_gated_scan_backward(_ptr(dout), _sized(gate, shape, dtype, "gate"), _sized(out, shape, dtype, "out"),
                                          _sized(reset, (B, T), torch.uint8, "reset"), _sized(valid, (B, T), torch.uint8, "valid"),
                                          B, T, D, code, _sized(h0, (B, D), torch.float32, "h0"),
                                          _sized(dstate, (B, D), torch.float32, "dstate"), _sized(dgate, shape, dtype, "dgate"),
                                          _sized(dx, shape, dtype, "dx"), _sized(dh0, (B, D), torch.float32, "dh0"), _ptr(workspace),
                                          _room(workspace), _stream()))
    return dgate, dx, dh0


def bload_rotary_frequencies(rot_dim: int, base: float = 10000.0, factor: float = 1.0, trained: int = 0, slow: float = 1.0,
                             fast: float = 32.0) -> torch.Tensor:
    """float32[rot_dim / 2] on the host: base^(-2 i / rot_dim), stretched for contexts ``factor`` times as long as the
    ``trained`` frames (0: all alike; else only the frequencies of few turns over that length)."""
    out = torch.empty(max(0, rot_dim // 2), dtype=torch.float32)
    _check(_lib.bload_rotary_frequencies(rot_dim, base, factor, trained, slow, fast, out.data_ptr()))
    return out


def bload_rotary(x: torch.Tensor, positions: torch.Tensor, frequencies: torch.Tensor, layout: str = "half", scale: float = 1.0,
                 inverse: bool = False, out: torch.Tensor | None = None) -> torch.Tensor:
    """The first 2 * len(frequencies) elements of every head of x [B, T, heads, D] turned by positions * frequencies
    (int32[B, T], negative: padding, zeros; float32 radians per frame); inverse: turned back, the gradient.  out may
    be x.  Asynchronous on the current stream."""
    B, T, H, D = x.shape
    code = _type_code(x)
    if out is None:
        out = x.new_empty((B, T, H, D))
    _check(_lib.bload_rotary(_heads(x, x.shape, x.dtype, "x"), _sized(positions, (B, T), torch.int32, "positions"), B, T, H, D, code,
                             _ptr(frequencies, torch.float32), 2 * frequencies.shape[0], ROTARY_LAYOUTS[layout], scale, int(inverse),
                             _heads(out, x.shape, x.dtype, "out"), _stream()))
    return out


def _frames(t: torch.Tensor, shape, dtype, name: str) -> Heads:
    """A tensor [B, T, D] of any strides with the features of a slot side by side."""
    h = _heads(t, shape, dtype, name)
    h.slot_stride, h.head_stride = h.head_stride, 0
    return h


def _new(like: torch.Tensor, shape, row: int) -> tuple[torch.Tensor, Heads]:
    """A new tensor [B, T, ...] of like's type and what the library takes of it, whose rows have `row` elements.  (Nothing to
    check here, which is a microsecond a tensor.)"""
    t = like.new_empty(shape)
    slot = math.prod(shape[2:])
    return t, Heads(t.data_ptr(), shape[1] * slot, slot, row)


def _rows(t: torch.Tensor, shape, dtype, name: str) -> Heads:
    """A tensor [B, T, heads, D], or [B, T, D] for one head."""
    return _heads(t, shape, dtype, name) if len(shape) == 4 else _frames(t, shape, dtype, name)


def _row_sizes(shape):
    if len(shape) not in (3, 4):
        raise ValueError(f"x: expected [B, T, D] or [B, T, heads, D], got {tuple(shape)}")
    return shape if len(shape) == 4 else (shape[0], shape[1], 1, shape[2])


def bload_layer_norm(x: torch.Tensor, weight: torch.Tensor | None = None, bias: torch.Tensor | None = None,
                     residual: torch.Tensor | None = None, valid: torch.Tensor | None = None, eps: float = 1e-5, center: bool = True,
                     training: bool = False, out: torch.Tensor | None = None, total: torch.Tensor | None = None):
    """Layer norm (center) or root mean square norm of the last dimension of x: [B, T, D] or [B, T, heads, D] of float16, bfloat16 or
    float32, any strides with the elements of a row side by side; weight, bias: float32[D].  residual (like x): their
    rounded sum is normalised.  valid (uint8[B, T]): padding is not read and becomes 0.  Returns the result; with residual also the sum
    (written to `total`); with training also float32[B, T(, heads), 2] for ``bload_layer_norm_backward``.  out may be x, total may be
    residual.  Asynchronous on the current stream."""
    shape, dtype, code = x.shape, x.dtype, _type_code(x)
    B, T, H, D = _row_sizes(shape)
    if residual is None and total is not None:
        raise ValueError("total is the sum with a residual")
    hx = _rows(x, shape, dtype, "x")
    out, ho = _new(x, shape, D) if out is None else (out, _rows(out, shape, dtype, "out"))
    hr = hs = None
    if residual is not None:
        hr = _rows(residual, shape, dtype, "residual")
        total, hs = _new(x, shape, D) if total is None else (total, _rows(total, shape, dtype, "total"))
    stats = x.new_empty((*shape[:-1], 2), dtype=torch.float32) if training else None
    _check(_lib.bload_layer_norm(hx, hr, _sized(valid, (B, T), torch.uint8, "valid"), B, T, H, D, code, int(center), eps,
                                 _sized(weight, (D,), torch.float32, "weight"), _sized(bias, (D,), torch.float32, "bias"), ho, hs,
                                 stats.data_ptr() if training else 0, _stream()))
    result = (out,) if residual is None else (out, total)
    if training:
        result += (stats,)
    return result if len(result) > 1 else out


def bload_layer_norm_backward_workspace_bytes(num_blocks: int, t_blk: int, heads: int, dim: int, dtype: torch.dtype) -> int:
    return int(_lib.bload_layer_norm_backward_workspace_bytes(num_blocks, t_blk, heads, dim, TYPE_CODE[dtype]))


def bload_layer_norm_backward(dout: torch.Tensor, x: torch.Tensor, stats: torch.Tensor, weight: torch.Tensor | None = None,
                              valid: torch.Tensor | None = None, dsum: torch.Tensor | None = None, center: bool = True, grads=None,
                              workspace: torch.Tensor | None = None):
    """Gradients (dx, dweight, dbias) of sum(out * dout) + sum(total * dsum); x is what was normalised: the forward call's x, or its
    sum where it had a residual.  dx is the gradient of both then.  grads: three tensors to write into, the last two float32[D] or None
    to leave them out.  Asynchronous on the current stream."""
    shape, dtype, code = x.shape, x.dtype, _type_code(x)
    B, T, H, D = _row_sizes(shape)
    real, hx = torch.float32, _rows(x, shape, dtype, "x")
    if grads is None:
        dx, hdx = _new(x, shape, D)
        dweight, dbias = x.new_empty(D, dtype=real), x.new_empty(D, dtype=real)
        pw, pb = dweight.data_ptr(), dbias.data_ptr()
    else:
        dx, dweight, dbias = grads
        hdx, pw, pb = _rows(dx, shape, dtype, "dx"), _sized(dweight, (D,), real, "dweight"), _sized(dbias, (D,), real, "dbias")
    if workspace is None and (dweight is not None or dbias is not None):
        need = _lib.bload_layer_norm_backward_workspace_bytes(B, T, H, D, code)
        workspace = torch.empty(max(16, need), dtype=torch.uint8, device=x.device)
    _check(_lib.bload_layer_norm_backward(
        _rows(dout, shape, dtype, "dout"), hx, _sized(stats, (*shape[:-1], 2), real, "stats"), _sized(valid, (B, T), torch.uint8, "valid"),
        B, T, H, D, code, int(center), _sized(weight, (D,), real, "weight"), None if dsum is None else _rows(dsum, shape, dtype, "dsum"),
        hdx, pw, pb, _ptr(workspace), _room(workspace), _stream()))
    return dx, dweight, dbias


def bload_segment_conv(x: torch.Tensor, weight: torch.Tensor, reset: torch.Tensor, valid: torch.Tensor, bias: torch.Tensor | None = None,
                       silu: bool = False, state_in: torch.Tensor | None = None, out: torch.Tensor | None = None,
                       state: torch.Tensor | None = None):
    """A short causal convolution of every feature inside the sequences of packed blocks, with silu p / (1 + e^-p) of it; 0 on padding.
    x: [B, T, D] of float16, bfloat16 or float32, any strides with the features of a slot side by side; weight: float32[D, taps],
    taps up to 8, the last one for the slot itself; bias: float32[D]; state_in: [B, taps - 1, D] like x, the inputs in front of the
    blocks, the oldest first.  Returns the result and the last inputs of every block, written to `state`, which may be state_in where
    T <= 8 and is refused where it meets state_in in any other way.  Asynchronous on the current stream."""
    B, T, D = shape = x.shape
    dtype, code, K = x.dtype, _type_code(x), weight.shape[-1]
    hx = _frames(x, shape, dtype, "x")
    out, ho = _new(x, shape, D) if out is None else (out, _frames(out, shape, dtype, "out"))
    if state is None:
        state = x.new_empty((B, K - 1, D))
    _check(_lib.bload_segment_conv(hx, _sized(weight, (D, K), torch.float32, "weight"), _sized(bias, (D,), torch.float32, "bias"),
                                   _sized(reset, (B, T), torch.uint8, "reset"), _sized(valid, (B, T), torch.uint8, "valid"), B, T, D, K,
                                   code, int(silu), _sized(state_in, (B, K - 1, D), dtype, "state_in"), ho,
                                   _sized(state, (B, K - 1, D), dtype, "state"), _stream()))
    return out, state


def bload_segment_conv_backward_workspace_bytes(num_blocks: int, t_blk: int, feat_dim: int, taps: int, dtype: torch.dtype) -> int:
    return int(_lib.bload_segment_conv_backward_workspace_bytes(num_blocks, t_blk, feat_dim, taps, TYPE_CODE[dtype]))


def bload_segment_conv_backward(dout: torch.Tensor, x: torch.Tensor, weight: torch.Tensor, reset: torch.Tensor, valid: torch.Tensor,
                                bias: torch.Tensor | None = None, silu: bool = False, state_in: torch.Tensor | None = None,
                                dstate: torch.Tensor | None = None, grads=None, workspace: torch.Tensor | None = None):
    """Gradients (dx, dweight, dbias, dstate_in) of sum(out * dout) + sum(state * dstate).  grads: four tensors to write into, the
    last three None to leave them out.  Asynchronous on the current stream."""
    B, T, D = shape = x.shape
    dtype, code, K, real = x.dtype, _type_code(x), weight.shape[-1], torch.float32
    hx = _frames(x, shape, dtype, "x")
    if grads is None:
        dx, hdx = _new(x, shape, D)
        dweight, dbias, dstate_in = x.new_empty((D, K), dtype=real), x.new_empty(D, dtype=real), x.new_empty((B, K - 1, D))
        pw, pb, ps = dweight.data_ptr(), dbias.data_ptr(), dstate_in.data_ptr()
    else:
        dx, dweight, dbias, dstate_in = grads
        hdx, pw, pb = _frames(dx, shape, dtype, "dx"), _sized(dweight, (D, K), real, "dweight"), _sized(dbias, (D,), real, "dbias")
        ps = _sized(dstate_in, (B, K - 1, D), dtype, "dstate_in")
    if workspace is None and (dweight is not None or dbias is not None):
        need = _lib.bload_segment_conv_backward_workspace_bytes(B, T, D, K, code)
        workspace = torch.empty(max(16, need), dtype=torch.uint8, device=x.device)
    _check(_lib.bload_segment_conv_backward(
        _frames(dout, shape, dtype, "dout"), hx, _sized(weight, (D, K), real, "weight"), _sized(bias, (D,), real, "bias"),
        _sized(reset, (B, T), torch.uint8, "reset"), _sized(valid, (B, T), torch.uint8, "valid"), B, T, D, K, code, int(silu),
        _sized(state_in, (B, K - 1, D), dtype, "state_in"), _sized(dstate, (B, K - 1, D), dtype, "dstate"), hdx, pw, pb, ps,
        _ptr(workspace), _room(workspace), _stream()))
    return dx, dweight, dbias, dstate_in


def bload_selective_scan_workspace_bytes(num_blocks: int, t_blk: int, feat_dim: int, states: int, groups: int = 1) -> int:
    return int(_lib.bload_selective_scan_workspace_bytes(num_blocks, t_blk, feat_dim, states, groups))


def bload_selective_scan_saved_bytes(num_blocks: int, t_blk: int, feat_dim: int, states: int, groups: int = 1) -> int:
    return int(_lib.bload_selective_scan_saved_bytes(num_blocks, t_blk, feat_dim, states, groups))


def bload_selective_scan_backward_workspace_bytes(num_blocks: int, t_blk: int, feat_dim: int, states: int, groups: int = 1) -> int:
    return int(_lib.bload_selective_scan_backward_workspace_bytes(num_blocks, t_blk, feat_dim, states, groups))


def _selective(x, dt, rate, b, c, reset, valid, skip, z, dt_bias, softplus, h0) -> Selective:
    B, T, D = shape = x.shape
    dtype, code = x.dtype, _type_code(x)
    if b.dim() != 4:
        raise ValueError("b: expected [B, T, groups, states]")
    G, N = b.shape[2:]
    pair = (B, T, G, N)
    return Selective(_frames(x, shape, dtype, "x"), _frames(dt, shape, dtype, "dt"),
                     Heads() if z is None else _frames(z, shape, dtype, "z"), _heads(b, pair, dtype, "b"), _heads(c, pair, dtype, "c"),
                     _sized(rate, (D, N), torch.float32, "rate"), _sized(skip, (D,), torch.float32, "skip"),
                     _sized(dt_bias, (D,), torch.float32, "dt_bias"), _sized(reset, (B, T), torch.uint8, "reset"),
                     _sized(valid, (B, T), torch.uint8, "valid"), _sized(h0, (B, D, N), torch.float32, "h0"), B, T, D, N, G, code,
                     int(softplus))


def bload_selective_scan(x: torch.Tensor, dt: torch.Tensor, rate: torch.Tensor, b: torch.Tensor, c: torch.Tensor, reset: torch.Tensor,
                         valid: torch.Tensor, skip: torch.Tensor | None = None, z: torch.Tensor | None = None,
                         dt_bias: torch.Tensor | None = None, softplus: bool = True, h0: torch.Tensor | None = None,
                         training: bool = False, out: torch.Tensor | None = None, state: torch.Tensor | None = None,
                         workspace: torch.Tensor | None = None):
    """A selective state space inside the sequences of packed blocks: step = softplus(dt + dt_bias), h = e^(step rate) h + step b x,
    y = c.h + skip x, times z sigmoid(z).  x, dt, z: [B, T, D] and b, c: [B, T, groups, N] of float16, bfloat16 or
    float32, any strides with the elements of a row side by side; rate: float32[D, N], N up to 64; skip, dt_bias: float32[D];
    h0: float32[B, D, N], the state in front of the blocks.  Returns the result and the state behind the last slots (float32[B, D, N]),
    written to `state`, which may be h0 where T <= 8 and is refused where it meets h0 in any other way; with training also what
    ``bload_selective_scan_backward`` needs.  Asynchronous on the current stream."""
    B, T, D = shape = x.shape
    s = _selective(x, dt, rate, b, c, reset, valid, skip, z, dt_bias, softplus, h0)
    N, G = s.states, s.groups
    out, ho = _new(x, shape, D) if out is None else (out, _frames(out, shape, x.dtype, "out"))
    if state is None:
        state = x.new_empty((B, D, N), dtype=torch.float32)
        ps = state.data_ptr()
    else:
        ps = _sized(state, (B, D, N), torch.float32, "state")
    saved = x.new_empty((B, -(-T // 16), D, N), dtype=torch.float32) if training else None
    if workspace is None:
        need = _lib.bload_selective_scan_workspace_bytes(B, T, D, N, G)
        workspace = torch.empty(need, dtype=torch.uint8, device=x.device) if need else None
    _check(_lib.bload_selective_scan(s, ho, ps, saved.data_ptr() if training else 0, _ptr(workspace), _room(workspace), _stream()))
    return (out, state, saved) if training else (out, state)


def bload_selective_scan_backward(dout: torch.Tensor, x: torch.Tensor, dt: torch.Tensor, rate: torch.Tensor, b: torch.Tensor,
                                  c: torch.Tensor, reset: torch.Tensor, valid: torch.Tensor, saved: torch.Tensor,
                                  skip: torch.Tensor | None = None, z: torch.Tensor | None = None, dt_bias: torch.Tensor | None = None,
                                  softplus: bool = True, h0: torch.Tensor | None = None, dstate: torch.Tensor | None = None, grads=None,
                                  workspace: torch.Tensor | None = None):
    """Gradients (dx, ddt, drate, db, dc, dskip, dz, ddt_bias, dh0) of sum(out * dout) + sum(state * dstate), None in the place of
    inputs that are None; saved is the forward call's.  grads: nine tensors to write into, None for drate, dskip, ddt_bias and dh0
    to leave them out.  Asynchronous on the current stream."""
    B, T, D = shape = x.shape
    s = _selective(x, dt, rate, b, c, reset, valid, skip, z, dt_bias, softplus, h0)
    N, G, dtype, real = s.states, s.groups, x.dtype, torch.float32
    if grads is None:
        floats = lambda t: None if t is None else x.new_empty(t.shape, dtype=real)
        (dx, hx), (ddt, hdt), (db, hb), (dc, hc) = _new(x, shape, D), _new(x, shape, D), _new(x, b.shape, N), _new(x, b.shape, N)
        dz, hz = (None, None) if z is None else _new(x, shape, D)
        drate, dskip, ddt_bias, dh0 = floats(rate), floats(skip), floats(dt_bias), floats(h0)
        pr, pk, pb, ph = (0 if t is None else t.data_ptr() for t in (drate, dskip, ddt_bias, dh0))
    else:
        dx, ddt, drate, db, dc, dskip, dz, ddt_bias, dh0 = grads
        pair = (B, T, G, N)
        hx, hdt = _frames(dx, shape, dtype, "dx"), _frames(ddt, shape, dtype, "ddt")
        hb, hc, hz = _heads(db, pair, dtype, "db"), _heads(dc, pair, dtype, "dc"), None if z is None else _frames(dz, shape, dtype, "dz")
        pr, pk = _sized(drate, (D, N), real, "drate"), _sized(dskip, (D,), real, "dskip")
        pb, ph = _sized(ddt_bias, (D,), real, "ddt_bias"), _sized(dh0, (B, D, N), real, "dh0")
    if workspace is None:
        need = _lib.bload_selective_scan_backward_workspace_bytes(B, T, D, N, G)
        workspace = torch.empty(max(16, need), dtype=torch.uint8, device=x.device)
    _check(_lib.bload_selective_scan_backward(
        s, _frames(dout, shape, dtype, "dout"), _sized(saved, (B, -(-T // 16), D, N), real, "saved"), _sized(dstate, (B, D, N), real, "dstate"),
        hx, hdt, pr, hb, hc, pk, hz, pb, ph, _ptr(workspace), _room(workspace), _stream()))
    return dx, ddt, drate, db, dc, dskip, dz, ddt_bias, dh0
