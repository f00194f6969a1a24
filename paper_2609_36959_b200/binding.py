"""ctypes binding of libcobalt.so: same names as the C ABI, argument marshalling only.

Every step of the routing path runs in the library's CUDA kernels.  torch is used for device
memory and streams: tensors are passed as raw device pointers and the current torch stream is
the stream the kernels are enqueued on.  There is no CPU fallback: if the shared library is
missing or a call fails, a CobaltError is raised.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libcobalt.so")

OK = 0
ERR_INVALID_ARG = -1
ERR_WORKSPACE_TOO_SMALL = -2
ERR_UNSUPPORTED = -3
ERR_CUDA = -4
ERR_SCRATCH_LIMIT = -5
ERR_HOST_ALLOC = -6
STATIC_SCRATCH_WORDS = 1 << 20

DEVERR_BAD_EXPERT_ID = 0x1
DEVERR_DUPLICATE_ID = 0x2
DEVERR_BAD_SRC_RANK = 0x4
DEVERR_BAD_SLOT = 0x8
DEVERR_WAIT_TIMEOUT = 0x10

STATS_ACCUMULATE = 0x1
ASSIGN_NAIVE = 0x1
ASSIGN_ROUND_ROBIN = 0x2
SEED_ON_DEVICE = 0x4
STATS_TILE16 = 0x10
STATS_TILE32 = 0x20
ROUTE_SEPARATE_KERNELS = 0x40
EMA_INITIALISE = 0x1
GATE_SIGMOID = 0x1
BF16, F32, E4M3, I8 = 0, 1, 2, 3
ACTIVATIONS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3}
PACK_GROUP = 128
IMPL_VECTOR = 0x100
IMPL_BULK = 0x200

# every symbol include/cobalt.h declares
EXPORTS = (
    "cobalt_status_string", "cobalt_version", "cobalt_last_cuda_error",
    "cobalt_layout_check", "cobalt_layout_create", "cobalt_layout_destroy", "cobalt_layout_num_dests",
    "cobalt_coact_stats_workspace_bytes", "cobalt_coact_stats",
    "cobalt_assign_workspace_bytes", "cobalt_assign",
    "cobalt_permute_workspace_bytes", "cobalt_permute_index", "cobalt_permute_rows", "cobalt_permute",
    "cobalt_permute_index_static", "cobalt_permute_rows_block", "cobalt_combine_block",
    "cobalt_route_index_workspace_bytes", "cobalt_route_index",
    "cobalt_permute_backward", "cobalt_combine_backward",
    "cobalt_ema_update", "cobalt_ochiai", "cobalt_rebalance_intra_node",
    "cobalt_dedup_workspace_bytes", "cobalt_dedup_index", "cobalt_forward_rows",
    "cobalt_combine", "cobalt_read_and_clear_device_error",
    "cobalt_layer_norm", "cobalt_layer_norm_workspace_bytes", "cobalt_layer_norm_backward",
    "cobalt_gate_topk", "cobalt_gate_topk_backward",
    "cobalt_expert_ffn_workspace_bytes", "cobalt_expert_ffn", "cobalt_expert_ffn_backward",
    "cobalt_dropout_add", "cobalt_dropout_add_backward",
    "cobalt_pack_rows", "cobalt_unpack_rows",
    "cobalt_rms_norm", "cobalt_rms_norm_workspace_bytes", "cobalt_rms_norm_backward",
    "cobalt_linear_workspace_bytes", "cobalt_linear", "cobalt_linear_backward",
)


class CobaltError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: {status_string(status)} (status {status}, cuda error {last_cuda_error()})")


def _load() -> C.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2609_36959_b200.build` "
            "(there is no fallback path)")
    lib = C.CDLL(LIB_PATH)
    vp, i32, i64, u32, u64, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_uint32, C.c_uint64, C.c_size_t
    sig = {
        "cobalt_status_string": (C.c_char_p, [C.c_int]),
        "cobalt_version": (C.c_int, []),
        "cobalt_last_cuda_error": (C.c_int, []),
        "cobalt_layout_check": (C.c_int, [i32, i32, i32, i32, vp, vp]),
        "cobalt_layout_create": (C.c_int, [C.POINTER(vp), i32, i32, i32, i32, vp, vp]),
        "cobalt_layout_destroy": (C.c_int, [vp]),
        "cobalt_layout_num_dests": (i32, [vp]),
        "cobalt_coact_stats_workspace_bytes": (sz, [i64, i32, i32]),
        "cobalt_coact_stats": (C.c_int, [vp, i64, i32, i32, vp, vp, u32, vp, sz, vp]),
        "cobalt_assign_workspace_bytes": (sz, [vp, i64, i32]),
        "cobalt_assign": (C.c_int, [vp, vp, vp, i32, i64, i32, u64, vp, vp, vp, vp, u32, vp, sz, vp]),
        "cobalt_permute_workspace_bytes": (sz, [i64, i32, i32]),
        "cobalt_permute_index": (C.c_int, [vp, i64, i32, i32, vp, vp, vp, vp, vp, sz, vp]),
        "cobalt_permute_index_static": (C.c_int, [vp, i64, i32, i32, vp, vp, vp, vp, vp]),
        "cobalt_permute_rows": (C.c_int, [vp, vp, i64, i32, i32, vp, u32, vp]),
        "cobalt_permute": (C.c_int, [vp, i64, i32, i32, vp, i32, vp, vp, vp, vp, vp, u32, vp, sz, vp]),
        "cobalt_combine": (C.c_int, [vp, vp, vp, i64, i32, i32, vp, u32, vp]),
        "cobalt_route_index_workspace_bytes": (sz, [vp, i64, i32]),
        "cobalt_route_index": (C.c_int, [vp, vp, vp, i32, i64, i32, u64, vp, vp, vp, vp, vp, vp, vp, vp, vp, u32, vp,
                                         sz, vp]),
        "cobalt_permute_backward": (C.c_int, [vp, vp, i64, i32, i32, vp, u32, vp]),
        "cobalt_combine_backward": (C.c_int, [vp, vp, vp, vp, i64, i32, i32, vp, vp, u32, vp]),
        "cobalt_ema_update": (C.c_int, [vp, vp, i64, C.c_float, u32, vp]),
        "cobalt_ochiai": (C.c_int, [vp, i32, vp, vp]),
        "cobalt_rebalance_intra_node": (C.c_int, [i32, i32, i32, i32, vp, vp, vp, vp, vp]),
        "cobalt_dedup_workspace_bytes": (sz, [i64, i32, i32]),
        "cobalt_dedup_index": (C.c_int, [vp, vp, i32, i64, i32, i32, i32, i32, vp, vp, vp, vp, vp, vp, sz, vp]),
        "cobalt_forward_rows": (C.c_int, [vp, vp, vp, i64, i32, vp, i64, i64, vp]),
        "cobalt_permute_rows_block": (C.c_int, [vp, vp, i64, i32, i32, vp, i64, u32, vp]),
        "cobalt_combine_block": (C.c_int, [vp, vp, vp, i64, i32, i32, vp, i64, u32, vp]),
        "cobalt_layer_norm": (C.c_int, [vp, vp, vp, i64, i32, i32, C.c_float, vp, vp, vp, vp]),
        "cobalt_layer_norm_workspace_bytes": (sz, [i64, i32]),
        "cobalt_layer_norm_backward": (C.c_int, [vp, vp, vp, vp, vp, i64, i32, i32, vp, vp, vp, vp, sz, vp]),
        "cobalt_gate_topk": (C.c_int, [vp, i64, i32, i32, i32, vp, vp, u32, vp]),
        "cobalt_gate_topk_backward": (C.c_int, [vp, vp, vp, vp, i64, i32, i32, i32, vp, u32, vp]),
        "cobalt_expert_ffn_workspace_bytes": (sz, [i64, i32, i32, i32, i32]),
        "cobalt_expert_ffn": (C.c_int, [vp, vp, vp, i64, i32, i32, i32, i32, vp, vp, vp, vp, vp, vp, sz, vp]),
        "cobalt_expert_ffn_backward": (C.c_int, [vp, vp, vp, vp, i64, i32, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp,
                                                 sz, vp]),
        "cobalt_dropout_add": (C.c_int, [vp, vp, i64, i32, C.c_double, u64, vp, u32, vp]),
        "cobalt_dropout_add_backward": (C.c_int, [vp, i64, i32, C.c_double, u64, vp, u32, vp]),
        "cobalt_pack_rows": (C.c_int, [vp, i64, i32, i32, i32, i32, vp, vp, vp]),
        "cobalt_unpack_rows": (C.c_int, [vp, vp, i64, i32, i32, i32, i32, vp, vp]),
        "cobalt_rms_norm": (C.c_int, [vp, vp, vp, i64, i32, i32, C.c_float, vp, vp, vp, vp, i32, i32, vp, vp]),
        "cobalt_rms_norm_workspace_bytes": (sz, [i64, i32]),
        "cobalt_rms_norm_backward": (C.c_int, [vp, vp, vp, vp, i32, i32, vp, vp, i64, i32, i32, vp, vp, vp, sz, vp]),
        "cobalt_linear_workspace_bytes": (sz, [i64, i32, i32]),
        "cobalt_linear": (C.c_int, [vp, vp, vp, vp, vp, vp, i64, i32, i32, i32, i32, i32, vp, vp, i32, vp, vp, sz, vp]),
        "cobalt_linear_backward": (C.c_int, [vp, vp, vp, vp, vp, i32, i64, i32, i32, i32, i32, vp, vp, vp, vp, vp, sz, vp]),
        "cobalt_read_and_clear_device_error": (C.c_int, [C.POINTER(u32), vp]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    return lib


_lib = _load()


def status_string(status: int) -> str:
    return _lib.cobalt_status_string(status).decode()


def version() -> int:
    return _lib.cobalt_version()


def last_cuda_error() -> int:
    return _lib.cobalt_last_cuda_error()


def _check(status: int, what: str) -> None:
    if status != OK:
        raise CobaltError(status, what)


def _ptr(t: Optional[torch.Tensor], dtype: Optional[torch.dtype] = None, what: str = "tensor") -> Optional[int]:
    if t is None:
        return None
    if not t.is_cuda:
        raise TypeError(f"{what} must be a CUDA tensor")
    if not t.is_contiguous():
        raise TypeError(f"{what} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{what} must be {dtype}, got {t.dtype}")
    return t.data_ptr()


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream() -> int:
    """Handle of torch's current stream on the current device (the raw query costs a fraction of a
    microsecond; building a torch.cuda.Stream object for it costs about three)."""
    if _raw_stream is not None:
        return _raw_stream(torch.cuda.current_device())
    return torch.cuda.current_stream().cuda_stream


def _seed_arg(seed, flags: int):
    """A Python int is passed by value; a one-element int64 CUDA tensor is passed by address and read
    by the kernel when it runs (COBALT_SEED_ON_DEVICE), which lets a captured graph be replayed with
    another seed."""
    if isinstance(seed, torch.Tensor):
        if seed.numel() != 1:
            raise TypeError("a seed tensor must have one element")
        return _ptr(seed, torch.int64, "seed"), flags | SEED_ON_DEVICE
    return seed & (2**64 - 1), flags


def _host_i32(a) -> "C.Array":
    vals = [int(v) for v in a]
    return (C.c_int32 * len(vals))(*vals)


def layout_check(N: int, Q: int, S: int, E: int, slot_expert, primary_slot=None) -> int:
    """Host-only validation of a layout; returns the status code (no device needed)."""
    se = _host_i32(slot_expert)
    if len(se) != N * Q * S:
        return ERR_INVALID_ARG
    pr = None if primary_slot is None else _host_i32(primary_slot)
    if pr is not None and len(pr) != E:
        return ERR_INVALID_ARG
    return _lib.cobalt_layout_check(N, Q, S, E, se, pr)


class Layout:
    """Owns a cobalt_layout_t (device tables of R_{e,n}, N_e and the primaries)."""

    def __init__(self, N: int, Q: int, S: int, E: int, slot_expert, primary_slot=None):
        se = _host_i32(slot_expert)
        if len(se) != N * Q * S:
            raise CobaltError(ERR_INVALID_ARG, "layout_create (slot_expert size)")
        pr = None if primary_slot is None else _host_i32(primary_slot)
        if pr is not None and len(pr) != E:
            raise CobaltError(ERR_INVALID_ARG, "layout_create (primary_slot size)")
        handle = C.c_void_p()
        _check(_lib.cobalt_layout_create(C.byref(handle), N, Q, S, E, se, pr), "cobalt_layout_create")
        self._h = handle
        self.N, self.Q, self.S, self.E = N, Q, S, E
        self.G, self.D = N * Q, N * Q * S

    @property
    def handle(self) -> C.c_void_p:
        if self._h is None:
            raise CobaltError(ERR_INVALID_ARG, "layout already destroyed")
        return self._h

    def destroy(self) -> None:
        if getattr(self, "_h", None) is not None:
            h, self._h = self._h, None
            _check(_lib.cobalt_layout_destroy(h), "cobalt_layout_destroy")

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def coact_stats_workspace_bytes(T: int, K: int, E: int) -> int:
    return _lib.cobalt_coact_stats_workspace_bytes(T, K, E)


def coact_stats(topk_ids: torch.Tensor, E: int, coact: torch.Tensor, load: torch.Tensor, *,
                flags: int = 0, workspace: Optional[torch.Tensor] = None) -> None:
    T, K = topk_ids.shape
    if coact.numel() != E * E or load.numel() != E:
        raise CobaltError(ERR_INVALID_ARG, "coact_stats (output sizes)")
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(_lib.cobalt_coact_stats(_ptr(topk_ids, torch.int32, "topk_ids"), T, K, E,
                                   _ptr(coact, torch.int32, "coact"), _ptr(load, torch.int32, "load"), flags,
                                   _ptr(workspace), ws_bytes, _stream()), "cobalt_coact_stats")


def assign_workspace_bytes(layout: Layout, T: int, K: int) -> int:
    return _lib.cobalt_assign_workspace_bytes(layout.handle, T, K)


def assign(layout: Layout, topk_ids: torch.Tensor, src_rank, seed: int, assigned_slot: torch.Tensor, *,
           slot_load: Optional[torch.Tensor] = None, remote_nodes: Optional[torch.Tensor] = None,
           totals: Optional[torch.Tensor] = None, flags: int = 0,
           workspace: Optional[torch.Tensor] = None) -> None:
    """src_rank: int32 tensor [T], or a Python int used for every token.  seed: a Python int, or a
    one-element int64 CUDA tensor read when the kernel runs."""
    T, K = topk_ids.shape
    if assigned_slot.numel() != T * K:
        raise CobaltError(ERR_INVALID_ARG, "assign (assigned_slot size)")
    if slot_load is not None and slot_load.numel() != layout.D:
        raise CobaltError(ERR_INVALID_ARG, "assign (slot_load size)")
    if remote_nodes is not None and remote_nodes.numel() != T:
        raise CobaltError(ERR_INVALID_ARG, "assign (remote_nodes size)")
    if totals is not None and totals.numel() != 2:
        raise CobaltError(ERR_INVALID_ARG, "assign (totals size)")
    if isinstance(src_rank, int):
        src_ptr, src_uniform = None, src_rank
    else:
        if src_rank.numel() != T:
            raise CobaltError(ERR_INVALID_ARG, "assign (src_rank size)")
        src_ptr, src_uniform = _ptr(src_rank, torch.int32, "src_rank"), 0
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    seed, flags = _seed_arg(seed, flags)
    _check(_lib.cobalt_assign(layout.handle, _ptr(topk_ids, torch.int32, "topk_ids"), src_ptr, src_uniform,
                              T, K, seed, _ptr(assigned_slot, torch.int32, "assigned_slot"),
                              _ptr(slot_load, torch.int32, "slot_load"),
                              _ptr(remote_nodes, torch.uint8, "remote_nodes"),
                              _ptr(totals, torch.int64, "totals"), flags, _ptr(workspace), ws_bytes,
                              _stream()), "cobalt_assign")


def route_index_workspace_bytes(layout: Layout, T: int, K: int) -> int:
    return _lib.cobalt_route_index_workspace_bytes(layout.handle, T, K)


def route_index(layout: Layout, topk_ids: torch.Tensor, src_rank, seed: int, coact: torch.Tensor,
                load: torch.Tensor, assigned_slot: torch.Tensor, dest_counts: torch.Tensor,
                dest_offsets: torch.Tensor, row_of_pair: torch.Tensor, workspace: torch.Tensor, *,
                remote_nodes: Optional[torch.Tensor] = None, totals: Optional[torch.Tensor] = None,
                pair_of_row: Optional[torch.Tensor] = None, flags: int = 0) -> None:
    """Statistics, assignment and the permutation index in one pass over the ids."""
    T, K = topk_ids.shape
    E, D = layout.E, layout.D
    if coact.numel() != E * E or load.numel() != E or assigned_slot.numel() != T * K:
        raise CobaltError(ERR_INVALID_ARG, "route_index (output sizes)")
    _check_index_outputs(T, K, D, dest_counts, dest_offsets, row_of_pair, pair_of_row, "route_index")
    if remote_nodes is not None and remote_nodes.numel() != T:
        raise CobaltError(ERR_INVALID_ARG, "route_index (remote_nodes size)")
    if totals is not None and totals.numel() != 2:
        raise CobaltError(ERR_INVALID_ARG, "route_index (totals size)")
    if isinstance(src_rank, int):
        src_ptr, src_uniform = None, src_rank
    else:
        if src_rank.numel() != T:
            raise CobaltError(ERR_INVALID_ARG, "route_index (src_rank size)")
        src_ptr, src_uniform = _ptr(src_rank, torch.int32, "src_rank"), 0
    seed, flags = _seed_arg(seed, flags)
    _check(_lib.cobalt_route_index(layout.handle, _ptr(topk_ids, torch.int32, "topk_ids"), src_ptr, src_uniform, T, K,
                                   seed, _ptr(coact, torch.int32, "coact"),
                                   _ptr(load, torch.int32, "load"), _ptr(assigned_slot, torch.int32, "assigned_slot"),
                                   _ptr(remote_nodes, torch.uint8, "remote_nodes"), _ptr(totals, torch.int64, "totals"),
                                   _ptr(dest_counts, torch.int32, "dest_counts"),
                                   _ptr(dest_offsets, torch.int32, "dest_offsets"),
                                   _ptr(row_of_pair, torch.int32, "row_of_pair"),
                                   _ptr(pair_of_row, torch.int32, "pair_of_row"), flags, _ptr(workspace),
                                   _ws_bytes(workspace), _stream()), "cobalt_route_index")


def permute_workspace_bytes(T: int, K: int, D: int) -> int:
    return _lib.cobalt_permute_workspace_bytes(T, K, D)


def _ws_bytes(workspace: Optional[torch.Tensor]) -> int:
    return 0 if workspace is None else workspace.numel() * workspace.element_size()


def _check_index_outputs(T, K, D, dest_counts, dest_offsets, row_of_pair, pair_of_row, what):
    if dest_counts.numel() != D or dest_offsets.numel() != D + 1 or row_of_pair.numel() != T * K or (
            pair_of_row is not None and pair_of_row.numel() != T * K):
        raise CobaltError(ERR_INVALID_ARG, f"{what} (output sizes)")


def permute_index(assigned_slot: torch.Tensor, D: int, dest_counts: torch.Tensor, dest_offsets: torch.Tensor,
                  row_of_pair: torch.Tensor, pair_of_row: Optional[torch.Tensor],
                  workspace: torch.Tensor) -> None:
    T, K = assigned_slot.shape
    _check_index_outputs(T, K, D, dest_counts, dest_offsets, row_of_pair, pair_of_row, "permute_index")
    _check(_lib.cobalt_permute_index(_ptr(assigned_slot, torch.int32, "assigned_slot"), T, K, D,
                                     _ptr(dest_counts, torch.int32, "dest_counts"),
                                     _ptr(dest_offsets, torch.int32, "dest_offsets"),
                                     _ptr(row_of_pair, torch.int32, "row_of_pair"),
                                     _ptr(pair_of_row, torch.int32, "pair_of_row"),
                                     _ptr(workspace), _ws_bytes(workspace), _stream()), "cobalt_permute_index")


def permute_index_static(assigned_slot: torch.Tensor, D: int, dest_counts: torch.Tensor,
                         dest_offsets: torch.Tensor, row_of_pair: torch.Tensor,
                         pair_of_row: Optional[torch.Tensor]) -> None:
    """permute_index for callers that cannot hand over device scratch (a framework hot path that
    bans allocator calls, a plugin given only its inputs and outputs, a fully committed memory
    pool): the scratch is a fixed 4 MiB array inside the library.  Same outputs as
    permute_index; raises with ERR_SCRATCH_LIMIT when D * chunks exceeds STATIC_SCRATCH_WORDS.
    Calls share that array, so do not let two of them overlap on the GPU; make the first call
    on a device outside stream capture (it looks up the array's address)."""
    T, K = assigned_slot.shape
    _check_index_outputs(T, K, D, dest_counts, dest_offsets, row_of_pair, pair_of_row, "permute_index_static")
    _check(_lib.cobalt_permute_index_static(_ptr(assigned_slot, torch.int32, "assigned_slot"), T, K, D,
                                            _ptr(dest_counts, torch.int32, "dest_counts"),
                                            _ptr(dest_offsets, torch.int32, "dest_offsets"),
                                            _ptr(row_of_pair, torch.int32, "row_of_pair"),
                                            _ptr(pair_of_row, torch.int32, "pair_of_row"), _stream()),
           "cobalt_permute_index_static")


def permute_rows(x: torch.Tensor, row_of_pair: torch.Tensor, K: int, send: torch.Tensor, *, flags: int = 0) -> None:
    T, H = x.shape
    if row_of_pair.numel() != T * K or send.numel() != T * K * H:
        raise CobaltError(ERR_INVALID_ARG, "permute_rows (sizes)")
    _check(_lib.cobalt_permute_rows(_ptr(x, torch.bfloat16, "x"), _ptr(row_of_pair, torch.int32, "row_of_pair"),
                                    T, K, H, _ptr(send, torch.bfloat16, "send"), flags, _stream()),
           "cobalt_permute_rows")


def permute(assigned_slot: torch.Tensor, D: int, x: torch.Tensor, send: torch.Tensor, dest_counts: torch.Tensor,
            dest_offsets: torch.Tensor, row_of_pair: torch.Tensor, pair_of_row: Optional[torch.Tensor],
            workspace: torch.Tensor, *, flags: int = 0) -> None:
    T, K = assigned_slot.shape
    H = x.shape[1]
    if x.shape[0] != T or send.numel() != T * K * H:
        raise CobaltError(ERR_INVALID_ARG, "permute (x / send sizes)")
    _check_index_outputs(T, K, D, dest_counts, dest_offsets, row_of_pair, pair_of_row, "permute")
    _check(_lib.cobalt_permute(_ptr(assigned_slot, torch.int32, "assigned_slot"), T, K, D,
                               _ptr(x, torch.bfloat16, "x"), H, _ptr(send, torch.bfloat16, "send"),
                               _ptr(dest_counts, torch.int32, "dest_counts"),
                               _ptr(dest_offsets, torch.int32, "dest_offsets"),
                               _ptr(row_of_pair, torch.int32, "row_of_pair"),
                               _ptr(pair_of_row, torch.int32, "pair_of_row"), flags,
                               _ptr(workspace), _ws_bytes(workspace), _stream()), "cobalt_permute")


def combine(expert_out: torch.Tensor, row_of_pair: torch.Tensor, gate_w: torch.Tensor, y: torch.Tensor, *,
            flags: int = 0) -> None:
    T, K = gate_w.shape
    H = y.shape[1]
    if y.shape[0] != T or expert_out.numel() != T * K * H or row_of_pair.numel() != T * K:
        raise CobaltError(ERR_INVALID_ARG, "combine (sizes)")
    _check(_lib.cobalt_combine(_ptr(expert_out, torch.bfloat16, "expert_out"),
                               _ptr(row_of_pair, torch.int32, "row_of_pair"),
                               _ptr(gate_w, torch.float32, "gate_w"), T, K, H, _ptr(y, torch.bfloat16, "y"),
                               flags, _stream()), "cobalt_combine")


def _elem_ptr(t: torch.Tensor, offset_elems: int) -> int:
    return t.data_ptr() + offset_elems * t.element_size()


def permute_rows_block(x: torch.Tensor, row_of_pair_block: torch.Tensor, K: int, send: torch.Tensor, t0: int,
                       t1: int, *, flags: int = 0) -> None:
    """cobalt_permute_rows on tokens t0:t1 only (x and send are the whole buffers; row_of_pair_block
    holds the rows of pairs t0*K : t1*K, which index the whole send buffer)."""
    T, H = x.shape
    if not (0 <= t0 <= t1 <= T) or row_of_pair_block.numel() != (t1 - t0) * K or send.numel() != T * K * H:
        raise CobaltError(ERR_INVALID_ARG, "permute_rows_block (sizes)")
    _ptr(x, torch.bfloat16, "x"), _ptr(send, torch.bfloat16, "send")
    _check(_lib.cobalt_permute_rows_block(_elem_ptr(x, t0 * H), _ptr(row_of_pair_block, torch.int32, "row_of_pair"),
                                          t1 - t0, K, H, send.data_ptr(), T * K, flags, _stream()),
           "cobalt_permute_rows_block")


def combine_block(expert_out: torch.Tensor, row_of_pair_block: torch.Tensor, gate_w: torch.Tensor,
                  y: torch.Tensor, t0: int, t1: int, *, flags: int = 0) -> None:
    """cobalt_combine on tokens t0:t1 only (expert_out is the whole [P, H] buffer)."""
    T, K = gate_w.shape
    H = y.shape[1]
    if not (0 <= t0 <= t1 <= T) or row_of_pair_block.numel() != (t1 - t0) * K or expert_out.numel() != T * K * H:
        raise CobaltError(ERR_INVALID_ARG, "combine_block (sizes)")
    _ptr(expert_out, torch.bfloat16, "expert_out"), _ptr(gate_w, torch.float32, "gate_w"), _ptr(y, torch.bfloat16, "y")
    _check(_lib.cobalt_combine_block(expert_out.data_ptr(), _ptr(row_of_pair_block, torch.int32, "row_of_pair"),
                                     _elem_ptr(gate_w, t0 * K), t1 - t0, K, H, _elem_ptr(y, t0 * H), T * K, flags,
                                     _stream()), "cobalt_combine_block")


def permute_backward(grad_send: torch.Tensor, row_of_pair: torch.Tensor, K: int, grad_x: torch.Tensor, *,
                     flags: int = 0) -> None:
    """grad_x[t] = sum of the K rows of grad_send that token t was sent to."""
    T, H = grad_x.shape
    if row_of_pair.numel() != T * K or grad_send.numel() != T * K * H:
        raise CobaltError(ERR_INVALID_ARG, "permute_backward (sizes)")
    _check(_lib.cobalt_permute_backward(_ptr(grad_send, torch.bfloat16, "grad_send"),
                                        _ptr(row_of_pair, torch.int32, "row_of_pair"), T, K, H,
                                        _ptr(grad_x, torch.bfloat16, "grad_x"), flags, _stream()),
           "cobalt_permute_backward")


def combine_backward(grad_y: torch.Tensor, expert_out: Optional[torch.Tensor], row_of_pair: torch.Tensor,
                     gate_w: torch.Tensor, grad_expert_out: Optional[torch.Tensor],
                     grad_gate_w: Optional[torch.Tensor], *, flags: int = 0) -> None:
    T, K = gate_w.shape
    H = grad_y.shape[1]
    if grad_y.shape[0] != T or row_of_pair.numel() != T * K:
        raise CobaltError(ERR_INVALID_ARG, "combine_backward (sizes)")
    for name, t in (("expert_out", expert_out), ("grad_expert_out", grad_expert_out)):
        if t is not None and t.numel() != T * K * H:
            raise CobaltError(ERR_INVALID_ARG, f"combine_backward ({name} size)")
    if grad_gate_w is not None and grad_gate_w.numel() != T * K:
        raise CobaltError(ERR_INVALID_ARG, "combine_backward (grad_gate_w size)")
    _check(_lib.cobalt_combine_backward(_ptr(grad_y, torch.bfloat16, "grad_y"),
                                        _ptr(expert_out, torch.bfloat16, "expert_out"),
                                        _ptr(row_of_pair, torch.int32, "row_of_pair"),
                                        _ptr(gate_w, torch.float32, "gate_w"), T, K, H,
                                        _ptr(grad_expert_out, torch.bfloat16, "grad_expert_out"),
                                        _ptr(grad_gate_w, torch.float32, "grad_gate_w"), flags, _stream()),
           "cobalt_combine_backward")


def ema_update(counts: torch.Tensor, ema: torch.Tensor, decay: float, *, flags: int = 0) -> None:
    """ema = decay * ema + (1 - decay) * counts, element-wise on the device (counts int32, ema float32)."""
    if counts.numel() != ema.numel():
        raise CobaltError(ERR_INVALID_ARG, "ema_update (sizes)")
    _check(_lib.cobalt_ema_update(_ptr(counts, torch.int32, "counts"), _ptr(ema, torch.float32, "ema"),
                                  counts.numel(), decay, flags, _stream()), "cobalt_ema_update")


def ochiai(coact: torch.Tensor, out: torch.Tensor) -> None:
    E = coact.shape[0]
    if coact.numel() != E * E or out.numel() != E * E:
        raise CobaltError(ERR_INVALID_ARG, "ochiai (sizes)")
    _check(_lib.cobalt_ochiai(_ptr(coact, torch.int32, "coact"), E, _ptr(out, torch.float32, "ochiai"), _stream()),
           "cobalt_ochiai")


def rebalance_intra_node(N: int, Q: int, S: int, E: int, slot_expert, slot_load):
    """Stage-2 greedy rebalancing on host arrays -> (new_slot_expert, moved_from, nodes_kept) as Python lists/int."""
    D = N * Q * S
    se = _host_i32(slot_expert)
    ld = (C.c_float * D)(*[float(v) for v in slot_load])
    if len(se) != D:
        raise CobaltError(ERR_INVALID_ARG, "rebalance_intra_node (slot_expert size)")
    new = (C.c_int32 * D)()
    moved = (C.c_int32 * D)()
    kept = C.c_int32(0)
    _check(_lib.cobalt_rebalance_intra_node(N, Q, S, E, se, ld, new, moved, C.byref(kept)),
           "cobalt_rebalance_intra_node")
    return list(new), list(moved), int(kept.value)


def dedup_workspace_bytes(T: int, K: int, N: int) -> int:
    return _lib.cobalt_dedup_workspace_bytes(T, K, N)


def dedup_index(assigned_slot: torch.Tensor, src_rank, N: int, Q: int, S: int, node_counts: torch.Tensor,
                node_offsets: torch.Tensor, node_row_of_token: torch.Tensor, fwd_src_row: torch.Tensor,
                workspace: torch.Tensor, *, cross_node_rows: Optional[torch.Tensor] = None) -> None:
    """One row per (token, destination node): see cobalt_dedup_index."""
    T, K = assigned_slot.shape
    if (node_counts.numel() != N or node_offsets.numel() != N + 1 or node_row_of_token.numel() != T * N or
            fwd_src_row.numel() != T * K or (cross_node_rows is not None and cross_node_rows.numel() != 1)):
        raise CobaltError(ERR_INVALID_ARG, "dedup_index (output sizes)")
    if isinstance(src_rank, int):
        src_ptr, src_uniform = None, src_rank
    else:
        src_ptr, src_uniform = _ptr(src_rank, torch.int32, "src_rank"), 0
    _check(_lib.cobalt_dedup_index(_ptr(assigned_slot, torch.int32, "assigned_slot"), src_ptr, src_uniform, T, K,
                                   N, Q, S, _ptr(node_counts, torch.int32, "node_counts"),
                                   _ptr(node_offsets, torch.int32, "node_offsets"),
                                   _ptr(node_row_of_token, torch.int32, "node_row_of_token"),
                                   _ptr(fwd_src_row, torch.int32, "fwd_src_row"),
                                   _ptr(cross_node_rows, torch.int64, "cross_node_rows"), _ptr(workspace),
                                   _ws_bytes(workspace), _stream()), "cobalt_dedup_index")


def dedup_rows(x: torch.Tensor, node_row_of_token: torch.Tensor, N: int, dedup_send: torch.Tensor, *,
               flags: int = 0) -> None:
    """Fill the deduplicated buffer: the row mover with N optional copies per token."""
    T, H = x.shape
    if node_row_of_token.numel() != T * N or dedup_send.shape[1] != H:
        raise CobaltError(ERR_INVALID_ARG, "dedup_rows (sizes)")
    _check(_lib.cobalt_permute_rows_block(_ptr(x, torch.bfloat16, "x"),
                                          _ptr(node_row_of_token, torch.int32, "node_row_of_token"), T, N, H,
                                          _ptr(dedup_send, torch.bfloat16, "dedup_send"), dedup_send.shape[0], flags,
                                          _stream()), "cobalt_permute_rows_block")


def forward_rows(dedup_send: torch.Tensor, fwd_src_row: torch.Tensor, row_of_pair: torch.Tensor,
                 recv: torch.Tensor) -> None:
    """recv[row_of_pair[p]] = dedup_send[fwd_src_row[p]]."""
    P = fwd_src_row.numel()
    H = dedup_send.shape[1]
    if row_of_pair.numel() != P or recv.shape[1] != H:
        raise CobaltError(ERR_INVALID_ARG, "forward_rows (sizes)")
    _check(_lib.cobalt_forward_rows(_ptr(dedup_send, torch.bfloat16, "dedup_send"),
                                    _ptr(fwd_src_row, torch.int32, "fwd_src_row"),
                                    _ptr(row_of_pair, torch.int32, "row_of_pair"), P, H,
                                    _ptr(recv, torch.bfloat16, "recv"), dedup_send.shape[0], recv.shape[0], _stream()),
           "cobalt_forward_rows")


# ---- the layer around the routed rows ------------------------------------------------------

_DTYPES = {torch.bfloat16: BF16, torch.float32: F32}


def _dtype_code(t: torch.Tensor, what: str) -> int:
    code = _DTYPES.get(t.dtype)
    if code is None:
        raise TypeError(f"{what} must be bfloat16 or float32, got {t.dtype}")
    return code


def layer_norm(x: torch.Tensor, gamma: torch.Tensor, beta: torch.Tensor, eps: float, y: torch.Tensor,
               mean: torch.Tensor, rstd: torch.Tensor) -> None:
    """y = (x - mean) * rstd * gamma + beta over the rows of x [T, H] (bfloat16 or float32; gamma, beta float32 [H]).
    mean and rstd (float32 [T]) are kept for layer_norm_backward."""
    T, H = x.shape
    code = _dtype_code(x, "x")
    if gamma.numel() != H or beta.numel() != H or y.shape != x.shape or mean.numel() != T or rstd.numel() != T:
        raise CobaltError(ERR_INVALID_ARG, "layer_norm (sizes)")
    _check(_lib.cobalt_layer_norm(_ptr(x, None, "x"), _ptr(gamma, torch.float32, "gamma"), _ptr(beta, torch.float32, "beta"),
                                  T, H, code, eps, _ptr(y, x.dtype, "y"), _ptr(mean, torch.float32, "mean"),
                                  _ptr(rstd, torch.float32, "rstd"), _stream()), "cobalt_layer_norm")


def layer_norm_workspace_bytes(T: int, H: int) -> int:
    return _lib.cobalt_layer_norm_workspace_bytes(T, H)


def layer_norm_backward(grad_y: torch.Tensor, x: torch.Tensor, gamma: torch.Tensor, mean: torch.Tensor,
                        rstd: torch.Tensor, grad_x: torch.Tensor, grad_gamma: torch.Tensor, grad_beta: torch.Tensor,
                        workspace: torch.Tensor) -> None:
    """Gradients of layer_norm: grad_x like x, grad_gamma and grad_beta float32 [H] (overwritten)."""
    T, H = x.shape
    code = _dtype_code(x, "x")
    if (grad_y.shape != x.shape or grad_x.shape != x.shape or gamma.numel() != H or mean.numel() != T or
            rstd.numel() != T or grad_gamma.numel() != H or grad_beta.numel() != H):
        raise CobaltError(ERR_INVALID_ARG, "layer_norm_backward (sizes)")
    _check(_lib.cobalt_layer_norm_backward(_ptr(grad_y, x.dtype, "grad_y"), _ptr(x, None, "x"),
                                           _ptr(gamma, torch.float32, "gamma"), _ptr(mean, torch.float32, "mean"),
                                           _ptr(rstd, torch.float32, "rstd"), T, H, code, _ptr(grad_x, x.dtype, "grad_x"),
                                           _ptr(grad_gamma, torch.float32, "grad_gamma"),
                                           _ptr(grad_beta, torch.float32, "grad_beta"), _ptr(workspace),
                                           _ws_bytes(workspace), _stream()), "cobalt_layer_norm_backward")


def gate_topk(logits: torch.Tensor, topk_ids: torch.Tensor, gate_w: torch.Tensor, *, flags: int = 0) -> None:
    """The K largest logits of each token (descending, ties to the lowest id) and their weights: softmax over the
    chosen, or with flags=GATE_SIGMOID their sigmoids divided by the sum.  logits [T, E] bfloat16 or float32;
    topk_ids int32 [T, K] and gate_w float32 [T, K] are the gating output that the routing stages take."""
    T, E = logits.shape
    code = _dtype_code(logits, "logits")
    if topk_ids.dim() != 2 or topk_ids.shape[0] != T or gate_w.shape != topk_ids.shape:
        raise CobaltError(ERR_INVALID_ARG, "gate_topk (output sizes)")
    _check(_lib.cobalt_gate_topk(_ptr(logits, None, "logits"), T, E, topk_ids.shape[1], code,
                                 _ptr(topk_ids, torch.int32, "topk_ids"), _ptr(gate_w, torch.float32, "gate_w"), flags,
                                 _stream()), "cobalt_gate_topk")


def gate_topk_backward(grad_gate_w: torch.Tensor, logits: torch.Tensor, topk_ids: torch.Tensor, gate_w: torch.Tensor,
                       grad_logits: torch.Tensor, *, flags: int = 0) -> None:
    """grad_logits [T, E] (like logits) from grad_gate_w [T, K], e.g. that of combine_backward."""
    T, E = logits.shape
    code = _dtype_code(logits, "logits")
    if (topk_ids.dim() != 2 or topk_ids.shape[0] != T or gate_w.shape != topk_ids.shape or
            grad_gate_w.shape != topk_ids.shape or grad_logits.shape != logits.shape):
        raise CobaltError(ERR_INVALID_ARG, "gate_topk_backward (sizes)")
    _check(_lib.cobalt_gate_topk_backward(_ptr(grad_gate_w, torch.float32, "grad_gate_w"), _ptr(logits, None, "logits"),
                                          _ptr(topk_ids, torch.int32, "topk_ids"), _ptr(gate_w, torch.float32, "gate_w"),
                                          T, E, topk_ids.shape[1], code, _ptr(grad_logits, logits.dtype, "grad_logits"),
                                          flags, _stream()), "cobalt_gate_topk_backward")


def expert_ffn_workspace_bytes(P: int, D: int, E: int, H: int, F: int) -> int:
    return _lib.cobalt_expert_ffn_workspace_bytes(P, D, E, H, F)


def _ffn_sizes(rows, dest_offsets, slot_expert, w_gate_up, w_down, what):
    P, H = rows.shape
    if w_down.dim() != 3 or w_gate_up.dim() != 3:
        raise CobaltError(ERR_INVALID_ARG, f"{what} (weights must be [E, 2F, H] and [E, H, F])")
    E, F = w_down.shape[0], w_down.shape[2]
    D = slot_expert.numel()
    if tuple(w_gate_up.shape) != (E, 2 * F, H) or w_down.shape[1] != H or dest_offsets.numel() != D + 1:
        raise CobaltError(ERR_INVALID_ARG, f"{what} (sizes)")
    return P, H, E, F, D


def _ffn_buffer(t: Optional[torch.Tensor], shape, what: str) -> Optional[int]:
    if t is not None and tuple(t.shape) != tuple(shape):
        raise CobaltError(ERR_INVALID_ARG, f"{what} (size)")
    return _ptr(t, torch.bfloat16, what)


def expert_ffn(rows: torch.Tensor, dest_offsets: torch.Tensor, slot_expert: torch.Tensor, w_gate_up: torch.Tensor,
               w_down: torch.Tensor, act: torch.Tensor, out: torch.Tensor, workspace: torch.Tensor, *,
               pre: Optional[torch.Tensor] = None) -> None:
    """out = (silu(x Wg^T) * (x Wu^T)) Wd^T for the rows of every slot, with the weights of the slot's expert.

    rows, out bfloat16 [P, H] in the order of the send buffer; dest_offsets int32 [D+1] and slot_expert int32 [D] on
    the device; w_gate_up [E, 2F, H] (gate rows first), w_down [E, H, F].  act [P, F] and, if a backward pass follows,
    pre [P, 2F] are written and kept for expert_ffn_backward (pre holds 16-bit codes of the library's own, not bfloat16
    values)."""
    P, H, E, F, D = _ffn_sizes(rows, dest_offsets, slot_expert, w_gate_up, w_down, "expert_ffn")
    _check(_lib.cobalt_expert_ffn(_ptr(rows, torch.bfloat16, "rows"), _ptr(dest_offsets, torch.int32, "dest_offsets"),
                                  _ptr(slot_expert, torch.int32, "slot_expert"), P, D, E, H, F,
                                  _ptr(w_gate_up, torch.bfloat16, "w_gate_up"), _ptr(w_down, torch.bfloat16, "w_down"),
                                  _ffn_buffer(act, (P, F), "act"), _ffn_buffer(pre, (P, 2 * F), "pre"),
                                  _ffn_buffer(out, (P, H), "out"), _ptr(workspace), _ws_bytes(workspace), _stream()),
           "cobalt_expert_ffn")


def expert_ffn_backward(grad_out: torch.Tensor, rows: torch.Tensor, dest_offsets: torch.Tensor, slot_expert: torch.Tensor,
                        w_gate_up: torch.Tensor, w_down: torch.Tensor, pre: torch.Tensor, act: torch.Tensor,
                        grad_pre: torch.Tensor, workspace: torch.Tensor, *, grad_rows: Optional[torch.Tensor] = None,
                        grad_w_gate_up: Optional[torch.Tensor] = None,
                        grad_w_down: Optional[torch.Tensor] = None) -> None:
    """Gradients of expert_ffn from grad_out [P, H] and the act and pre of the forward call.  grad_pre [P, 2F] is
    scratch and may be `pre`.  Each of the three results may be left out; weight gradients are overwritten."""
    P, H, E, F, D = _ffn_sizes(rows, dest_offsets, slot_expert, w_gate_up, w_down, "expert_ffn_backward")
    _check(_lib.cobalt_expert_ffn_backward(
        _ffn_buffer(grad_out, (P, H), "grad_out"), _ptr(rows, torch.bfloat16, "rows"),
        _ptr(dest_offsets, torch.int32, "dest_offsets"), _ptr(slot_expert, torch.int32, "slot_expert"), P, D, E, H, F,
        _ptr(w_gate_up, torch.bfloat16, "w_gate_up"), _ptr(w_down, torch.bfloat16, "w_down"),
        _ffn_buffer(pre, (P, 2 * F), "pre"), _ffn_buffer(act, (P, F), "act"), _ffn_buffer(grad_pre, (P, 2 * F), "grad_pre"),
        _ffn_buffer(grad_rows, (P, H), "grad_rows"), _ffn_buffer(grad_w_gate_up, (E, 2 * F, H), "grad_w_gate_up"),
        _ffn_buffer(grad_w_down, (E, H, F), "grad_w_down"), _ptr(workspace), _ws_bytes(workspace), _stream()),
        "cobalt_expert_ffn_backward")


def dropout_add(x: torch.Tensor, residual: Optional[torch.Tensor], p: float, seed, out: torch.Tensor) -> None:
    """out = residual + dropout(x) (residual None: dropout alone), bfloat16 or float32.  The mask is a function of
    (seed, element index) and is drawn again by dropout_add_backward; seed as in assign: an int, or a one-element
    int64 CUDA tensor read when the kernel runs."""
    code = _dtype_code(x, "x")
    if out.shape != x.shape or (residual is not None and residual.shape != x.shape):
        raise CobaltError(ERR_INVALID_ARG, "dropout_add (sizes)")
    seed, flags = _seed_arg(seed, 0)
    _check(_lib.cobalt_dropout_add(_ptr(x, None, "x"), _ptr(residual, x.dtype, "residual"), x.numel(), code, p, seed,
                                   _ptr(out, x.dtype, "out"), flags, _stream()), "cobalt_dropout_add")


def dropout_add_backward(grad_out: torch.Tensor, p: float, seed, grad_x: torch.Tensor) -> None:
    """grad_x = grad_out * scale where dropout_add with this p and seed kept the element, 0 elsewhere."""
    code = _dtype_code(grad_out, "grad_out")
    if grad_x.shape != grad_out.shape:
        raise CobaltError(ERR_INVALID_ARG, "dropout_add_backward (sizes)")
    seed, flags = _seed_arg(seed, 0)
    _check(_lib.cobalt_dropout_add_backward(_ptr(grad_out, None, "grad_out"), grad_out.numel(), code, p, seed,
                                            _ptr(grad_x, grad_out.dtype, "grad_x"), flags, _stream()),
           "cobalt_dropout_add_backward")


# ---- the dense part of a layer --------------------------------------------------------------
# These calls are a few microseconds of GPU time for a token or two, so the checks query every tensor once.

_CODES = {torch.float8_e4m3fn: E4M3, torch.int8: I8}
_get_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _current_device() -> int:
    try:
        return _get_device()
    except RuntimeError:                         # no driver: no tensor is there either
        return -2


def _here(t: Optional[torch.Tensor], device: int, dtype: torch.dtype, shape, what: str) -> Optional[int]:
    """The pointer of a contiguous tensor of this type and shape on this device."""
    if t is None:
        return None
    if t.get_device() == device and t.dtype is dtype and t.shape == shape and t.is_contiguous():
        return t.data_ptr()
    if not t.is_cuda:
        raise TypeError(f"{what} must be a CUDA tensor")
    if t.dtype != dtype:
        raise TypeError(f"{what} must be {dtype}, got {t.dtype}")
    if t.shape != shape:
        raise CobaltError(ERR_INVALID_ARG, f"{what} (size {tuple(t.shape)}, not {tuple(shape)})")
    if not t.is_contiguous():
        raise TypeError(f"{what} must be contiguous")
    raise CobaltError(ERR_INVALID_ARG, f"{what} (on device {t.get_device()}, the current one is {device})")


def _workspace(t: torch.Tensor, device: int) -> int:
    if t.get_device() != device or not t.is_contiguous():
        raise TypeError("workspace must be a contiguous tensor on the current device")
    return t.data_ptr()


def _stream_on(device: int) -> int:
    return _raw_stream(device) if _raw_stream is not None else torch.cuda.current_stream().cuda_stream


def _packed(packed, device: int, T: int, H: int, what: str):
    """(codes pointer, scales pointer, code, group) of rows in 8 bits: codes float8_e4m3fn or int8 [T, H], scales float32 with
    one value a row ([T] or [T, 1]) or one for each 128 columns ([T, ceil(H / 128)])."""
    q, scales = packed
    code = _CODES.get(q.dtype)
    if code is None:
        raise TypeError(f"{what} must be float8_e4m3fn or int8, got {q.dtype}")
    groups = -(-H // PACK_GROUP)
    size = scales.shape
    if len(size) == 2 and size[1] == groups:
        group = PACK_GROUP if groups > 1 else 0
    elif len(size) == 1 or (len(size) == 2 and size[1] == 1):
        group = 0
    else:
        raise CobaltError(ERR_INVALID_ARG, f"{what} scales (size {tuple(size)})")
    if size[0] != T:
        raise CobaltError(ERR_INVALID_ARG, f"{what} scales (size {tuple(size)})")
    return _here(q, device, q.dtype, (T, H), what), _here(scales, device, torch.float32, size, what), code, group


def pack_rows(x: torch.Tensor, q: torch.Tensor, scales: torch.Tensor) -> None:
    """Rows of x [T, H] (bfloat16 or float32) in 8 bits: q float8_e4m3fn or int8 [T, H], scales float32, one a row ([T] or
    [T, 1]) or one for each 128 columns ([T, ceil(H / 128)]).  A group's largest absolute value becomes the largest code."""
    shape, device = x.shape, _current_device()
    T, H = shape
    q_ptr, scales_ptr, code, group = _packed((q, scales), device, T, H, "q")
    _check(_lib.cobalt_pack_rows(_here(x, device, x.dtype, shape, "x"), T, H, _dtype_code(x, "x"), code, group, q_ptr, scales_ptr,
                                 _stream_on(device)), "cobalt_pack_rows")


def unpack_rows(q: torch.Tensor, scales: torch.Tensor, out: torch.Tensor) -> None:
    """out [T, H] (bfloat16 or float32) = the values of rows that pack_rows (or rms_norm, or linear) left in 8 bits."""
    shape, device = out.shape, _current_device()
    T, H = shape
    q_ptr, scales_ptr, code, group = _packed((q, scales), device, T, H, "q")
    _check(_lib.cobalt_unpack_rows(q_ptr, scales_ptr, T, H, code, group, _dtype_code(out, "out"),
                                   _here(out, device, out.dtype, shape, "out"), _stream_on(device)), "cobalt_unpack_rows")


def rms_norm(x: torch.Tensor, gamma: torch.Tensor, eps: float, *, residual: Optional[torch.Tensor] = None,
             sum_out: Optional[torch.Tensor] = None, y: Optional[torch.Tensor] = None, packed=None,
             rstd: Optional[torch.Tensor] = None) -> None:
    """y = s * rstd * gamma over the rows of s = x + residual [T, H] (bfloat16 or float32, s in the same type; gamma float32
    [H]).  Written where given: the sum, y, packed = (q, scales) with y in 8 bits as in pack_rows, and rstd float32 [T] for
    rms_norm_backward."""
    shape, dtype, device = x.shape, x.dtype, _current_device()
    T, H = shape
    q_ptr, scales_ptr, q_code, group = (None, None, 0, 0) if packed is None else _packed(packed, device, T, H, "packed")
    _check(_lib.cobalt_rms_norm(_here(x, device, dtype, shape, "x"), _here(residual, device, dtype, shape, "residual"),
                                _here(gamma, device, torch.float32, (H,), "gamma"), T, H, _dtype_code(x, "x"), eps,
                                _here(sum_out, device, dtype, shape, "sum_out"), _here(y, device, dtype, shape, "y"), q_ptr, scales_ptr,
                                q_code, group, _here(rstd, device, torch.float32, (T,), "rstd"), _stream_on(device)), "cobalt_rms_norm")


def rms_norm_workspace_bytes(T: int, H: int) -> int:
    return _lib.cobalt_rms_norm_workspace_bytes(T, H)


def rms_norm_backward(grad_y: torch.Tensor, rows, gamma: torch.Tensor, rstd: torch.Tensor, grad_x: torch.Tensor,
                      grad_gamma: torch.Tensor, workspace: torch.Tensor, *, grad_sum: Optional[torch.Tensor] = None) -> None:
    """Gradients of rms_norm: grad_x [T, H] (of x and of residual alike) and grad_gamma float32 [H].  rows is the sum that was
    normalised, or (q, scales) as pack_rows left it; grad_sum is the gradient that reaches the sum past the norm."""
    shape, dtype, device = grad_y.shape, grad_y.dtype, _current_device()
    T, H = shape
    code = _dtype_code(grad_y, "grad_y")
    if isinstance(rows, tuple):
        rows_ptr, scales_ptr, rows_type, group = _packed(rows, device, T, H, "rows")
    else:
        rows_ptr, scales_ptr, rows_type, group = _here(rows, device, dtype, shape, "rows"), None, code, 0
    _check(_lib.cobalt_rms_norm_backward(_here(grad_y, device, dtype, shape, "grad_y"), _here(grad_sum, device, dtype, shape, "grad_sum"),
                                         rows_ptr, scales_ptr, rows_type, group, _here(gamma, device, torch.float32, (H,), "gamma"),
                                         _here(rstd, device, torch.float32, (T,), "rstd"), T, H, code,
                                         _here(grad_x, device, dtype, shape, "grad_x"),
                                         _here(grad_gamma, device, torch.float32, (H,), "grad_gamma"), _workspace(workspace, device),
                                         _ws_bytes(workspace),
                                         _stream_on(device)), "cobalt_rms_norm_backward")


def linear_workspace_bytes(T: int, K: int, N: int) -> int:
    """For linear and linear_backward on x [T, K] and w [N, K]; what T tokens need serves fewer."""
    return _lib.cobalt_linear_workspace_bytes(T, K, N)


def _activation(act: str) -> int:
    code = ACTIVATIONS.get(act)
    if code is None:
        raise ValueError(f"act must be one of {', '.join(ACTIVATIONS)}, got {act!r}")
    return code


def _pre(pre, device: int, T: int, N: int, what: str):
    if pre is None:
        return None, None, BF16
    if isinstance(pre, tuple):
        q_ptr, scales_ptr, code, group = _packed(pre, device, T, N, "pre")
        if code != I8 or (group == 0 and N > PACK_GROUP):
            raise CobaltError(ERR_INVALID_ARG, f"{what} (pre in 8 bits is int8 with a scale for each 128 columns)")
        return q_ptr, scales_ptr, I8
    return _here(pre, device, torch.bfloat16, (T, N), "pre"), None, BF16


def linear(x, w, out: torch.Tensor, workspace: torch.Tensor, *, bias: Optional[torch.Tensor] = None,
           residual: Optional[torch.Tensor] = None, act: str = "none", pre=None) -> None:
    """out [T, N] (bfloat16 or float32) = act(x w^T + bias) + residual.

    x [T, K] and w [N, K] are both bfloat16, or both (q, scales) in float8_e4m3fn with one scale a row, as pack_rows and
    rms_norm leave them.  bias bfloat16 [N]; residual like out.  act: none, relu, silu or gelu.  pre, where a backward pass
    follows an activation: bfloat16 [T, N], or (int8 [T, N], float32 [T, ceil(N / 128)]) to keep it in 8 bits."""
    shape, device = out.shape, _current_device()
    T, N = shape
    if isinstance(x, tuple) != isinstance(w, tuple):
        raise TypeError("x and w must both be bfloat16, or both (q, scales)")
    if isinstance(x, tuple):
        K = x[0].shape[1]
        x_ptr, x_scales, code, group = _packed(x, device, T, K, "x")
        w_ptr, w_scales, w_code, w_group = _packed(w, device, N, K, "w")
        if (code, group, w_code, w_group) != (E4M3, 0, E4M3, 0):
            raise CobaltError(ERR_INVALID_ARG, "linear (8-bit operands are float8_e4m3fn with one scale a row)")
    else:
        K = x.shape[1]
        x_ptr, x_scales, code = _here(x, device, torch.bfloat16, (T, K), "x"), None, BF16
        w_ptr, w_scales = _here(w, device, torch.bfloat16, (N, K), "w"), None
    pre_ptr, pre_scales, pre_type = _pre(pre, device, T, N, "linear")
    _check(_lib.cobalt_linear(x_ptr, x_scales, w_ptr, w_scales, _here(bias, device, torch.bfloat16, (N,), "bias"),
                              _here(residual, device, out.dtype, shape, "residual"), T, K, N, code, _activation(act), _dtype_code(out, "out"),
                              pre_ptr, pre_scales, pre_type, _here(out, device, out.dtype, shape, "out"), _workspace(workspace, device),
                              _ws_bytes(workspace), _stream_on(device)), "cobalt_linear")


def linear_backward(grad_out: torch.Tensor, x: Optional[torch.Tensor], w: Optional[torch.Tensor], workspace: torch.Tensor, *,
                    act: str = "none", pre=None, grad_pre: Optional[torch.Tensor] = None, grad_x: Optional[torch.Tensor] = None,
                    grad_w: Optional[torch.Tensor] = None, grad_bias: Optional[torch.Tensor] = None) -> None:
    """Gradients of linear for bfloat16 x and w, from grad_out [T, N] (bfloat16 or float32) and the pre of the forward call:
    grad_x [T, K], grad_w [N, K], grad_bias [N], bfloat16, each of which may be left out (x is read for grad_w, w for grad_x).
    grad_pre [T, N] bfloat16 is scratch, needed with an activation or a float32 grad_out; it may be a bfloat16 grad_out."""
    shape, device = grad_out.shape, _current_device()
    T, N = shape
    K = next((t.shape[1] for t in (x, w, grad_x, grad_w) if t is not None), 8)
    pre_ptr, pre_scales, pre_type = _pre(pre, device, T, N, "linear_backward")
    bf16 = torch.bfloat16
    _check(_lib.cobalt_linear_backward(_here(grad_out, device, grad_out.dtype, shape, "grad_out"), _here(x, device, bf16, (T, K), "x"),
                                       _here(w, device, bf16, (N, K), "w"),
                                       pre_ptr, pre_scales, pre_type, T, K, N, _activation(act), _dtype_code(grad_out, "grad_out"),
                                       _here(grad_pre, device, bf16, shape, "grad_pre"), _here(grad_x, device, bf16, (T, K), "grad_x"),
                                       _here(grad_w, device, bf16, (N, K), "grad_w"), _here(grad_bias, device, bf16, (N,), "grad_bias"), _workspace(workspace, device),
                                       _ws_bytes(workspace), _stream_on(device)), "cobalt_linear_backward")


def read_and_clear_device_error() -> int:
    bits = C.c_uint32(0)
    _check(_lib.cobalt_read_and_clear_device_error(C.byref(bits), _stream()),
           "cobalt_read_and_clear_device_error")
    return int(bits.value)
