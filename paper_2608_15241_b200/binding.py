"""Thin ctypes binding of the C-ABI library (include/lora_mixed_linear.h).

Argument marshalling only: every step of the layer runs in the library's CUDA kernels.
PyTorch supplies device memory and streams.  There is no CPU fallback: if the shared
library is missing, or a call returns an error status, this module raises.

Module-level functions carry the C names (lml_table_create, register_adapter,
retire_version, lml_segment_tokens, lora_mixed_linear, ...) and take raw pointers/ints;
`Table` wraps them for torch tensors.
"""
from __future__ import annotations

import ctypes
import operator
import os
from typing import Optional, Tuple

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "liblora_mixed_linear.so")

LML_OK = 0
STATUS_NAMES = {0: "LML_OK", 1: "LML_ERR_INVALID_ARG", 2: "LML_ERR_BAD_SLOT", 3: "LML_ERR_TABLE_FULL",
                4: "LML_ERR_DUPLICATE", 5: "LML_ERR_NOT_FOUND", 6: "LML_ERR_UNSUPPORTED",
                7: "LML_ERR_CUDA", 8: "LML_ERR_TIMEOUT", 9: "LML_ERR_WORKSPACE", 10: "LML_ERR_TOO_LARGE"}
FLAG_BAD_SLOT, FLAG_BAD_OFFSETS, FLAG_BAD_PERM, FLAG_TIMEOUT = 1, 2, 4, 8
MAX_SLOTS, MAX_RANK, DECODE_MAX_TOKENS, MAX_ADAPTER_IDS = 64, 64, 16, 4096
ERR_INVALID_ARG, ERR_BAD_SLOT, ERR_NOT_FOUND = 1, 2, 5

EXPORTS = ("lml_status_string", "lml_table_create", "lml_table_destroy", "register_adapter",
           "retire_version", "lml_lookup", "lml_slot_info", "lml_workspace_bytes",
           "lml_segment_tokens", "lora_mixed_linear", "lml_host_workspace_bytes",
           "lora_mixed_linear_host", "lml_device_status", "lml_last_launch_count",
           "lora_mixed_linear_decode_static", "lml_tokens_workspace_bytes", "lora_mixed_linear_tokens",
           "lml_publish", "lml_pin", "lml_unpin", "lml_resolve", "lml_slot_state",
           "lml_segment_tokens_adapters", "lora_mixed_linear_adapters",
           "lml_dual_workspace_bytes", "lora_mixed_linear_dual", "register_adapter_transposed",
           "lml_backward_workspace_bytes", "lora_mixed_linear_backward_adapters", "retire_version_on",
           "lml_multi_workspace_bytes", "lora_mixed_linear_multi", "lml_checkpoint_data_bytes", "lml_checkpoint_scale_bytes",
           "lml_checkpoint_store", "lml_checkpoint_load", "lml_backward_rows_workspace_bytes",
           "lora_mixed_linear_backward_adapters_rows", "lml_block_norm", "lml_block_norm_workspace_bytes",
           "lml_block_norm_backward")
ROWS_BF16, ROWS_INT8, ROWS_E4M3 = 0, 1, 2
ROW_FORMS = {"bf16": ROWS_BF16, "int8": ROWS_INT8, "e4m3": ROWS_E4M3}
MAX_NORM_WIDTH = 16384


class Rows(ctypes.Structure):
    """lml_rows: rows of activations, bf16 or an 8-bit checkpoint."""
    _fields_ = [("data", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("format", ctypes.c_int)]


class BlockNormDesc(ctypes.Structure):
    """lml_block_norm_desc."""
    _fields_ = [("d", ctypes.c_int), ("eps", ctypes.c_float), ("scale", ctypes.c_float), ("w_post", ctypes.c_void_p),
                ("w_pre", ctypes.c_void_p), ("gate", ctypes.c_void_p)]


class LmlError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {STATUS_NAMES.get(status, status)}")


_lib = None


def lib() -> ctypes.CDLL:
    """Load the shared library; fails loudly when it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} not found: build it with "
                              "`python -m paper_2608_15241_b200.build` (there is no fallback path)")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
        L.lml_status_string.restype = ctypes.c_char_p
        L.lml_status_string.argtypes = [i32]
        L.lml_table_create.argtypes = [ctypes.POINTER(vp), i32, i32, i32, i32]
        L.lml_table_destroy.argtypes = [vp]
        L.register_adapter.argtypes = [vp, i32, i32, vp, vp, i32, ctypes.c_float, vp, ctypes.POINTER(i32)]
        L.retire_version.argtypes = [vp, i32, i32]
        L.retire_version_on.argtypes = [vp, i32, i32, vp]
        L.lml_lookup.argtypes = [vp, i32, i32, ctypes.POINTER(i32)]
        L.lml_slot_info.argtypes = [vp, i32, ctypes.POINTER(i32), ctypes.POINTER(i32), ctypes.POINTER(i32),
                                    ctypes.POINTER(ctypes.c_float)]
        L.lml_workspace_bytes.restype = sz
        L.lml_workspace_bytes.argtypes = [vp, i32, i32]
        L.lml_host_workspace_bytes.restype = sz
        L.lml_host_workspace_bytes.argtypes = [vp, i32, i32]
        L.lml_segment_tokens.argtypes = [vp, vp, i32, vp, vp, vp, vp]
        L.lora_mixed_linear.argtypes = [vp, vp, vp, i32, vp, vp, i32, vp, vp, vp, sz, vp]
        L.lora_mixed_linear_host.argtypes = [vp, vp, vp, i32, vp, vp, i32, vp, vp, vp, sz, vp]
        L.lora_mixed_linear_decode_static.argtypes = [vp, vp, vp, i32, vp, vp, i32, vp, vp, vp]
        L.lml_tokens_workspace_bytes.restype = sz
        L.lml_tokens_workspace_bytes.argtypes = [vp, i32]
        L.lora_mixed_linear_tokens.argtypes = [vp, vp, vp, i32, vp, vp, vp, sz, vp]
        L.lora_mixed_linear_adapters.argtypes = [vp, vp, vp, i32, vp, vp, vp, sz, vp]
        L.lml_segment_tokens_adapters.argtypes = [vp, vp, i32, vp, vp, vp, vp]
        L.register_adapter_transposed.argtypes = [vp, i32, i32, vp, vp, i32, ctypes.c_float, vp, ctypes.POINTER(i32)]
        L.lml_backward_workspace_bytes.restype = sz
        L.lml_backward_workspace_bytes.argtypes = [vp, i32, i32]
        L.lora_mixed_linear_backward_adapters.argtypes = [vp, vp, vp, vp, i32, vp, vp, vp, i32, vp, vp, vp, sz, vp]
        L.lml_dual_workspace_bytes.restype = sz
        L.lml_dual_workspace_bytes.argtypes = [vp, i32, i32]
        L.lora_mixed_linear_dual.argtypes = [vp, vp, vp, i32, vp, vp, vp, i32, vp, vp, vp, vp, sz, vp]
        L.lml_multi_workspace_bytes.restype = sz
        L.lml_multi_workspace_bytes.argtypes = [ctypes.POINTER(vp), i32, i32]
        L.lora_mixed_linear_multi.argtypes = [ctypes.POINTER(vp), i32, vp, ctypes.POINTER(vp), i32, ctypes.POINTER(vp),
                                              ctypes.POINTER(vp), vp, sz, vp]
        rows, desc = ctypes.POINTER(Rows), ctypes.POINTER(BlockNormDesc)
        L.lml_checkpoint_data_bytes.argtypes = [i32, i32]
        L.lml_checkpoint_scale_bytes.argtypes = [i32, i32]
        L.lml_checkpoint_store.argtypes = [i32, vp, i32, i32, rows, vp]
        L.lml_checkpoint_load.argtypes = [i32, rows, i32, i32, vp, vp]
        L.lml_backward_rows_workspace_bytes.argtypes = [vp, i32, i32]
        L.lora_mixed_linear_backward_adapters_rows.argtypes = [vp, vp, rows, vp, i32, vp, vp, vp, i32, vp, vp, i32, vp, sz, vp]
        L.lml_block_norm.argtypes = [i32, desc, i32, vp, vp, vp, vp, vp, rows, rows, vp]
        L.lml_block_norm_workspace_bytes.argtypes = [i32, i32, i32]
        L.lml_block_norm_backward.argtypes = [i32, desc, i32, rows, rows, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        for name in ("lml_checkpoint_data_bytes", "lml_checkpoint_scale_bytes", "lml_backward_rows_workspace_bytes",
                     "lml_block_norm_workspace_bytes"):
            getattr(L, name).restype = sz
        L.lml_publish.argtypes = [vp, i32, i32, vp, ctypes.POINTER(i32)]
        L.lml_pin.argtypes = [vp, i32]
        L.lml_unpin.argtypes = [vp, i32]
        L.lml_resolve.argtypes = [vp, i32, ctypes.POINTER(i32), ctypes.POINTER(i32)]
        L.lml_slot_state.argtypes = [vp, i32, ctypes.POINTER(i32), ctypes.POINTER(i32)]
        L.lml_device_status.argtypes = [vp, ctypes.POINTER(ctypes.c_uint32), vp]
        L.lml_last_launch_count.argtypes = [vp]
        for name in EXPORTS:
            if name not in ("lml_status_string", "lml_workspace_bytes", "lml_host_workspace_bytes",
                            "lml_tokens_workspace_bytes", "lml_dual_workspace_bytes", "lml_backward_workspace_bytes",
                            "lml_multi_workspace_bytes", "lml_checkpoint_data_bytes", "lml_checkpoint_scale_bytes",
                            "lml_backward_rows_workspace_bytes", "lml_block_norm_workspace_bytes"):
                getattr(L, name).restype = i32
        _lib = L
    return _lib


def _check(status: int, where: str) -> None:
    if status != LML_OK:
        raise LmlError(status, where)


# ---- C names, raw arguments ---------------------------------------------------------------------

def lml_status_string(status: int) -> str:
    return lib().lml_status_string(status).decode()


def lml_table_create(device: int, d_in: int, d_out: int, max_slots: int) -> int:
    h = ctypes.c_void_p()
    _check(lib().lml_table_create(ctypes.byref(h), device, d_in, d_out, max_slots), "lml_table_create")
    return h.value


def lml_table_destroy(table: int) -> None:
    _check(lib().lml_table_destroy(table), "lml_table_destroy")


def register_adapter(table: int, adapter_id: int, version: int, A_ptr: int, B_ptr: int, rank: int,
                     scale: float, stream: int = 0) -> int:
    slot = ctypes.c_int(-1)
    _check(lib().register_adapter(table, adapter_id, version, A_ptr, B_ptr, rank, scale, stream,
                                  ctypes.byref(slot)), "register_adapter")
    return slot.value


def retire_version(table: int, adapter_id: int, version: int) -> None:
    _check(lib().retire_version(table, adapter_id, version), "retire_version")


def retire_version_on(table: int, adapter_id: int, version: int, stream: int = 0) -> None:
    """retire_version whose device-side part (the serving entry leaves the adapter map) runs on `stream`."""
    _check(lib().retire_version_on(table, adapter_id, version, stream), "retire_version_on")


def lml_lookup(table: int, adapter_id: int, version: int) -> int:
    slot = ctypes.c_int(-1)
    _check(lib().lml_lookup(table, adapter_id, version, ctypes.byref(slot)), "lml_lookup")
    return slot.value


def lml_slot_info(table: int, slot: int) -> Tuple[int, int, int, float]:
    a, v, r, s = ctypes.c_int(), ctypes.c_int(), ctypes.c_int(), ctypes.c_float()
    _check(lib().lml_slot_info(table, slot, ctypes.byref(a), ctypes.byref(v), ctypes.byref(r), ctypes.byref(s)),
           "lml_slot_info")
    return a.value, v.value, r.value, s.value


def lml_workspace_bytes(table: int, max_tokens: int, max_segments: int) -> int:
    return int(lib().lml_workspace_bytes(table, max_tokens, max_segments))


def lml_host_workspace_bytes(table: int, max_tokens: int, max_segments: int) -> int:
    return int(lib().lml_host_workspace_bytes(table, max_tokens, max_segments))


def lml_segment_tokens(table: int, token_slots_ptr: int, T: int, perm_ptr: int, seg_offsets_ptr: int,
                       seg_slot_ids_ptr: int, stream: int = 0) -> None:
    _check(lib().lml_segment_tokens(table, token_slots_ptr, T, perm_ptr, seg_offsets_ptr, seg_slot_ids_ptr,
                                    stream), "lml_segment_tokens")


def lora_mixed_linear(table: int, x_ptr: int, W0_ptr: int, T: int, seg_offsets_ptr: int, slot_ids_ptr: int,
                      G: int, perm_ptr: int, y_ptr: int, workspace_ptr: int, workspace_bytes: int,
                      stream: int = 0) -> None:
    _check(lib().lora_mixed_linear(table, x_ptr, W0_ptr, T, seg_offsets_ptr, slot_ids_ptr, G, perm_ptr, y_ptr,
                                   workspace_ptr, workspace_bytes, stream), "lora_mixed_linear")


def lora_mixed_linear_host(table: int, x_host_ptr: int, W0_ptr: int, T: int, seg_offsets_host_ptr: int,
                           slot_ids_host_ptr: int, G: int, perm_host_ptr: int, y_host_ptr: int,
                           workspace_ptr: int, workspace_bytes: int, stream: int = 0) -> None:
    _check(lib().lora_mixed_linear_host(table, x_host_ptr, W0_ptr, T, seg_offsets_host_ptr, slot_ids_host_ptr, G,
                                        perm_host_ptr, y_host_ptr, workspace_ptr, workspace_bytes, stream),
           "lora_mixed_linear_host")


def lml_tokens_workspace_bytes(table: int, max_tokens: int) -> int:
    return int(lib().lml_tokens_workspace_bytes(table, max_tokens))


def lora_mixed_linear_tokens(table: int, x_ptr: int, W0_ptr: int, T: int, token_slots_ptr: int, y_ptr: int,
                             workspace_ptr: int, workspace_bytes: int, stream: int = 0) -> None:
    """Segmentation and layer in one call: one slot id per token instead of segments."""
    _check(lib().lora_mixed_linear_tokens(table, x_ptr, W0_ptr, T, token_slots_ptr, y_ptr, workspace_ptr,
                                          workspace_bytes, stream), "lora_mixed_linear_tokens")


def _ptr_array(values):
    arr = (ctypes.c_void_p * len(values))()
    for i, v in enumerate(values):
        arr[i] = v
    return arr


def lml_multi_workspace_bytes(tables, max_tokens: int) -> int:
    return int(lib().lml_multi_workspace_bytes(_ptr_array(tables), len(tables), max_tokens))


def lora_mixed_linear_multi(tables, x_ptr: int, W0_ptrs, T: int, token_slots_ptrs, y_ptrs, workspace_ptr: int,
                            workspace_bytes: int, stream: int = 0) -> None:
    """Several projections of the same x in one call (table handles and per-projection pointers as lists)."""
    P = len(tables)
    assert len(W0_ptrs) == P and len(token_slots_ptrs) == P and len(y_ptrs) == P
    _check(lib().lora_mixed_linear_multi(_ptr_array(tables), P, x_ptr, _ptr_array(W0_ptrs), T,
                                         _ptr_array(token_slots_ptrs), _ptr_array(y_ptrs), workspace_ptr,
                                         workspace_bytes, stream), "lora_mixed_linear_multi")


def register_adapter_transposed(table_T: int, adapter_id: int, version: int, A_ptr: int, B_ptr: int, rank: int,
                                scale: float, stream: int = 0) -> int:
    """Register the forward adapter (A [rank][K], B [N][rank]) in the transposed table (d_in = N, d_out = K)."""
    slot = ctypes.c_int32(-1)
    _check(lib().register_adapter_transposed(table_T, adapter_id, version, A_ptr, B_ptr, rank, scale, stream,
                                             ctypes.byref(slot)), "register_adapter_transposed")
    return int(slot.value)


def lml_backward_workspace_bytes(table: int, max_tokens: int, max_segments: int) -> int:
    return int(lib().lml_backward_workspace_bytes(table, max_tokens, max_segments))


def lora_mixed_linear_backward_adapters(table: int, table_T: int, x_ptr: int, dy_ptr: int, T: int, seg_offsets_ptr: int,
                                        slot_ids_ptr: int, slot_ids_T_ptr: int, G: int, dA_ptr: int, dB_ptr: int,
                                        workspace_ptr: int, workspace_bytes: int, stream: int = 0) -> None:
    """dA, dB (fp32, packed like the arena) += this batch's adapter gradients."""
    _check(lib().lora_mixed_linear_backward_adapters(table, table_T, x_ptr, dy_ptr, T, seg_offsets_ptr, slot_ids_ptr,
                                                     slot_ids_T_ptr, G, dA_ptr, dB_ptr, workspace_ptr, workspace_bytes,
                                                     stream), "lora_mixed_linear_backward_adapters")


def lml_dual_workspace_bytes(table: int, max_tokens: int, max_segments: int) -> int:
    return int(lib().lml_dual_workspace_bytes(table, max_tokens, max_segments))


def lora_mixed_linear_dual(table: int, x_ptr: int, W0_ptr: int, T: int, seg_offsets_ptr: int, slot_ids_a_ptr: int,
                           slot_ids_b_ptr: int, G: int, perm_ptr: int, y_a_ptr: int, y_b_ptr: int, workspace_ptr: int,
                           workspace_bytes: int, stream: int = 0) -> None:
    """The same tokens under two slot bindings in one call; the base product is shared for T > 16."""
    _check(lib().lora_mixed_linear_dual(table, x_ptr, W0_ptr, T, seg_offsets_ptr, slot_ids_a_ptr, slot_ids_b_ptr, G,
                                        perm_ptr, y_a_ptr, y_b_ptr, workspace_ptr, workspace_bytes, stream),
           "lora_mixed_linear_dual")


STATE_RESIDENT, STATE_SERVING, STATE_RETIRING = 0, 1, 2


def lml_publish(table: int, adapter_id: int, version: int, stream: int = 0) -> int:
    """Make (adapter_id, version) the adapter's serving version from this point of the stream on.
    Returns the version that served before, or -1."""
    prev = ctypes.c_int32(-1)
    _check(lib().lml_publish(table, adapter_id, version, stream, ctypes.byref(prev)), "lml_publish")
    return int(prev.value)


def lml_pin(table: int, slot: int) -> None:
    _check(lib().lml_pin(table, slot), "lml_pin")


def lml_unpin(table: int, slot: int) -> None:
    _check(lib().lml_unpin(table, slot), "lml_unpin")


def lml_resolve(table: int, adapter_id: int):
    """(slot, version) of the adapter's serving entry; raises LmlError(NOT_FOUND) if none."""
    slot, ver = ctypes.c_int32(-1), ctypes.c_int32(-1)
    _check(lib().lml_resolve(table, adapter_id, ctypes.byref(slot), ctypes.byref(ver)), "lml_resolve")
    return int(slot.value), int(ver.value)


def lml_slot_state(table: int, slot: int):
    """(state, pins) of a live slot."""
    st, pins = ctypes.c_int32(-1), ctypes.c_int32(-1)
    _check(lib().lml_slot_state(table, slot, ctypes.byref(st), ctypes.byref(pins)), "lml_slot_state")
    return int(st.value), int(pins.value)


def lml_segment_tokens_adapters(table: int, token_adapter_ids_ptr: int, T: int, perm_ptr: int, seg_offsets_ptr: int,
                                seg_slot_ids_ptr: int, stream: int = 0) -> None:
    _check(lib().lml_segment_tokens_adapters(table, token_adapter_ids_ptr, T, perm_ptr, seg_offsets_ptr,
                                             seg_slot_ids_ptr, stream), "lml_segment_tokens_adapters")


def lora_mixed_linear_adapters(table: int, x_ptr: int, W0_ptr: int, T: int, token_adapter_ids_ptr: int, y_ptr: int,
                               workspace_ptr: int, workspace_bytes: int, stream: int = 0) -> None:
    """lora_mixed_linear_tokens with adapter ids, resolved on the device to each adapter's serving slot."""
    _check(lib().lora_mixed_linear_adapters(table, x_ptr, W0_ptr, T, token_adapter_ids_ptr, y_ptr, workspace_ptr,
                                            workspace_bytes, stream), "lora_mixed_linear_adapters")


def lora_mixed_linear_decode_static(table: int, x_ptr: int, W0_ptr: int, T: int, seg_offsets_ptr: int,
                                    slot_ids_ptr: int, G: int, perm_ptr: int, y_ptr: int, stream: int = 0) -> None:
    """Decode form (T <= 16) that takes no workspace: its scratch is a fixed array inside the
    library, so the call allocates nothing.  For callers that cannot obtain device memory."""
    _check(lib().lora_mixed_linear_decode_static(table, x_ptr, W0_ptr, T, seg_offsets_ptr, slot_ids_ptr, G,
                                                 perm_ptr, y_ptr, stream), "lora_mixed_linear_decode_static")


def lml_checkpoint_data_bytes(T: int, d: int) -> int:
    return int(lib().lml_checkpoint_data_bytes(T, d))


def lml_checkpoint_scale_bytes(T: int, d: int) -> int:
    return int(lib().lml_checkpoint_scale_bytes(T, d))


def lml_checkpoint_store(device: int, x_ptr: int, T: int, d: int, kept: Rows, stream: int = 0) -> None:
    _check(lib().lml_checkpoint_store(device, x_ptr, T, d, kept, stream), "lml_checkpoint_store")


def lml_checkpoint_load(device: int, kept: Rows, T: int, d: int, x_ptr: int, stream: int = 0) -> None:
    _check(lib().lml_checkpoint_load(device, kept, T, d, x_ptr, stream), "lml_checkpoint_load")


def lml_backward_rows_workspace_bytes(table: int, max_tokens: int, max_segments: int) -> int:
    return int(lib().lml_backward_rows_workspace_bytes(table, max_tokens, max_segments))


def lora_mixed_linear_backward_adapters_rows(table: int, table_T: int, x: Rows, dy_ptr: int, T: int, seg_offsets_ptr: int,
                                             slot_ids_ptr: int, slot_ids_T_ptr: int, G: int, dA_ptr: int, dB_ptr: int,
                                             accumulate: bool, workspace_ptr: int, workspace_bytes: int, stream: int = 0) -> None:
    """dA, dB of one batch with x as bf16 rows or as a checkpoint; accumulate: added to, else written."""
    _check(lib().lora_mixed_linear_backward_adapters_rows(table, table_T, x, dy_ptr, T, seg_offsets_ptr, slot_ids_ptr, slot_ids_T_ptr,
                                                          G, dA_ptr, dB_ptr, 1 if accumulate else 0, workspace_ptr, workspace_bytes,
                                                          stream), "lora_mixed_linear_backward_adapters_rows")


def lml_block_norm(device: int, desc: BlockNormDesc, T: int, h_ptr: int, o_ptr: int, gate_rows_ptr: int, h_new_ptr: int, x_ptr: int,
                   x_kept: Optional[Rows], h_kept: Optional[Rows], stream: int = 0) -> None:
    _check(lib().lml_block_norm(device, desc, T, h_ptr, o_ptr, gate_rows_ptr, h_new_ptr, x_ptr, x_kept, h_kept, stream), "lml_block_norm")


def lml_block_norm_workspace_bytes(device: int, T: int, d: int) -> int:
    return int(lib().lml_block_norm_workspace_bytes(device, T, d))


def lml_block_norm_backward(device: int, desc: BlockNormDesc, T: int, h_new: Optional[Rows], o: Optional[Rows], gate_rows_ptr: int,
                            dx_ptr: int, dh_new_ptr: int, dh_ptr: int, d_o_ptr: int, dw_pre_ptr: int, dw_post_ptr: int, dgate_ptr: int,
                            dgate_rows_ptr: int, workspace_ptr: int, workspace_bytes: int, stream: int = 0) -> None:
    _check(lib().lml_block_norm_backward(device, desc, T, h_new, o, gate_rows_ptr, dx_ptr, dh_new_ptr, dh_ptr, d_o_ptr, dw_pre_ptr,
                                         dw_post_ptr, dgate_ptr, dgate_rows_ptr, workspace_ptr, workspace_bytes, stream),
           "lml_block_norm_backward")


def lml_device_status(table: int, stream: int = 0) -> int:
    f = ctypes.c_uint32(0)
    _check(lib().lml_device_status(table, ctypes.byref(f), stream), "lml_device_status")
    return int(f.value)


def lml_last_launch_count(table: int) -> int:
    return int(lib().lml_last_launch_count(table))


# ---- torch convenience ------------------------------------------------------------------------------

def _ptr(t) -> int:
    return 0 if t is None else int(t.data_ptr())


_current_raw_stream = None


def _stream(stream) -> int:
    if stream is not None:
        return int(stream.cuda_stream)
    # the current stream of the current device, as a number: torch.cuda.current_stream() builds a Stream object for it at
    # every call (1.5 us of a small call's 17 us)
    global _current_raw_stream
    if _current_raw_stream is None:
        import torch
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        if raw is None:
            _current_raw_stream = lambda: torch.cuda.current_stream().cuda_stream  # noqa: E731
        else:
            device = torch.cuda.current_device
            _current_raw_stream = lambda: raw(device())  # noqa: E731
    return int(_current_raw_stream())


_raw_stream_of = None
_bf16 = _f32 = _u8 = None


def _stream_on(device: int, stream) -> int:
    """The given stream, or the current one of the tensors' device (which need not be the current device)."""
    if stream is not None:
        return int(stream.cuda_stream)
    global _raw_stream_of
    if _raw_stream_of is None:
        import torch
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        _raw_stream_of = raw if raw is not None else (lambda d: torch.cuda.current_stream(d).cuda_stream)
    return _raw_stream_of(device)


def _with_stream(stream, device: int):
    """For a call that allocates: the given stream as the current one, so that what it allocates (results and, above all, a workspace that nobody
    holds when the call returns) is that stream's memory.  A stream of another device than the tensors' is refused: the call would run on the
    current stream of theirs."""
    import torch
    assert stream.device.index == device, ("stream", stream.device, device)
    return torch.cuda.stream(stream)


def _bf16_rows(t, shape, name, device: int) -> int:
    """Checks a bf16 [T][d] tensor of a call on cuda:`device` and gives its address; None is 0."""
    if t is None:
        return 0
    global _bf16
    if _bf16 is None:
        import torch
        _bf16 = torch.bfloat16
    assert t.dtype is _bf16 and t.shape == shape and t.is_contiguous(), (name, t.shape, t.dtype)
    assert t.get_device() == device, (name, t.device)
    return t.data_ptr()


def _sums(t, shape, name, device: int) -> int:
    """Checks a float32 [d] tensor that a call adds to, and gives its address; None is 0."""
    if t is None:
        return 0
    global _f32
    if _f32 is None:
        import torch
        _f32 = torch.float32
    assert t.dtype is _f32 and t.shape == shape and t.is_contiguous() and t.get_device() == device, (name, t.shape, t.dtype)
    return t.data_ptr()


def _kept_uint8(t, shape, name, device: int) -> None:
    global _u8
    if _u8 is None:
        import torch
        _u8 = torch.uint8
    assert t.dtype is _u8 and t.shape == shape and t.is_contiguous() and t.get_device() == device, (name, t.shape, t.dtype)


def _cuda_index(t, name) -> int:
    assert t.is_cuda, name
    return t.get_device()


class Checkpoint:
    """Activations kept in 8 bits (`form` "int8" or "e4m3") with a power-of-two scale per row and 32 columns; see lml_rows in the C header.
    data uint8 [T][width up to a multiple of 32], scales uint8 [ceil(width / 128)][T][4]."""

    def __init__(self, data, scales, width: int, form: str):
        T = data.shape[0]
        assert form in ("int8", "e4m3"), form
        self.device = _cuda_index(data, "data")
        _kept_uint8(data, (T, (width + 31) // 32 * 32), "data", self.device)
        _kept_uint8(scales, ((width + 127) // 128, T, 4), "scales", self.device)
        assert width > 0 and width % 8 == 0, width
        self._data, self._scales, self.tokens, self.width, self.form = data, scales, T, int(width), form
        self.rows = Rows(data.data_ptr(), scales.data_ptr(), ROW_FORMS[form])

    @classmethod
    def empty(cls, tokens: int, width: int, form: str, device="cuda") -> "Checkpoint":
        import torch
        return cls._in(torch.empty(cls._bytes(tokens, width), dtype=torch.uint8, device=device), tokens, width, form)

    @staticmethod
    def _bytes(tokens: int, width: int) -> int:
        return tokens * ((width + 31) // 32 * 32 + (width + 127) // 128 * 4)

    @classmethod
    def _in(cls, buffer, tokens: int, width: int, form: str) -> "Checkpoint":
        """Both arrays in one buffer (one allocation instead of two views of it: they are made when somebody asks for them)."""
        assert form in ("int8", "e4m3") and width > 0 and width % 8 == 0, (form, width)
        self = cls.__new__(cls)
        self.device = _cuda_index(buffer, "device")
        self.tokens, self.width, self.form = tokens, width, form
        self._data = self._scales = None
        self._buffer, at = buffer, buffer.data_ptr()
        self.rows = Rows(at, at + tokens * ((width + 31) // 32 * 32), ROW_FORMS[form])
        return self

    @property
    def data(self):
        if self._data is None:
            pitch = (self.width + 31) // 32 * 32
            self._data = self._buffer[:self.tokens * pitch].view(self.tokens, pitch)
        return self._data

    @property
    def scales(self):
        if self._scales is None:
            groups = (self.width + 127) // 128
            self._scales = self._buffer[self.tokens * ((self.width + 31) // 32 * 32):].view(groups, self.tokens, 4)
        return self._scales

    def nbytes(self) -> int:
        """Device memory that it takes."""
        return self._bytes(self.tokens, self.width)

    def store(self, x, stream=None) -> "Checkpoint":
        """Keep x (bf16 [tokens][width])."""
        lml_checkpoint_store(self.device, _bf16_rows(x, (self.tokens, self.width), "x", self.device), self.tokens, self.width, self.rows,
                             _stream_on(self.device, stream))
        return self

    def load(self, out=None, stream=None):
        """The values it stands for, bf16 [tokens][width]."""
        import torch
        if stream is not None:
            with _with_stream(stream, self.device):
                return self.load(out)
        shape, dev = (self.tokens, self.width), self.device
        if out is None:
            out = (self._data if self._data is not None else self._buffer).new_empty(shape, dtype=torch.bfloat16)
            at = out.data_ptr()
        else:
            at = _bf16_rows(out, shape, "out", dev)
        lml_checkpoint_load(dev, self.rows, self.tokens, self.width, at, _stream_on(dev, None))
        return out


def checkpoint_store(x, form: str = "int8", stream=None) -> Checkpoint:
    """A new checkpoint of x (bf16 [T][d])."""
    import torch
    if stream is not None:
        with _with_stream(stream, _cuda_index(x, "x")):
            return checkpoint_store(x, form)
    T, d = x.shape
    return Checkpoint._in(x.new_empty(Checkpoint._bytes(T, d), dtype=torch.uint8), T, d, form).store(x)


def _as_rows(x, shape, name, device: int):
    """Rows of a call: a bf16 tensor or a Checkpoint."""
    if x is None:
        return None
    if isinstance(x, Checkpoint):
        assert (x.tokens, x.width) == shape and x.device == device, (name, x.tokens, x.width)
        return x.rows
    return Rows(_bf16_rows(x, shape, name, device), None, ROWS_BF16)


class BlockNorm:
    """The norms between two blocks (lml_block_norm): weights and gate bf16 [d] or None, kept by the caller's program.

        n = rmsnorm(o) w_post;  h' = h + scale gate n;  x = rmsnorm(h') w_pre

    The weights may be written to, but not replaced: the descriptor holds their addresses.
    """
    d, w_post, w_pre, gate, scale, eps = (property(operator.attrgetter("_" + name)) for name in ("d", "w_post", "w_pre", "gate", "scale", "eps"))

    def __init__(self, d: int, w_post=None, w_pre=None, gate=None, scale: float = 1.0, eps: float = 1e-5):
        import torch
        assert 0 < d <= MAX_NORM_WIDTH and d % 8 == 0, d
        for name, w in (("w_post", w_post), ("w_pre", w_pre), ("gate", gate)):
            assert w is None or (w.dtype == torch.bfloat16 and w.is_cuda and w.is_contiguous() and tuple(w.shape) == (d,)), name
        self._d, self._w_post, self._w_pre, self._gate, self._scale, self._eps = d, w_post, w_pre, gate, float(scale), float(eps)
        self.device = next((w.get_device() for w in (w_post, w_pre, gate) if w is not None), None)
        assert all(w is None or w.get_device() == self.device for w in (w_post, w_pre, gate)), "weights on several devices"
        self.desc = BlockNormDesc(d, eps, scale, _ptr(w_post), _ptr(w_pre), _ptr(gate))

    def forward(self, h, o=None, gate_rows=None, h_new=None, x=None, x_checkpoint=None, h_checkpoint=None, stream=None):
        """-> (h', x).  o None: h' is h.  gate_rows: a gate per token, bf16 [T][d].  h_new / x: where to write them (new tensors otherwise);
        x_checkpoint / h_checkpoint: Checkpoints that the same pass fills.  x is None without w_pre."""
        import torch
        if stream is not None:
            with _with_stream(stream, _cuda_index(h, "h")):
                return self.forward(h, o, gate_rows, h_new, x, x_checkpoint, h_checkpoint)
        T, dev = int(h.shape[0]), _cuda_index(h, "h")
        shape = (T, self.d)
        assert self.device is None or dev == self.device, dev
        h_at = _bf16_rows(h, shape, "h", dev)
        if h_new is None and o is not None:
            h_new = torch.empty_like(h)
            h_new_at = h_new.data_ptr()
        else:
            h_new_at = _bf16_rows(h_new, shape, "h_new", dev)
        if x is None and self.w_pre is not None:
            x = torch.empty_like(h)
            x_at = x.data_ptr()
        else:
            x_at = _bf16_rows(x, shape, "x", dev)
        lml_block_norm(dev, self.desc, T, h_at, _bf16_rows(o, shape, "o", dev), _bf16_rows(gate_rows, shape, "gate_rows", dev), h_new_at, x_at,
                       _as_rows(x_checkpoint, shape, "x_checkpoint", dev), _as_rows(h_checkpoint, shape, "h_checkpoint", dev), _stream_on(dev, None))
        return (h if o is None else h_new), x

    def backward(self, h_new, o, dx, dh_new, gate_rows=None, dh=None, d_o=None, dw_pre=None, dw_post=None, dgate=None, workspace=None,
                 stream=None):
        """-> (dh, d_o, dgate).  h_new and o: bf16 tensors or Checkpoints; dx, dh_new: the gradients of x and h' (either may be None).
        dw_pre, dw_post, dgate: float32 [d] that the sums over the tokens are added to, or None (frozen).  The third result is dgate, or with
        gate_rows their gradient, bf16 [T][d]."""
        import torch
        some = dx if dx is not None else dh_new
        if stream is not None:
            with _with_stream(stream, _cuda_index(some, "dx")):
                return self.backward(h_new, o, dx, dh_new, gate_rows, dh, d_o, dw_pre, dw_post, dgate, workspace)
        T, d, dev = int(some.shape[0]), self.d, _cuda_index(some, "dx")
        shape = (T, d)
        assert self.device is None or dev == self.device, dev
        dx_at, dh_new_at = _bf16_rows(dx, shape, "dx", dev), _bf16_rows(dh_new, shape, "dh_new", dev)
        gate_at = _bf16_rows(gate_rows, shape, "gate_rows", dev)
        if dh is None:
            dh = torch.empty_like(some)
            dh_at = dh.data_ptr()
        else:
            dh_at = _bf16_rows(dh, shape, "dh", dev)
        if d_o is None and o is not None:
            d_o = torch.empty_like(some)
            d_o_at = d_o.data_ptr()
        else:
            d_o_at = _bf16_rows(d_o, shape, "d_o", dev)
        dgate_rows = torch.empty_like(gate_rows) if gate_rows is not None else None
        n_ws = 0
        if dw_pre is not None or dw_post is not None or dgate is not None:
            if workspace is None:
                n_ws = max(lml_block_norm_workspace_bytes(dev, T, d), 256)
                workspace = some.new_empty(n_ws, dtype=torch.uint8)
            else:
                assert workspace.get_device() == dev and workspace.is_contiguous(), "workspace"
                n_ws = workspace.numel() * workspace.element_size()
        lml_block_norm_backward(dev, self.desc, T, _as_rows(h_new, shape, "h_new", dev), _as_rows(o, shape, "o", dev), gate_at, dx_at, dh_new_at,
                                dh_at, d_o_at, _sums(dw_pre, (d,), "dw_pre", dev), _sums(dw_post, (d,), "dw_post", dev),
                                _sums(dgate, (d,), "dgate", dev), _ptr(dgate_rows), _ptr(workspace) if n_ws else 0, n_ws, _stream_on(dev, None))
        return dh, d_o, (dgate_rows if gate_rows is not None else dgate)


def fuse_projection_adapters(parts):
    """Adapters of several projections that read the same x (q/k/v, or gate/up) as ONE adapter of
    the projection with the concatenated weight: parts = [(A_p [r_p, d_in], B_p [d_out_p, r_p]), ...]
    gives A = cat(A_p) [sum r_p, d_in] and B = blockdiag(B_p) [sum d_out_p, sum r_p], so that
    x.W0cat + s (x.A^T).B^T equals the per-projection results side by side (same scale for all
    parts; sum r_p <= 64).  One call then reads x once and launches once instead of once per
    projection.  Layout plumbing only (torch cat / copy); the arithmetic stays in the kernels."""
    import torch
    A = torch.cat([a for a, _ in parts], dim=0).contiguous()
    rank = int(A.shape[0])
    assert rank <= MAX_RANK, "fused rank exceeds the table's maximum"
    n_total = sum(int(b.shape[0]) for _, b in parts)
    B = torch.zeros((n_total, rank), dtype=parts[0][1].dtype, device=parts[0][1].device)
    n0 = r0 = 0
    for a, b in parts:
        r, n = int(a.shape[0]), int(b.shape[0])
        B[n0:n0 + n, r0:r0 + r] = b
        n0 += n
        r0 += r
    return A, B


def multi_projection(tables, x, W0s, token_slots, ys=None, workspace=None, stream=None):
    """lora_mixed_linear_multi for torch tensors: tables = [Table, ...], W0s / token_slots per projection
    (token_slots may also be one tensor for all).  Returns the list of outputs."""
    import torch
    P, T = len(tables), int(x.shape[0])
    if not isinstance(token_slots, (list, tuple)):
        token_slots = [token_slots] * P
    if ys is None:
        ys = [torch.empty((T, t.d_out), dtype=torch.bfloat16, device=x.device) for t in tables]
    handles = [t.handle for t in tables]
    if workspace is None:
        workspace = torch.empty(max(lml_multi_workspace_bytes(handles, T), 256), dtype=torch.uint8, device=x.device)
    lora_mixed_linear_multi(handles, _ptr(x), [_ptr(w) for w in W0s], T, [_ptr(s) for s in token_slots],
                            [_ptr(y) for y in ys], _ptr(workspace), int(workspace.numel()), _stream(stream))
    return ys


class Table:
    """Adapter slot table of one linear site, for torch tensors (bf16 CUDA, contiguous)."""

    def __init__(self, d_in: int, d_out: int, max_slots: int = MAX_SLOTS, device: int = 0):
        self.d_in, self.d_out, self.max_slots, self.device = d_in, d_out, max_slots, device
        self.handle = lml_table_create(device, d_in, d_out, max_slots)
        self._ws = None

    def close(self) -> None:
        if self.handle:
            lml_table_destroy(self.handle)
            self.handle = 0

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def register_adapter(self, adapter_id: int, version: int, A, B, scale: float, stream=None) -> int:
        import torch
        assert A.dtype == torch.bfloat16 and B.dtype == torch.bfloat16 and A.is_cuda and B.is_cuda
        assert A.is_contiguous() and B.is_contiguous()
        rank = int(A.shape[0])
        assert A.shape == (rank, self.d_in) and B.shape == (self.d_out, rank), (A.shape, B.shape)
        return register_adapter(self.handle, adapter_id, version, _ptr(A), _ptr(B), rank, float(scale),
                                _stream(stream))

    def retire_version(self, adapter_id: int, version: int, stream="legacy") -> None:
        """stream="legacy": the C call retire_version (legacy default stream); a torch stream or None (the
        current stream): retire_version_on."""
        if isinstance(stream, str):
            retire_version(self.handle, adapter_id, version)
        else:
            retire_version_on(self.handle, adapter_id, version, _stream(stream))

    def lookup(self, adapter_id: int, version: int) -> int:
        return lml_lookup(self.handle, adapter_id, version)

    def slot_info(self, slot: int):
        return lml_slot_info(self.handle, slot)

    def workspace_bytes(self, max_tokens: int, max_segments: int) -> int:
        return lml_workspace_bytes(self.handle, max_tokens, max_segments)

    def workspace(self, T: int, G: int, host: bool = False):
        """A cached torch byte buffer large enough for (T, G); grown on demand (outside the hot call)."""
        import torch
        need = (lml_host_workspace_bytes if host else lml_workspace_bytes)(self.handle, T, G)
        if self._ws is None or self._ws.numel() < need:
            self._ws = torch.empty(max(need, 1024), dtype=torch.uint8, device=f"cuda:{self.device}")
        return self._ws

    def segment_tokens(self, token_slots, stream=None):
        """token_slots int32[T] (cuda) -> (perm int32[T], seg_offsets int32[max_slots+2],
        seg_slot_ids int32[max_slots+1]); G = max_slots + 1."""
        import torch
        assert token_slots.dtype == torch.int32 and token_slots.is_cuda and token_slots.is_contiguous()
        T = int(token_slots.shape[0])
        dev = token_slots.device
        perm = torch.empty(max(T, 1), dtype=torch.int32, device=dev)
        seg_offsets = torch.empty(self.max_slots + 2, dtype=torch.int32, device=dev)
        seg_slot_ids = torch.empty(self.max_slots + 1, dtype=torch.int32, device=dev)
        lml_segment_tokens(self.handle, _ptr(token_slots), T, _ptr(perm), _ptr(seg_offsets), _ptr(seg_slot_ids),
                           _stream(stream))
        return perm[:T], seg_offsets, seg_slot_ids

    def lora_mixed_linear(self, x, W0, seg_offsets, slot_ids, perm=None, y=None, workspace=None, stream=None):
        import torch
        assert x.dtype == torch.bfloat16 and W0.dtype == torch.bfloat16 and x.is_cuda and W0.is_cuda
        assert x.is_contiguous() and W0.is_contiguous()
        T = int(x.shape[0])
        assert x.shape[1] == self.d_in and W0.shape == (self.d_out, self.d_in)
        G = 0 if slot_ids is None else int(slot_ids.shape[0])
        if G:
            assert seg_offsets.dtype == torch.int32 and slot_ids.dtype == torch.int32
            assert seg_offsets.shape[0] == G + 1 and seg_offsets.is_cuda and slot_ids.is_cuda
        if perm is not None:
            assert perm.dtype == torch.int32 and perm.shape[0] == T and perm.is_cuda
        if y is None:
            y = torch.empty((T, self.d_out), dtype=torch.bfloat16, device=x.device)
        if workspace is None:
            workspace = self.workspace(T, G)
        lora_mixed_linear(self.handle, _ptr(x), _ptr(W0), T, _ptr(seg_offsets) if G else 0,
                          _ptr(slot_ids) if G else 0, G, _ptr(perm), _ptr(y), _ptr(workspace),
                          int(workspace.numel()), _stream(stream))
        return y

    def publish(self, adapter_id: int, version: int, stream=None) -> int:
        return lml_publish(self.handle, adapter_id, version, _stream(stream))

    def pin(self, slot: int) -> None:
        lml_pin(self.handle, slot)

    def unpin(self, slot: int) -> None:
        lml_unpin(self.handle, slot)

    def resolve(self, adapter_id: int):
        return lml_resolve(self.handle, adapter_id)

    def slot_state(self, slot: int):
        return lml_slot_state(self.handle, slot)

    def register_adapter_transposed(self, adapter_id: int, version: int, A, B, scale: float, stream=None) -> int:
        """On the TRANSPOSED table (d_in = N, d_out = K): A [rank][K], B [N][rank] of the forward layer."""
        rank = int(A.shape[0])
        assert A.shape[1] == self.d_out and B.shape == (self.d_in, rank)
        return register_adapter_transposed(self.handle, adapter_id, version, _ptr(A), _ptr(B), rank, float(scale),
                                           _stream(stream))

    def backward_adapters(self, table_T, x, dy, seg_offsets, slot_ids, slot_ids_T, dA, dB, stream=None):
        """dA fp32 [max_slots][64][d_in], dB fp32 [max_slots][d_out][64] += gradients of this batch."""
        import torch
        T, G = int(x.shape[0]), int(slot_ids.shape[0])
        assert dA.dtype == torch.float32 and dB.dtype == torch.float32
        assert tuple(dA.shape) == (self.max_slots, 64, self.d_in) and tuple(dB.shape) == (self.max_slots, self.d_out, 64)
        ws = torch.empty(max(lml_backward_workspace_bytes(self.handle, T, G), 256), dtype=torch.uint8, device=x.device)
        lora_mixed_linear_backward_adapters(self.handle, table_T.handle, _ptr(x), _ptr(dy), T, _ptr(seg_offsets),
                                            _ptr(slot_ids), _ptr(slot_ids_T), G, _ptr(dA), _ptr(dB), _ptr(ws),
                                            int(ws.numel()), _stream(stream))

    def backward_adapters_rows(self, table_T, x, dy, seg_offsets, slot_ids, slot_ids_T, dA, dB, accumulate=True, workspace=None, stream=None):
        """backward_adapters with x as a Checkpoint (or a bf16 tensor) and unrounded small products.  accumulate=False: the rows j < rank of
        every live slot are written, so that dA and dB need not be zeroed before a step's first batch."""
        import torch
        if stream is not None:
            with _with_stream(stream, self.device):
                return self.backward_adapters_rows(table_T, x, dy, seg_offsets, slot_ids, slot_ids_T, dA, dB, accumulate, workspace)
        T, G, dev = int(dy.shape[0]), int(slot_ids.shape[0]), self.device
        assert dA.dtype is torch.float32 and dB.dtype is torch.float32 and dA.is_contiguous() and dB.is_contiguous()
        assert dA.shape == (self.max_slots, 64, self.d_in) and dB.shape == (self.max_slots, self.d_out, 64)
        assert seg_offsets.dtype is slot_ids.dtype is slot_ids_T.dtype is torch.int32
        assert seg_offsets.shape[0] == G + 1 and slot_ids_T.shape[0] == G
        assert seg_offsets.is_contiguous() and slot_ids.is_contiguous() and slot_ids_T.is_contiguous()
        for t in (dA, dB, seg_offsets, slot_ids, slot_ids_T):
            assert t.get_device() == dev, t.device
        dy_at = _bf16_rows(dy, (T, self.d_out), "dy", dev)
        if workspace is None:
            workspace = dy.new_empty(max(lml_backward_rows_workspace_bytes(self.handle, T, G), 256), dtype=torch.uint8)
        assert workspace.get_device() == dev and workspace.is_contiguous(), "workspace"
        lora_mixed_linear_backward_adapters_rows(self.handle, table_T.handle, _as_rows(x, (T, self.d_in), "x", dev), dy_at, T,
                                                 seg_offsets.data_ptr(), slot_ids.data_ptr(), slot_ids_T.data_ptr(), G, dA.data_ptr(),
                                                 dB.data_ptr(), accumulate, workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                                                 _stream_on(dev, None))

    def lora_mixed_linear_dual(self, x, W0, seg_offsets, slot_ids_a, slot_ids_b, perm=None, stream=None):
        """-> (y_a, y_b): the layer under two slot bindings of the same segments."""
        import torch
        T, G = int(x.shape[0]), int(slot_ids_a.shape[0])
        assert slot_ids_b.shape[0] == G and seg_offsets.shape[0] == G + 1
        y_a = torch.empty((T, self.d_out), dtype=torch.bfloat16, device=x.device)
        y_b = torch.empty_like(y_a)
        ws = torch.empty(max(lml_dual_workspace_bytes(self.handle, T, G), 256), dtype=torch.uint8, device=x.device)
        lora_mixed_linear_dual(self.handle, _ptr(x), _ptr(W0), T, _ptr(seg_offsets), _ptr(slot_ids_a), _ptr(slot_ids_b),
                               G, _ptr(perm), _ptr(y_a), _ptr(y_b), _ptr(ws), int(ws.numel()), _stream(stream))
        return y_a, y_b

    def lora_mixed_linear_adapters(self, x, W0, token_adapter_ids, y=None, workspace=None, stream=None):
        """As lora_mixed_linear_tokens, with one ADAPTER id per token (resolved on the device)."""
        return self.lora_mixed_linear_tokens(x, W0, token_adapter_ids, y, workspace, stream, by_adapter=True)

    def lora_mixed_linear_tokens(self, x, W0, token_slots, y=None, workspace=None, stream=None, by_adapter=False):
        """x bf16 [T][d_in], W0 bf16 [d_out][d_in], token_slots int32[T] (all cuda) -> y bf16 [T][d_out]."""
        import torch
        assert x.dtype == torch.bfloat16 and W0.dtype == torch.bfloat16 and token_slots.dtype == torch.int32
        assert x.is_cuda and W0.is_cuda and token_slots.is_cuda and x.is_contiguous() and W0.is_contiguous()
        T = int(x.shape[0])
        assert token_slots.shape[0] == T and x.shape[1] == self.d_in and W0.shape == (self.d_out, self.d_in)
        if y is None:
            y = torch.empty((T, self.d_out), dtype=torch.bfloat16, device=x.device)
        if workspace is None:
            workspace = torch.empty(max(lml_tokens_workspace_bytes(self.handle, T), 256), dtype=torch.uint8,
                                    device=x.device)
        fn = lora_mixed_linear_adapters if by_adapter else lora_mixed_linear_tokens
        fn(self.handle, _ptr(x), _ptr(W0), T, _ptr(token_slots), _ptr(y), _ptr(workspace), int(workspace.numel()),
           _stream(stream))
        return y

    def lora_mixed_linear_host(self, x_host, W0, seg_offsets_host, slot_ids_host, y_host, perm_host=None,
                               workspace=None, stream=None):
        """x_host / y_host: CPU bf16 tensors (pinned for asynchronous copies); W0 on the device."""
        T = int(x_host.shape[0])
        G = 0 if slot_ids_host is None else int(slot_ids_host.shape[0])
        assert not x_host.is_cuda and not y_host.is_cuda and W0.is_cuda
        if workspace is None:
            workspace = self.workspace(T, G, host=True)
        lora_mixed_linear_host(self.handle, _ptr(x_host), _ptr(W0), T, _ptr(seg_offsets_host) if G else 0,
                               _ptr(slot_ids_host) if G else 0, G, _ptr(perm_host), _ptr(y_host),
                               _ptr(workspace), int(workspace.numel()), _stream(stream))
        return y_host

    def device_status(self, stream=None) -> int:
        return lml_device_status(self.handle, _stream(stream))

    def last_launch_count(self) -> int:
        return lml_last_launch_count(self.handle)
