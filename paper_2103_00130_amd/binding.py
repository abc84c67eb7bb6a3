"""ctypes binding of libabftgemm.so: same names as include/abft_gemm.h and include/abft_eb.h.

Argument marshalling only.  torch tensors supply device memory and the current
stream; every step of the method runs in the HIP kernels behind the C ABI.
Importing this module fails loudly when the library has not been built
(`python -m paper_2103_00130_amd.build`): there is no fallback path.  The calls
of a serving loop, the checked GEMM, the checked lookup and those of a decoding step, are
marshalled natively (csrc/fastcall.cpp); operands that it does not take - and so every wrong one - go
through the Python code that follows, which says what is wrong with them.
"""
from __future__ import annotations

import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
# ABFT_LIBRARY: path of another build of the same library (the diagnostic build with in-kernel clock traces)
LIB_PATH = os.environ.get("ABFT_LIBRARY") or os.path.join(_HERE, "libabftgemm.so")

ABFT_OK, ABFT_EINVAL, ABFT_EUNSUPPORTED, ABFT_EHIP = 0, -1, -2, -3
ABFT_CHECK, ABFT_NOCHECK, ABFT_MOD127, ABFT_ERRCOUNT_ACCUMULATE = 0, 1, 2, 4
ABFT_VARIANT_TILE256, ABFT_VARIANT_TILE128, ABFT_VARIANT_TILE64, ABFT_VARIANT_SMALLM = 0x100, 0x200, 0x300, 0x400

EXPORTS = (
    "abft_pack_b_checksum", "abft_packed_b_dims", "abft_packed_b_get_checksum", "abft_packed_b_get_checksum_mod127",
    "abft_packed_b_get_col_offsets",
    "abft_packed_b_flip_bit", "abft_packed_b_flip_checksum_bit", "abft_packed_b_flip_checksum_bit_mod127",
    "abft_packed_b_destroy", "abft_packed_b_trim",
    "abft_gemm_workspace_bytes", "abft_workspace_init", "abft_gemm_u8s8s32_checked", "abft_gemm_u8s8s32_checked_static",
    "abft_requantize_u8",
    "abft_verify_rows", "abft_row_checksum", "abft_recover_scratch_bytes", "abft_recompute_flagged_rows",
    "abft_recompute_flagged_rows_async",
    "abft_locate_scratch_bytes", "abft_locate_correct", "abft_calib_copy", "abft_clock_probe", "abft_mfma_peak_probe", "abft_clock_trace", "abft_last_error",
    "abft_w4_pack", "abft_w4_dims", "abft_w4_destroy", "abft_w4_gemv",
)
ABFT_LOCATE_CLEAN, ABFT_LOCATE_CORRECTED, ABFT_LOCATE_NOT_ONE_ELEMENT = 0, 1, 2
EXPORTS_EB = (
    "abft_eb_pack_rowsum", "abft_eb_table_dims", "abft_eb_table_get_rowsums", "abft_eb_table_flip_bit",
    "abft_eb_table_destroy", "abft_eb_u8_checked",
    "abft_kv_code_bytes", "abft_kv_plan", "abft_kv_append", "abft_kv_read", "abft_kv_attention_workspace_bytes", "abft_kv_attention",
)
ABFT_EB_CHECK, ABFT_EB_NOCHECK = 0, 1
ABFT_EB_VARIANT_BATCH, ABFT_EB_VARIANT_GROUP = 0x100, 0x200
ABFT_EB_ERR, ABFT_EB_BAD_INDEX = 1, 2
ABFT_EB_PACK_COMPACT, ABFT_EB_PACK_LINE_ALIGNED, ABFT_EB_PACK_INT4 = 0, 1, 2
ABFT_TYPE_F32, ABFT_TYPE_F16, ABFT_TYPE_BF16 = 0, 1, 2
ABFT_KV_NO_BLOCK, ABFT_KV_TABLE_FULL, ABFT_KV_NO_ROW, ABFT_KV_BAD_LENGTH, ABFT_KV_BAD_BLOCK = 1, 2, 4, 8, 16


class abft_requant_t(ctypes.Structure):
    _fields_ = [("zA", ctypes.c_int32), ("zC", ctypes.c_int32), ("mult", ctypes.c_void_p),
                ("per_channel", ctypes.c_int32), ("bias", ctypes.c_void_p)]


class abft_inject_t(ctypes.Structure):
    _fields_ = [("row", ctypes.c_int32), ("col", ctypes.c_int32), ("xor_mask", ctypes.c_uint32)]


class abft_kv_cache_t(ctypes.Structure):
    _fields_ = [("k_codes", ctypes.c_void_p), ("v_codes", ctypes.c_void_p), ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
                ("n_blocks", ctypes.c_int32), ("heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("block_tokens", ctypes.c_int32)]


class AbftError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"libabftgemm error {code}: {msg}")
        self.code = code


def _load() -> ctypes.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2103_00130_amd.build`")
    L = ctypes.CDLL(LIB_PATH)
    vp, i64, i32, u32, sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_uint32, ctypes.c_size_t
    L.abft_last_error.restype = ctypes.c_char_p
    L.abft_pack_b_checksum.argtypes = [vp, i64, i32, i32, i32, vp, ctypes.POINTER(vp)]
    L.abft_packed_b_dims.argtypes = [vp, ctypes.POINTER(i32), ctypes.POINTER(i32)]
    L.abft_packed_b_get_checksum.argtypes = [vp, vp, vp]
    L.abft_packed_b_get_checksum_mod127.argtypes = [vp, vp, vp]
    L.abft_packed_b_get_col_offsets.argtypes = [vp, vp, vp]
    L.abft_packed_b_flip_bit.argtypes = [vp, i32, i32, i32, vp]
    L.abft_packed_b_flip_checksum_bit.argtypes = [vp, i32, i32, vp]
    L.abft_packed_b_flip_checksum_bit_mod127.argtypes = [vp, i32, i32, vp]
    L.abft_packed_b_destroy.argtypes = [vp]
    L.abft_packed_b_destroy.restype = None
    L.abft_packed_b_trim.argtypes = []
    L.abft_gemm_workspace_bytes.argtypes = [i32, vp]
    L.abft_gemm_workspace_bytes.restype = sz
    L.abft_workspace_init.argtypes = [vp, sz, vp]
    L.abft_gemm_u8s8s32_checked.argtypes = [vp, i64, i32, vp, vp, i64, vp, vp, ctypes.POINTER(abft_requant_t), vp, i64,
                                            vp, i32, u32, vp, sz, vp]
    L.abft_gemm_u8s8s32_checked_static.argtypes = [vp, i64, i32, vp, vp, i64, vp, vp, ctypes.POINTER(abft_requant_t), vp, i64,
                                                   vp, i32, u32, vp]
    L.abft_requantize_u8.argtypes = [vp, i64, i32, i32, vp, ctypes.POINTER(abft_requant_t), vp, i64, vp]
    L.abft_verify_rows.argtypes = [vp, i64, i32, i32, vp, vp, vp, vp]
    L.abft_row_checksum.argtypes = [vp, i64, i32, vp, vp, vp]
    L.abft_calib_copy.argtypes = [vp, vp, sz, vp]
    L.abft_clock_probe.argtypes = [vp, i32, vp]
    L.abft_mfma_peak_probe.argtypes = [vp, i32, vp]
    L.abft_clock_trace.argtypes = [vp]
    L.abft_recover_scratch_bytes.argtypes = [i32, i32, vp]
    L.abft_recover_scratch_bytes.restype = sz
    L.abft_recompute_flagged_rows.argtypes = [vp, i64, i32, vp, vp, i64, vp, vp, ctypes.POINTER(abft_requant_t), vp, i64,
                                              i32, vp, sz, vp, ctypes.POINTER(i32), ctypes.POINTER(i32)]
    L.abft_recompute_flagged_rows_async.argtypes = [vp, i64, i32, vp, vp, i64, vp, vp, ctypes.POINTER(abft_requant_t), vp, i64,
                                                    i32, vp, sz, vp, vp]
    L.abft_locate_scratch_bytes.argtypes = [vp]
    L.abft_locate_scratch_bytes.restype = sz
    L.abft_locate_correct.argtypes = [vp, i64, i32, vp, vp, i64, vp, vp, ctypes.POINTER(abft_requant_t), vp, i64, vp, vp, vp, sz, vp]
    L.abft_eb_pack_rowsum.argtypes = [vp, i64, vp, vp, i64, i32, u32, vp, ctypes.POINTER(vp)]
    L.abft_eb_table_dims.argtypes = [vp, ctypes.POINTER(i64), ctypes.POINTER(i32), ctypes.POINTER(i32), ctypes.POINTER(i32)]
    L.abft_eb_table_get_rowsums.argtypes = [vp, vp, vp]
    L.abft_eb_table_flip_bit.argtypes = [vp, i64, i32, i32, vp]
    L.abft_eb_table_destroy.argtypes = [vp]
    L.abft_eb_table_destroy.restype = None
    L.abft_eb_u8_checked.argtypes = [vp, vp, i64, vp, i64, vp, vp, i64, vp, vp, vp, ctypes.c_double, u32, vp]
    L.abft_w4_pack.argtypes = [vp, i64, vp, vp, i64, i32, i32, i32, i32, vp, ctypes.POINTER(vp)]
    L.abft_w4_dims.argtypes = [vp, ctypes.POINTER(i32), ctypes.POINTER(i32), ctypes.POINTER(i32), ctypes.POINTER(sz)]
    L.abft_w4_destroy.argtypes = [vp]
    L.abft_w4_destroy.restype = None
    L.abft_w4_gemv.argtypes = [vp, i64, i32, i32, vp, vp, i64, vp]
    kv = ctypes.POINTER(abft_kv_cache_t)
    L.abft_kv_code_bytes.argtypes = [kv]
    L.abft_kv_code_bytes.restype = sz
    L.abft_kv_plan.argtypes = [vp, vp, i32, i32, vp, i64, i32, vp, i32, vp, vp, vp, i64, vp, vp, vp]
    L.abft_kv_append.argtypes = [kv, vp, i64, i64, vp, i64, i64, i32, vp, i64, vp]
    L.abft_kv_read.argtypes = [kv, vp, i64, vp, i64, i64, vp, i64, i64, i32, vp]
    L.abft_kv_attention_workspace_bytes.argtypes = [kv, i32, i32, i32, i32]
    L.abft_kv_attention_workspace_bytes.restype = sz
    L.abft_kv_attention.argtypes = [kv, vp, i64, i64, i32, i64, i32, vp, i64, i32, vp, vp, i32, i32, i32, ctypes.c_float, vp, i64, i64, vp, vp, vp, sz, vp]
    return L


lib = _load()

try:
    from . import _fastcall
except ImportError as e:
    raise ImportError(f"{e}: build it with `python -m paper_2103_00130_amd.build`") from e
_fastcall.bind([ctypes.cast(f, ctypes.c_void_p).value for f in (lib.abft_gemm_u8s8s32_checked, lib.abft_eb_u8_checked, lib.abft_w4_gemv, lib.abft_kv_plan,
                                                                 lib.abft_kv_append, lib.abft_kv_read, lib.abft_kv_attention)],
               torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream)


def _check(rc: int):
    if rc != ABFT_OK:
        raise AbftError(rc, lib.abft_last_error().decode())


def _stream(stream=None) -> int:
    if stream is None:   # (torch.cuda.current_stream(), which makes a Stream object, takes 2.7 us)
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return stream.cuda_stream


def _ptr(t, dtype, name):
    if t is None:
        return None
    if not t.is_cuda:
        raise TypeError(f"{name} must be a device tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    return t.data_ptr()


def _lent(t, name):
    """(address, bytes) of the memory that a caller lends: a contiguous device tensor of any type, or none."""
    if t is None:
        return None, 0
    if not t.is_cuda:
        raise TypeError(f"{name} must be a device tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr(), t.numel() * t.element_size()


def _ld(t, name):
    if t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError(f"{name} must be 2-D with unit column stride")
    return t.stride(0) if t.shape[0] > 1 else max(t.stride(0), t.shape[1])


class PackedB:
    """Owner of an abft_packed_b handle."""

    def __init__(self, handle: int, K: int, N: int):
        self.handle, self.K, self.N = handle, K, N

    def destroy(self):
        if self.handle:
            lib.abft_packed_b_destroy(self.handle)   # (work that still reads the weight is waited for before its memory is used again)
            self.handle = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def abft_pack_b_checksum(B: torch.Tensor, b_is_transposed: bool = False, stream=None) -> PackedB:
    """B: int8 device tensor, K x N (or N x K when b_is_transposed)."""
    ptr = _ptr(B, torch.int8, "B")
    ldb = _ld(B, "B")
    K, N = (B.shape[1], B.shape[0]) if b_is_transposed else (B.shape[0], B.shape[1])
    out = ctypes.c_void_p()
    _check(lib.abft_pack_b_checksum(ptr, ldb, K, N, int(b_is_transposed), _stream(stream), ctypes.byref(out)))
    return PackedB(out.value, K, N)


def abft_packed_b_trim():
    """Gives the memory that is kept for weights to come on the current device back to it."""
    _check(lib.abft_packed_b_trim())


def abft_packed_b_dims(Bp: PackedB):
    k, n = ctypes.c_int(), ctypes.c_int()
    _check(lib.abft_packed_b_dims(Bp.handle, ctypes.byref(k), ctypes.byref(n)))
    return k.value, n.value


def abft_packed_b_get_checksum(Bp: PackedB, S_B: torch.Tensor, stream=None):
    assert S_B.numel() >= Bp.K
    _check(lib.abft_packed_b_get_checksum(Bp.handle, _ptr(S_B, torch.int32, "S_B"), _stream(stream)))


def abft_packed_b_get_checksum_mod127(Bp: PackedB, row_sum: torch.Tensor, stream=None):
    assert row_sum.numel() >= Bp.K
    _check(lib.abft_packed_b_get_checksum_mod127(Bp.handle, _ptr(row_sum, torch.int32, "row_sum"), _stream(stream)))


def abft_packed_b_get_col_offsets(Bp: PackedB, colsum: torch.Tensor, stream=None):
    assert colsum.numel() >= Bp.N
    _check(lib.abft_packed_b_get_col_offsets(Bp.handle, _ptr(colsum, torch.int32, "colsum"), _stream(stream)))


def abft_packed_b_flip_bit(Bp: PackedB, k: int, j: int, bit: int, stream=None):
    _check(lib.abft_packed_b_flip_bit(Bp.handle, int(k), int(j), int(bit), _stream(stream)))


def abft_packed_b_flip_checksum_bit(Bp: PackedB, k: int, bit: int, stream=None):
    _check(lib.abft_packed_b_flip_checksum_bit(Bp.handle, int(k), int(bit), _stream(stream)))


def abft_packed_b_flip_checksum_bit_mod127(Bp: PackedB, k: int, bit: int, stream=None):
    _check(lib.abft_packed_b_flip_checksum_bit_mod127(Bp.handle, int(k), int(bit), _stream(stream)))


def abft_gemm_workspace_bytes(M: int, Bp: PackedB) -> int:
    return int(lib.abft_gemm_workspace_bytes(int(M), Bp.handle))


def abft_workspace_init(workspace: torch.Tensor, stream=None):
    _check(lib.abft_workspace_init(*_lent(workspace, "workspace"), _stream(stream)))


def make_requant(zA: int, zC: int, mult: torch.Tensor, bias: torch.Tensor | None = None) -> abft_requant_t:
    """Host struct holding device pointers; keep `mult`/`bias` alive while it is in use."""
    return abft_requant_t(int(zA), int(zC), _ptr(mult, torch.float32, "mult"), int(mult.numel() > 1),
                          _ptr(bias, torch.int32, "bias"))


def make_injections(entries, device="cuda") -> torch.Tensor:
    """[(row, col, xor_mask), ...] -> device tensor laid out as abft_inject_t[n]."""
    import numpy as np
    arr = np.zeros((len(entries), 3), dtype=np.uint32)
    for t, (r, c, m) in enumerate(entries):
        arr[t] = (r, c, m)
    return torch.from_numpy(arr.view(np.int32)).to(device)


def abft_gemm_u8s8s32_checked(A, Bp: PackedB, C, row_flags, err_count, rq=None, Cq=None, inj=None, n_inj=0,
                              flags=ABFT_CHECK, workspace=None, stream=None):
    if rq is None or type(rq) is abft_requant_t:
        rc = _fastcall.gemm(A, Bp.handle, Bp.K, Bp.N, C, row_flags, err_count, rq, Cq, inj, n_inj, flags, workspace, stream)
        if rc is not None:
            if rc != ABFT_OK:
                _check(rc)
            return
    M = A.shape[0]
    if A.shape[1] != Bp.K:
        raise ValueError(f"A is {tuple(A.shape)}, packed B has K={Bp.K}")
    for t, nm in ((C, "C"), (Cq, "Cq")):
        if t is not None and tuple(t.shape) != (M, Bp.N):
            raise ValueError(f"{nm} must be {M}x{Bp.N}")
    if row_flags is not None and row_flags.numel() < M:
        raise ValueError("row_flags shorter than M")
    if inj is not None and inj.numel() < 3 * n_inj:
        raise ValueError("injection tensor shorter than n_inj entries")
    _check(lib.abft_gemm_u8s8s32_checked(
        _ptr(A, torch.uint8, "A"), _ld(A, "A"), M, Bp.handle,
        _ptr(C, torch.int32, "C"), 0 if C is None else _ld(C, "C"),
        _ptr(row_flags, torch.int32, "row_flags"), _ptr(err_count, torch.int32, "err_count"),
        None if rq is None else ctypes.byref(rq), _ptr(Cq, torch.uint8, "Cq"), 0 if Cq is None else _ld(Cq, "Cq"),
        _ptr(inj, torch.int32, "inj"), int(n_inj), int(flags),
        *_lent(workspace, "workspace"), _stream(stream)))


ABFT_STATIC_WS_MAX_M = 131072


def abft_gemm_u8s8s32_checked_static(A, Bp: PackedB, C, row_flags, err_count, rq=None, Cq=None, inj=None, n_inj=0,
                                     flags=ABFT_CHECK, stream=None):
    """The checked GEMM on the library's built-in workspace (no allocation, no workspace argument)."""
    M = A.shape[0]
    if A.shape[1] != Bp.K:
        raise ValueError(f"A is {tuple(A.shape)}, packed B has K={Bp.K}")
    for t, nm in ((C, "C"), (Cq, "Cq")):
        if t is not None and tuple(t.shape) != (M, Bp.N):
            raise ValueError(f"{nm} must be {M}x{Bp.N}")
    if row_flags is not None and row_flags.numel() < M:
        raise ValueError("row_flags shorter than M")
    if inj is not None and inj.numel() < 3 * n_inj:
        raise ValueError("injection tensor shorter than n_inj entries")
    _check(lib.abft_gemm_u8s8s32_checked_static(
        _ptr(A, torch.uint8, "A"), _ld(A, "A"), M, Bp.handle,
        _ptr(C, torch.int32, "C"), 0 if C is None else _ld(C, "C"),
        _ptr(row_flags, torch.int32, "row_flags"), _ptr(err_count, torch.int32, "err_count"),
        None if rq is None else ctypes.byref(rq), _ptr(Cq, torch.uint8, "Cq"), 0 if Cq is None else _ld(Cq, "Cq"),
        _ptr(inj, torch.int32, "inj"), int(n_inj), int(flags), _stream(stream)))


def abft_requantize_u8(C, Bp: PackedB, rq: abft_requant_t, Cq, stream=None):
    M, N = C.shape
    _check(lib.abft_requantize_u8(_ptr(C, torch.int32, "C"), _ld(C, "C"), M, N, Bp.handle, ctypes.byref(rq),
                                  _ptr(Cq, torch.uint8, "Cq"), _ld(Cq, "Cq"), _stream(stream)))


def abft_verify_rows(C, row_chk, row_flags, err_count=None, stream=None):
    M, N = C.shape
    _check(lib.abft_verify_rows(_ptr(C, torch.int32, "C"), _ld(C, "C"), M, N, _ptr(row_chk, torch.int32, "row_chk"),
                                _ptr(row_flags, torch.int32, "row_flags"), _ptr(err_count, torch.int32, "err_count"),
                                _stream(stream)))


def abft_row_checksum(A, Bp: PackedB, row_chk, stream=None):
    _check(lib.abft_row_checksum(_ptr(A, torch.uint8, "A"), _ld(A, "A"), A.shape[0], Bp.handle,
                                 _ptr(row_chk, torch.int32, "row_chk"), _stream(stream)))


def abft_recover_scratch_bytes(M: int, max_rows_per_pass: int, Bp: PackedB) -> int:
    return int(lib.abft_recover_scratch_bytes(M, max_rows_per_pass, Bp.handle))


def abft_recompute_flagged_rows(A, Bp: PackedB, C, row_flags, err_count=None, rq=None, Cq=None, max_rows_per_pass=256,
                                scratch=None, stream=None):
    """Recomputes the flagged rows in place (synchronises the stream).  Returns
    (rows found flagged, rows still flagged after the recomputation)."""
    M = A.shape[0]
    if scratch is None:
        scratch = torch.empty(abft_recover_scratch_bytes(M, max_rows_per_pass, Bp), dtype=torch.uint8, device=A.device)
    before, after = ctypes.c_int(0), ctypes.c_int(0)
    _check(lib.abft_recompute_flagged_rows(
        _ptr(A, torch.uint8, "A"), _ld(A, "A"), M, Bp.handle,
        _ptr(C, torch.int32, "C"), _ld(C, "C") if C is not None else 0,
        _ptr(row_flags, torch.int32, "row_flags"), _ptr(err_count, torch.int32, "err_count"),
        ctypes.byref(rq) if rq is not None else None, _ptr(Cq, torch.uint8, "Cq"), _ld(Cq, "Cq") if Cq is not None else 0,
        max_rows_per_pass, *_lent(scratch, "scratch"), _stream(stream), ctypes.byref(before), ctypes.byref(after)))
    return before.value, after.value


def abft_recompute_flagged_rows_async(A, Bp: PackedB, C, row_flags, err_count=None, rq=None, Cq=None, max_rows=64,
                                      scratch=None, status=None, stream=None):
    """Recomputes up to max_rows flagged rows in place without synchronising; returns the device tensor
    `status` (rows found flagged, rows still flagged)."""
    M = A.shape[0]
    if scratch is None:
        scratch = torch.empty(abft_recover_scratch_bytes(M, max_rows, Bp), dtype=torch.uint8, device=A.device)
    if status is None:
        status = torch.empty(2, dtype=torch.int32, device=A.device)
    _check(lib.abft_recompute_flagged_rows_async(
        _ptr(A, torch.uint8, "A"), _ld(A, "A"), M, Bp.handle,
        _ptr(C, torch.int32, "C"), _ld(C, "C") if C is not None else 0,
        _ptr(row_flags, torch.int32, "row_flags"), _ptr(err_count, torch.int32, "err_count"),
        ctypes.byref(rq) if rq is not None else None, _ptr(Cq, torch.uint8, "Cq"), _ld(Cq, "Cq") if Cq is not None else 0,
        max_rows, *_lent(scratch, "scratch"), _ptr(status, torch.int32, "status"), _stream(stream)))
    return status


def abft_locate_scratch_bytes(Bp: PackedB) -> int:
    return int(lib.abft_locate_scratch_bytes(Bp.handle))


def abft_locate_correct(A, Bp: PackedB, C, row_flags, err_count=None, rq=None, Cq=None, col_flags=None, report=None,
                        scratch=None, stream=None):
    """Eq. 2a column check + repair of a single located element, in place, asynchronously.  Returns the device
    tensor holding the abft_locate_t report (8 int32: status, row, col, old, new, rows flagged, columns violated, -)."""
    M = A.shape[0]
    if scratch is None:
        scratch = torch.empty(abft_locate_scratch_bytes(Bp), dtype=torch.uint8, device=A.device)
    if report is None:
        report = torch.empty(8, dtype=torch.int32, device=A.device)
    if col_flags is not None and col_flags.numel() < Bp.N:
        raise ValueError("col_flags shorter than N")
    _check(lib.abft_locate_correct(
        _ptr(A, torch.uint8, "A"), _ld(A, "A"), M, Bp.handle, _ptr(C, torch.int32, "C"), _ld(C, "C"),
        _ptr(row_flags, torch.int32, "row_flags"), _ptr(err_count, torch.int32, "err_count"),
        ctypes.byref(rq) if rq is not None else None, _ptr(Cq, torch.uint8, "Cq"), _ld(Cq, "Cq") if Cq is not None else 0,
        _ptr(col_flags, torch.int32, "col_flags"), _ptr(report, torch.int32, "report"),
        *_lent(scratch, "scratch"), _stream(stream)))
    return report


def abft_calib_copy(src, dst, stream=None):
    if src.numel() * src.element_size() != dst.numel() * dst.element_size():
        raise ValueError("abft_calib_copy: src and dst differ in size")
    if not (src.is_cuda and dst.is_cuda and src.is_contiguous() and dst.is_contiguous()):
        raise ValueError("abft_calib_copy: contiguous device tensors expected")
    _check(lib.abft_calib_copy(src.data_ptr(), dst.data_ptr(), src.numel() * src.element_size(), _stream(stream)))


def abft_clock_probe(out: torch.Tensor, microseconds: int, stream=None):
    """out: int64 device tensor of 4 (wall ticks at 100 MHz and shader cycles, start and end)."""
    if out.dtype != torch.int64 or out.numel() < 4 or not out.is_cuda:
        raise ValueError("abft_clock_probe: out must be an int64 device tensor of at least 4 entries")
    _check(lib.abft_clock_probe(out.data_ptr(), int(microseconds), _stream(stream)))


def abft_mfma_peak_probe(out: torch.Tensor, iters: int, stream=None):
    """out: int64 device tensor of 4 * 256 (shader cycles, wall ticks before; the same after; per workgroup)."""
    if out.dtype != torch.int64 or out.numel() < 4 * 256 or not out.is_cuda:
        raise ValueError("abft_mfma_peak_probe: out must be an int64 device tensor of at least 1024 entries")
    _check(lib.abft_mfma_peak_probe(out.data_ptr(), int(iters), _stream(stream)))


def abft_clock_trace(buf: torch.Tensor | None):
    """Diagnostic library only: buf int64 device tensor, 6 entries per workgroup of the largest grid; None = off."""
    _check(lib.abft_clock_trace(None if buf is None else buf.data_ptr()))


class Workspace:
    """A zero-initialised workspace tensor sized for (M, Bp)."""

    def __init__(self, M: int, Bp: PackedB, device="cuda"):
        self.tensor = torch.empty(abft_gemm_workspace_bytes(M, Bp) // 4, dtype=torch.int32, device=device)
        abft_workspace_init(self.tensor)


# ---------------------------------------------------------------------------------------------
# include/abft_eb.h

class EbTable:
    """Owner of an abft_eb_table handle."""

    def __init__(self, handle: int, rows: int, d: int):
        self.handle, self.rows, self.d = handle, rows, d

    def destroy(self):
        if self.handle:
            torch.cuda.synchronize()
            lib.abft_eb_table_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def abft_eb_pack_rowsum(T: torch.Tensor, scale: torch.Tensor, bias: torch.Tensor, flags: int = 0, stream=None) -> EbTable:
    """T: uint8 device tensor, rows x d codes (rows x d/2 bytes with ABFT_EB_PACK_INT4); scale, bias: float32 [rows]."""
    ptr = _ptr(T, torch.uint8, "T")
    ldt = _ld(T, "T")
    rows, d = T.shape
    if flags & ABFT_EB_PACK_INT4:
        d *= 2
    if scale.numel() != rows or bias.numel() != rows or not scale.is_contiguous() or not bias.is_contiguous():
        raise ValueError("scale and bias must be contiguous with one entry per table row")
    out = ctypes.c_void_p()
    _check(lib.abft_eb_pack_rowsum(ptr, ldt, _ptr(scale, torch.float32, "scale"), _ptr(bias, torch.float32, "bias"),
                                   rows, d, int(flags), _stream(stream), ctypes.byref(out)))
    return EbTable(out.value, rows, d)


def abft_eb_table_dims(Tp: EbTable):
    rows, d, rec, bits = ctypes.c_int64(), ctypes.c_int(), ctypes.c_int(), ctypes.c_int()
    _check(lib.abft_eb_table_dims(Tp.handle, ctypes.byref(rows), ctypes.byref(d), ctypes.byref(rec), ctypes.byref(bits)))
    return rows.value, d.value, rec.value, bits.value


def abft_eb_table_get_rowsums(Tp: EbTable, C_T: torch.Tensor, stream=None):
    if C_T.numel() < Tp.rows or not C_T.is_contiguous():
        raise ValueError("C_T must be contiguous with one entry per table row")
    _check(lib.abft_eb_table_get_rowsums(Tp.handle, _ptr(C_T, torch.int32, "C_T"), _stream(stream)))


def abft_eb_table_flip_bit(Tp: EbTable, row: int, col: int, bit: int, stream=None):
    _check(lib.abft_eb_table_flip_bit(Tp.handle, int(row), int(col), int(bit), _stream(stream)))


def abft_eb_u8_checked(Tp: EbTable, indices: torch.Tensor, offsets: torch.Tensor, R: torch.Tensor,
                       bag_flags: torch.Tensor | None, weights: torch.Tensor | None = None,
                       rsum: torch.Tensor | None = None, csum: torch.Tensor | None = None,
                       rel_bound: float = 1e-5, flags: int = 0, stream=None):
    """Algorithm 2 for a batch: offsets has one entry more than there are lookups."""
    rc = _fastcall.eb(Tp.handle, Tp.d, indices, offsets, R, bag_flags, weights, rsum, csum, rel_bound, flags, stream)
    if rc is not None:
        if rc != ABFT_OK:
            _check(rc)
        return
    n_bags = offsets.numel() - 1
    if n_bags < 0 or not offsets.is_contiguous() or not indices.is_contiguous():
        raise ValueError("indices and offsets must be contiguous; offsets needs n_bags + 1 entries")
    if R.dim() != 2 or R.shape[0] < n_bags or R.shape[1] != Tp.d:
        raise ValueError("R must be n_bags x d")
    for name, t in (("bag_flags", bag_flags), ("rsum", rsum), ("csum", csum)):
        if t is not None and (t.numel() < n_bags or not t.is_contiguous()):
            raise ValueError(f"{name} must be contiguous with one entry per lookup")
    if weights is not None and (weights.numel() != indices.numel() or not weights.is_contiguous()):
        raise ValueError("weights must be contiguous with one entry per index")
    _check(lib.abft_eb_u8_checked(Tp.handle, _ptr(indices, torch.int64, "indices"), indices.numel(),
                                  _ptr(offsets, torch.int64, "offsets"), n_bags, _ptr(weights, torch.float32, "weights"),
                                  _ptr(R, torch.float32, "R"), _ld(R, "R"), _ptr(bag_flags, torch.int32, "bag_flags"),
                                  _ptr(rsum, torch.float64, "rsum"), _ptr(csum, torch.float64, "csum"),
                                  float(rel_bound), int(flags), _stream(stream)))


# ---------------------------------------------------------------------------------------------
# Operators of a decoding step: 4-bit weights (abft_gemm.h), the 8-bit key/value cache (abft_eb.h)

_TYPES = {torch.float32: ABFT_TYPE_F32, torch.float16: ABFT_TYPE_F16, torch.bfloat16: ABFT_TYPE_BF16}


def _typed(t, name):
    """(address, ABFT_TYPE_*) of a device tensor of activations."""
    if not t.is_cuda:
        raise TypeError(f"{name} must be a device tensor")
    if t.dtype not in _TYPES:
        raise TypeError(f"{name} must be float32, float16 or bfloat16, got {t.dtype}")
    return t.data_ptr(), _TYPES[t.dtype]


def _entries(t, dtype, n, name):
    """The address of a contiguous device tensor of at least n entries."""
    if t.numel() < n or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous with at least {n} entries")
    return _ptr(t, dtype, name)


class W4Weight:
    """Owner of an abft_w4 handle."""

    def __init__(self, handle: int, N: int, K: int, group: int):
        self.handle, self.N, self.K, self.group = handle, N, K, group

    def destroy(self):
        if self.handle:
            torch.cuda.synchronize()
            lib.abft_w4_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def abft_w4_pack(W: torch.Tensor, scale: torch.Tensor, bias: torch.Tensor | None = None, K: int | None = None, group: int = 128,
                 stream=None) -> W4Weight:
    """W: uint8 device tensor, N x ceil(K / 2) bytes of 4-bit codes (the even column in the low half; K defaults to twice the
    bytes); scale, bias: N x ceil(K / group), of one type.  The weight is scale * code + bias, or scale * (code - 8) without bias."""
    ptr = _ptr(W, torch.uint8, "W")
    ldw = _ld(W, "W")
    N, row = W.shape
    if K is None:
        K = 2 * row
    if row != (K + 1) // 2:
        raise ValueError(f"W has rows of {row} bytes, K={K} needs {(K + 1) // 2}")
    groups = -(-K // group) if group > 0 else 0
    s_ptr, s_type = _typed(scale, "scale")
    lds = _ld(scale, "scale")
    if tuple(scale.shape) != (N, groups):
        raise ValueError(f"scale must be {N}x{groups}")
    b_ptr = None
    if bias is not None:
        b_ptr, b_type = _typed(bias, "bias")
        if b_type != s_type or tuple(bias.shape) != (N, groups) or _ld(bias, "bias") != lds:
            raise ValueError("bias must have the type, shape and strides of scale")
    out = ctypes.c_void_p()
    _check(lib.abft_w4_pack(ptr, ldw, s_ptr, b_ptr, lds, s_type, N, K, group, _stream(stream), ctypes.byref(out)))
    return W4Weight(out.value, N, K, group)


def abft_w4_dims(Wp: W4Weight):
    n, k, g, size = ctypes.c_int(), ctypes.c_int(), ctypes.c_int(), ctypes.c_size_t()
    _check(lib.abft_w4_dims(Wp.handle, ctypes.byref(n), ctypes.byref(k), ctypes.byref(g), ctypes.byref(size)))
    return n.value, k.value, g.value, size.value


def abft_w4_gemv(X: torch.Tensor, Wp: W4Weight, Y: torch.Tensor, stream=None):
    """Y = X W^T: X M x K, Y M x N, both float32, float16 or bfloat16."""
    rc = _fastcall.w4(X, Wp.handle, Wp.N, Wp.K, Y, stream)
    if rc is not None:
        if rc != ABFT_OK:
            _check(rc)
        return
    x_ptr, x_type = _typed(X, "X")
    y_ptr, y_type = _typed(Y, "Y")
    ldx, ldy = _ld(X, "X"), _ld(Y, "Y")
    if X.shape[1] != Wp.K or tuple(Y.shape) != (X.shape[0], Wp.N):
        raise ValueError(f"X is {tuple(X.shape)} and Y {tuple(Y.shape)}, the weight has K={Wp.K}, N={Wp.N}")
    if x_type != y_type:
        raise TypeError("X and Y must have the same type")
    _check(lib.abft_w4_gemv(x_ptr, ldx, x_type, X.shape[0], Wp.handle, y_ptr, ldy, _stream(stream)))


class KvCache:
    """The buffers of an 8-bit key/value cache (abft_kv_cache_t): k_codes [n_blocks][heads][block_tokens][columns], v_codes
    [n_blocks][heads][block_tokens / 16][columns][16], k_scale and v_scale [n_blocks][heads]; columns is head_dim rounded up to 64."""

    def __init__(self, n_blocks: int, heads: int, head_dim: int, block_tokens: int = 64, device="cuda"):
        self.n_blocks, self.heads, self.head_dim, self.block_tokens = int(n_blocks), int(heads), int(head_dim), int(block_tokens)
        if not lib.abft_kv_code_bytes(ctypes.byref(abft_kv_cache_t(None, None, None, None, *self._sizes()))):
            raise ValueError(f"no cache of {n_blocks} blocks of {block_tokens} tokens, {heads} heads of {head_dim}: block_tokens must be 16, 32, 64 or 128, "
                             "head_dim 1..256, and there must be blocks and heads")
        if torch.device(device).type != "cuda":
            raise TypeError(f"a cache lies on a device, not on {device}: its addresses go to kernels")
        cols = (self.head_dim + 63) // 64 * 64
        self.k_codes = torch.zeros((self.n_blocks, self.heads, self.block_tokens, cols), dtype=torch.int8, device=device)
        self.v_codes = torch.zeros((self.n_blocks, self.heads, self.block_tokens // 16, cols, 16), dtype=torch.int8, device=device)
        self.k_scale = torch.zeros((self.n_blocks, self.heads), dtype=torch.float32, device=device)
        self.v_scale = torch.zeros((self.n_blocks, self.heads), dtype=torch.float32, device=device)
        self.struct = abft_kv_cache_t(self.k_codes.data_ptr(), self.v_codes.data_ptr(), self.k_scale.data_ptr(), self.v_scale.data_ptr(), *self._sizes())
        self.ref = ctypes.byref(self.struct)
        self.address = ctypes.addressof(self.struct)

    def _sizes(self):
        return self.n_blocks, self.heads, self.head_dim, self.block_tokens

    def load_codes(self, k, v, k_scale, v_scale):
        """Fill the cache from codes [n_blocks][heads][block_tokens][head_dim] and scales [n_blocks][heads] (a saved cache)."""
        self.k_codes[..., :self.head_dim] = k
        self.v_codes[..., :self.head_dim, :] = v.unflatten(2, (self.block_tokens // 16, 16)).transpose(3, 4)
        self.k_scale.copy_(k_scale)
        self.v_scale.copy_(v_scale)

    def codes(self):
        """(k, v): the codes as [n_blocks][heads][block_tokens][head_dim]."""
        return self.k_codes[..., :self.head_dim], self.v_codes[..., :self.head_dim, :].transpose(3, 4).flatten(2, 3)


def abft_kv_plan(ctx_len, new_len, block_tokens: int, table, free_blocks, seq_len, cu_new, slots, req_flags, taken, stream=None):
    """Block tables and slots of a step; table (int32, requests x blocks) is extended in place, seq_len, cu_new, slots (int64),
    req_flags and taken are overwritten."""
    rc = _fastcall.plan(ctx_len, new_len, block_tokens, table, free_blocks, seq_len, cu_new, slots, req_flags, taken, stream)
    if rc is not None:
        if rc != ABFT_OK:
            _check(rc)
        return
    R = ctx_len.numel()
    if table.dim() != 2 or table.shape[0] != R:
        raise ValueError("table must be 2-D with a row for each request")
    ldt = max(_ld(table, "table"), table.shape[1])
    _check(lib.abft_kv_plan(_entries(ctx_len, torch.int32, R, "ctx_len"), _entries(new_len, torch.int32, R, "new_len"), R, int(block_tokens),
                            _ptr(table, torch.int32, "table"), ldt, table.shape[1], _entries(free_blocks, torch.int32, 0, "free_blocks"),
                            free_blocks.numel(), _entries(seq_len, torch.int32, R, "seq_len"), _entries(cu_new, torch.int32, R + 1, "cu_new"),
                            _entries(slots, torch.int64, 0, "slots"), slots.numel(), _entries(req_flags, torch.int32, R, "req_flags"),
                            _entries(taken, torch.int32, 1, "taken"), _stream(stream)))


def _kv_rows(t, cache, n, name, heads=None):
    """(address, stride between tokens, stride between heads) of n x heads x head_dim values."""
    heads = cache.heads if heads is None else heads
    if tuple(t.shape) != (n, heads, cache.head_dim) or (cache.head_dim > 1 and t.stride(2) != 1):
        raise ValueError(f"{name} must be {n} x {heads} x {cache.head_dim} with unit column stride, got {tuple(t.shape)}")
    return t.data_ptr(), t.stride(0), t.stride(1)


def abft_kv_append(cache: KvCache, K, V, slots, stream=None):
    """Quantizes K and V (tokens x heads x head_dim) into the cache at `slots` (int64, as abft_kv_plan gives them)."""
    rc = _fastcall.append(cache.address, cache.heads, cache.head_dim, K, V, slots, stream)
    if rc is not None:
        if rc != ABFT_OK:
            _check(rc)
        return
    T = slots.numel()
    _, k_type = _typed(K, "K")
    _, v_type = _typed(V, "V")
    if k_type != v_type:
        raise TypeError("K and V must have the same type")
    _check(lib.abft_kv_append(cache.ref, *_kv_rows(K, cache, T, "K"), *_kv_rows(V, cache, T, "V"), k_type, _entries(slots, torch.int64, T, "slots"),
                              T, _stream(stream)))


def abft_kv_read(cache: KvCache, slots, K=None, V=None, stream=None):
    """The tokens at `slots` as values, into K and V (tokens x heads x head_dim); either may be None."""
    rc = _fastcall.read(cache.address, cache.heads, cache.head_dim, slots, K, V, stream)
    if rc is not None:
        if rc != ABFT_OK:
            _check(rc)
        return
    T = slots.numel()
    types = {_typed(t, name)[1] for t, name in ((K, "K"), (V, "V")) if t is not None}
    if len(types) > 1:
        raise TypeError("K and V must have the same type")
    none = (None, 0, 0)
    _check(lib.abft_kv_read(cache.ref, _entries(slots, torch.int64, T, "slots"), T, *(none if K is None else _kv_rows(K, cache, T, "K")),
                            *(none if V is None else _kv_rows(V, cache, T, "V")), types.pop() if types else ABFT_TYPE_F32, _stream(stream)))


def abft_kv_attention_workspace_bytes(cache: KvCache, n_req: int, q_heads: int, max_new: int, max_len: int) -> int:
    return int(lib.abft_kv_attention_workspace_bytes(cache.ref, int(n_req), int(q_heads), int(max_new), int(max_len)))


class KvWorkspace:
    """A workspace tensor for abft_kv_attention on up to n_req requests of up to max_new new tokens and max_len tokens in all (None
    where none is needed)."""

    def __init__(self, cache: KvCache, n_req: int, q_heads: int, max_new: int, max_len: int):
        size = abft_kv_attention_workspace_bytes(cache, n_req, q_heads, max_new, max_len)
        self.tensor = torch.empty(size // 4, dtype=torch.float32, device=cache.k_codes.device) if size else None


def abft_kv_attention(cache: KvCache, Q, table, seq_len, cu_new, O, max_new: int, max_len: int, scale: float | None = None, lse=None,
                      req_flags=None, workspace=None, stream=None):
    """Attention of the rows of Q (new tokens x query heads x head_dim) over their requests' tokens, into O.  scale: 1 / sqrt(head_dim)
    unless given."""
    if scale is None:
        scale = cache.head_dim ** -0.5
    rc = _fastcall.attention(cache.address, cache.head_dim, Q, table, seq_len, cu_new, O, max_new, max_len, scale, lse, req_flags, workspace, stream)
    if rc is not None:
        if rc != ABFT_OK:
            _check(rc)
        return
    if Q.dim() != 3 or table.dim() != 2:
        raise ValueError("Q must be rows x query heads x head_dim and table requests x blocks")
    n_rows, q_heads = Q.shape[:2]
    R = seq_len.numel()
    _, q_type = _typed(Q, "Q")
    _, o_type = _typed(O, "O")
    if q_type != o_type:
        raise TypeError("Q and O must have the same type")
    if table.shape[0] != R:
        raise ValueError("table must have a row for each request")
    _check(lib.abft_kv_attention(
        cache.ref, *_kv_rows(Q, cache, n_rows, "Q", q_heads), q_type, n_rows, q_heads, _ptr(table, torch.int32, "table"),
        max(_ld(table, "table"), table.shape[1]), table.shape[1], _entries(seq_len, torch.int32, R, "seq_len"),
        _entries(cu_new, torch.int32, R + 1, "cu_new"), R, int(max_new), int(max_len), float(scale),
        *_kv_rows(O, cache, n_rows, "O", q_heads), None if lse is None else _entries(lse, torch.float32, n_rows * q_heads, "lse"),
        None if req_flags is None else _entries(req_flags, torch.int32, R, "req_flags"), *_lent(workspace, "workspace"), _stream(stream)))
