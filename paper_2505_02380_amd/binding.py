"""ctypes binding of include/entro.h: same names, argument marshalling only."""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass
from typing import List, Optional, Sequence

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))

ENTRO_UNSIGNED, ENTRO_ASYMMETRIC = 0, 1
ENTRO_U8, ENTRO_U4_PACKED, ENTRO_F32, ENTRO_BF16 = 0, 1, 2, 3
ENTRO_OP_DECODE, ENTRO_OP_DEQUANT, ENTRO_OP_GEMV = 0, 1, 2
ENTRO_ROTARY_HALVES, ENTRO_ROTARY_PAIRS = 0, 1
ENTRO_NORM_NONE, ENTRO_NORM_RMS, ENTRO_NORM_CENTRED = 0, 1, 2
ENTRO_CONTEXT_AS_TRAINED, ENTRO_CONTEXT_LINEAR, ENTRO_CONTEXT_BY_PARTS = 0, 1, 2
ENTRO_OK = 0
(ENTRO_ERR_NULL, ENTRO_ERR_BITS, ENTRO_ERR_SCHEME, ENTRO_ERR_SIZE, ENTRO_ERR_NONFINITE, ENTRO_ERR_RANGE,
 ENTRO_ERR_SYMBOL, ENTRO_ERR_CODE_TOO_LONG, ENTRO_ERR_CAPACITY, ENTRO_ERR_CORRUPT, ENTRO_ERR_ALIGN,
 ENTRO_ERR_DEVICE) = range(1, 13)


class QParams(C.Structure):
    _fields_ = [("scale", C.c_float), ("zero_point", C.c_int32), ("bits", C.c_int32), ("scheme", C.c_int32)]


class Codebook(C.Structure):
    _fields_ = [("bits", C.c_int32), ("n_used", C.c_int32), ("max_len", C.c_int32), ("reserved", C.c_int32),
                ("len", C.c_uint8 * 256), ("code", C.c_uint32 * 256)]

    def lengths(self) -> np.ndarray:
        return np.frombuffer(self.len, dtype=np.uint8, count=1 << self.bits).copy()

    def codes(self) -> np.ndarray:
        return np.frombuffer(self.code, dtype=np.uint32, count=1 << self.bits).copy()


class CTensor(C.Structure):
    _fields_ = [("stream", C.c_void_p), ("stream_bytes", C.c_uint64), ("offsets", C.c_void_p),
                ("n", C.c_uint64), ("chunk_symbols", C.c_uint32), ("rows", C.c_uint32), ("cols", C.c_uint32),
                ("sub_symbols", C.c_uint32), ("cb", C.POINTER(Codebook)), ("qp", QParams), ("x", C.c_void_p),
                ("out", C.c_void_p), ("sub_bits", C.c_void_p)]


class Plan(C.Structure):
    _fields_ = [("workspace", C.c_void_p), ("workspace_bytes", C.c_uint64), ("op", C.c_uint32),
                ("out", C.c_uint32), ("count", C.c_uint32), ("n_items", C.c_uint32), ("n_fix", C.c_uint32),
                ("item_units", C.c_uint32), ("pair_tables", C.c_uint32), ("gemv_multirow", C.c_uint32), ("wide_tables", C.c_uint32), ("shared_wave_bytes", C.c_uint32), ("off_tensors", C.c_uint64), ("off_items", C.c_uint64),
                ("off_partials", C.c_uint64), ("off_fix", C.c_uint64)]


class CCache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p), ("layers", C.c_uint32),
                ("pages", C.c_uint32), ("page_tokens", C.c_uint32), ("kv_heads", C.c_uint32), ("head_dim", C.c_uint32),
                ("reserved", C.c_uint32)]


class CCacheTable(C.Structure):
    _fields_ = [("slots", C.c_void_p), ("lengths", C.c_void_p), ("seqs", C.c_uint32), ("stride", C.c_uint32)]


class CCacheRows(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_token_stride", C.c_uint64), ("k_head_stride", C.c_uint64),
                ("v_token_stride", C.c_uint64), ("v_head_stride", C.c_uint64), ("start", C.c_void_p), ("tokens", C.c_uint32),
                ("max_new", C.c_uint32), ("type", C.c_uint32), ("layer", C.c_uint32)]


class CCacheQuery(C.Structure):
    _fields_ = [("q", C.c_void_p), ("out", C.c_void_p), ("lse", C.c_void_p), ("q_token_stride", C.c_uint64),
                ("q_head_stride", C.c_uint64), ("out_token_stride", C.c_uint64), ("out_head_stride", C.c_uint64),
                ("start", C.c_void_p), ("tokens", C.c_uint32), ("max_new", C.c_uint32), ("max_len", C.c_uint32),
                ("q_heads", C.c_uint32), ("type", C.c_uint32), ("layer", C.c_uint32), ("window", C.c_uint32), ("sinks", C.c_uint32),
                ("scale", C.c_float), ("reserved", C.c_uint32)]


class CCacheGroups(C.Structure):
    _fields_ = [("first", C.c_void_p), ("shared", C.c_void_p), ("groups", C.c_uint32), ("max_seqs", C.c_uint32), ("max_shared", C.c_uint32),
                ("max_own", C.c_uint32)]


class CRotary(C.Structure):
    _fields_ = [("turns", C.c_void_p), ("q_gain", C.c_void_p), ("k_gain", C.c_void_p), ("q_gain_stride", C.c_uint32),
                ("k_gain_stride", C.c_uint32), ("dims", C.c_uint32), ("layout", C.c_uint32), ("norm", C.c_uint32), ("eps", C.c_float),
                ("amplitude", C.c_float), ("reserved", C.c_uint32)]


class CRotaryRows(C.Structure):
    _fields_ = [("x", C.c_void_p), ("y", C.c_void_p), ("x_token_stride", C.c_uint64), ("x_head_stride", C.c_uint64),
                ("y_token_stride", C.c_uint64), ("y_head_stride", C.c_uint64), ("heads", C.c_uint32), ("reserved", C.c_uint32)]


class EntroError(RuntimeError):
    def __init__(self, status: int, what: str):
        msg = f"{what}: {entro_status_string(status)} (status {status})"
        if status == ENTRO_ERR_DEVICE:
            msg += f" [{entro_last_device_error()}]"
        super().__init__(msg)
        self.status = status


_lib = None


def library_path() -> str:
    return os.path.join(HERE, "libentro.so")


def lib():
    """Load libentro.so (built in-tree by paper_2505_02380_amd/build.py).  No CPU fallback exists."""
    global _lib
    if _lib is not None:
        return _lib
    path = library_path()
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: run `python -m paper_2505_02380_amd.build` "
                           "(or __graft_entry__.build()) first; there is no CPU fallback")
    L = C.CDLL(path)
    u8p, u64p, f32p = C.POINTER(C.c_uint8), C.POINTER(C.c_uint64), C.POINTER(C.c_float)
    cbp, tp, pp = C.POINTER(Codebook), C.POINTER(CTensor), C.POINTER(Plan)
    kp, kt = C.POINTER(CCache), C.POINTER(CCacheTable)
    sig = {
        "entro_quantize": (C.c_int, [f32p, C.c_uint64, C.c_int, C.c_int, u8p, C.POINTER(QParams)]),
        "entro_build_codebook": (C.c_int, [u8p, C.c_uint64, C.c_int, cbp]),
        "entro_codebook_from_counts": (C.c_int, [u64p, C.c_int, cbp]),
        "entro_codebook_from_lengths": (C.c_int, [u8p, C.c_int, cbp]),
        "entro_codebook_from_counts_limited": (C.c_int, [u64p, C.c_int, C.c_int, cbp]),
        "entro_build_codebook_limited": (C.c_int, [u8p, C.c_uint64, C.c_int, C.c_int, cbp]),
        "entro_num_chunks": (C.c_uint64, [C.c_uint64, C.c_uint32]),
        "entro_encode_bound": (C.c_uint64, [C.c_uint64, cbp]),
        "entro_encode": (C.c_int, [u8p, C.c_uint64, cbp, C.c_uint32, u8p, C.c_uint64, u64p, u64p]),
        "entro_check_offsets": (C.c_int, [u64p, C.c_uint64, C.c_uint32, C.c_uint64, cbp]),
        "entro_sub_index": (C.c_int, [u8p, C.c_uint64, cbp, C.c_uint32, C.c_uint32, C.POINTER(C.c_uint16)]),
        "entro_bits_saved": (C.c_double, [C.c_int, C.c_double]),
        "entro_theoretical_speedup": (C.c_double, [C.c_int, C.c_double]),
        "entro_status_string": (C.c_char_p, [C.c_int]),
        "entro_decode": (C.c_int, [tp, C.c_int, C.c_void_p]),
        "entro_decode_dequant": (C.c_int, [tp, C.c_int, C.c_void_p]),
        "entro_gemv_workspace_bytes": (C.c_uint64, [tp]),
        "entro_decode_gemv": (C.c_int, [tp, C.c_int, C.c_void_p, C.c_uint64, C.c_void_p]),
        "entro_decode_gemv_static": (C.c_int, [tp, C.c_int, C.c_void_p]),
        "entro_workspace_bytes": (C.c_uint64, [tp, C.c_uint32, C.c_int]),
        "entro_plan_init": (C.c_int, [pp, tp, C.c_uint32, C.c_int, C.c_int, C.c_void_p, C.c_uint64, C.c_void_p]),
        "entro_plan_staging_bytes": (C.c_uint64, [tp, C.c_uint32, C.c_int]),
        "entro_plan_init_staged": (C.c_int, [pp, tp, C.c_uint32, C.c_int, C.c_int, C.c_void_p, C.c_uint64, C.c_void_p, C.c_uint64,
                                             C.c_void_p]),
        "entro_plan_run": (C.c_int, [pp, C.c_void_p]),
        "entro_decode_batch": (C.c_int, [tp, C.c_uint32, C.c_int, C.c_void_p, C.c_uint64, C.c_void_p]),
        "entro_decode_dequant_batch": (C.c_int, [tp, C.c_uint32, C.c_int, C.c_void_p, C.c_uint64, C.c_void_p]),
        "entro_decode_gemv_batch": (C.c_int, [tp, C.c_uint32, C.c_int, C.c_void_p, C.c_uint64, C.c_void_p]),
        "entro_last_device_error": (C.c_char_p, []),
        "entro_range_device": (C.c_int, [C.c_void_p, C.c_uint64, C.c_void_p, C.c_void_p]),
        "entro_qparams_from_range": (C.c_int, [C.c_float, C.c_float, C.c_uint32, C.c_int, C.c_int, C.POINTER(QParams)]),
        "entro_scheme_for_range": (C.c_int, [C.c_float, C.c_float]),
        "entro_quantize_device": (C.c_int, [C.c_void_p, C.c_uint64, C.POINTER(QParams), C.c_void_p, C.c_void_p, C.c_void_p]),
        "entro_encoded_bytes": (C.c_uint64, [u64p, cbp]),
        "entro_encode_device": (C.c_int, [C.c_void_p, C.c_uint64, cbp, C.c_uint32, C.c_void_p, C.c_uint64, C.c_void_p,
                                          C.c_void_p, C.c_void_p]),
        "entro_encode_device_status": (C.c_int, [C.c_uint32]),
        "entro_cache_width": (C.c_uint32, [C.c_uint32]),
        "entro_cache_codes_bytes": (C.c_uint64, [kp]),
        "entro_cache_append": (C.c_int, [kp, kt, C.POINTER(CCacheRows), C.c_void_p]),
        "entro_cache_read": (C.c_int, [kp, kt, C.POINTER(CCacheRows), C.c_void_p]),
        "entro_cache_attend_workspace_bytes": (C.c_uint64, [kp, kt, C.POINTER(CCacheQuery)]),
        "entro_cache_attend": (C.c_int, [kp, kt, C.POINTER(CCacheQuery), C.c_void_p, C.c_uint64, C.c_void_p]),
        "entro_cache_pages_workspace_bytes": (C.c_uint64, [kp, kt, kt]),
        "entro_cache_regroup": (C.c_int, [kp, kt, C.c_void_p, C.c_void_p, C.c_uint32, C.c_uint32, kt, C.c_void_p, C.c_void_p,
                                          C.c_uint64, C.c_void_p]),
        "entro_cache_compact": (C.c_int, [kp, kt, kt, C.c_void_p, C.c_void_p, C.c_uint64, C.c_void_p]),
        "entro_cache_status": (C.c_int, [C.c_int32]),
        "entro_cache_shared": (C.c_int, [kp, kt, C.POINTER(CCacheGroups), C.c_void_p]),
        "entro_cache_attend_shared_workspace_bytes": (C.c_uint64, [kp, kt, C.POINTER(CCacheQuery), C.POINTER(CCacheGroups)]),
        "entro_cache_attend_shared": (C.c_int, [kp, kt, C.POINTER(CCacheQuery), C.POINTER(CCacheGroups), C.c_void_p, C.c_uint64, C.c_void_p]),
        "entro_rotary_turns": (C.c_int, [C.c_uint32, C.c_double, C.c_uint32, C.c_double, C.c_double, C.c_double, C.c_double, u64p]),
        "entro_rotate": (C.c_int, [C.POINTER(CRotary), C.POINTER(CRotaryRows), C.POINTER(CRotaryRows), C.c_void_p, C.c_uint32, C.c_uint32, C.c_int,
                                   C.c_void_p]),
        "entro_cache_append_rotated": (C.c_int, [kp, kt, C.POINTER(CCacheRows), C.POINTER(CRotary), C.POINTER(CRotaryRows), C.c_void_p]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(L, name)
        fn.restype = res
        fn.argtypes = args
    _lib = L
    return L


EXPORTED = ["entro_quantize", "entro_build_codebook", "entro_codebook_from_counts",
            "entro_codebook_from_lengths", "entro_codebook_from_counts_limited", "entro_build_codebook_limited", "entro_num_chunks", "entro_encode_bound", "entro_encode",
            "entro_check_offsets", "entro_sub_index", "entro_bits_saved", "entro_theoretical_speedup", "entro_status_string",
            "entro_decode", "entro_decode_dequant", "entro_gemv_workspace_bytes", "entro_decode_gemv", "entro_decode_gemv_static",
            "entro_workspace_bytes", "entro_plan_init", "entro_plan_staging_bytes", "entro_plan_init_staged", "entro_plan_run", "entro_decode_batch",
            "entro_decode_dequant_batch", "entro_decode_gemv_batch", "entro_last_device_error",
            "entro_range_device", "entro_qparams_from_range", "entro_scheme_for_range", "entro_quantize_device",
            "entro_encoded_bytes", "entro_encode_device", "entro_encode_device_status",
            "entro_cache_width", "entro_cache_codes_bytes", "entro_cache_append", "entro_cache_read",
            "entro_cache_attend_workspace_bytes", "entro_cache_attend", "entro_cache_pages_workspace_bytes", "entro_cache_regroup",
            "entro_cache_compact", "entro_cache_status", "entro_rotary_turns", "entro_rotate", "entro_cache_append_rotated",
            "entro_cache_shared", "entro_cache_attend_shared_workspace_bytes", "entro_cache_attend_shared"]


def _ptr(a: np.ndarray, t):
    return a.ctypes.data_as(C.POINTER(t))


def _check(status: int, what: str):
    if status != ENTRO_OK:
        raise EntroError(status, what)


# ----------------------------------------------------------------- host calls
def entro_status_string(status: int) -> str:
    return lib().entro_status_string(status).decode()


def entro_last_device_error() -> str:
    return lib().entro_last_device_error().decode()


def entro_quantize(w: np.ndarray, bits: int, scheme: int):
    """-> (q uint8[n], QParams)."""
    w = np.ascontiguousarray(w, dtype=np.float32).ravel()
    q = np.empty(w.size, np.uint8)
    qp = QParams()
    _check(lib().entro_quantize(_ptr(w, C.c_float), w.size, bits, scheme, _ptr(q, C.c_uint8), C.byref(qp)),
           "entro_quantize")
    return q, qp


def entro_build_codebook(q: np.ndarray, bits: int) -> Codebook:
    q = np.ascontiguousarray(q, dtype=np.uint8).ravel()
    cb = Codebook()
    _check(lib().entro_build_codebook(_ptr(q, C.c_uint8), q.size, bits, C.byref(cb)), "entro_build_codebook")
    return cb


def entro_codebook_from_counts(counts: np.ndarray, bits: int) -> Codebook:
    counts = np.ascontiguousarray(counts, dtype=np.uint64)
    assert counts.size == 1 << bits
    cb = Codebook()
    _check(lib().entro_codebook_from_counts(_ptr(counts, C.c_uint64), bits, C.byref(cb)),
           "entro_codebook_from_counts")
    return cb


def entro_codebook_from_counts_limited(counts: np.ndarray, bits: int, max_len: int) -> Codebook:
    counts = np.ascontiguousarray(counts, dtype=np.uint64)
    assert counts.size == 1 << bits
    cb = Codebook()
    _check(lib().entro_codebook_from_counts_limited(_ptr(counts, C.c_uint64), bits, int(max_len), C.byref(cb)),
           "entro_codebook_from_counts_limited")
    return cb


def entro_build_codebook_limited(q: np.ndarray, bits: int, max_len: int) -> Codebook:
    q = np.ascontiguousarray(q, dtype=np.uint8).ravel()
    cb = Codebook()
    _check(lib().entro_build_codebook_limited(_ptr(q, C.c_uint8), q.size, bits, int(max_len), C.byref(cb)),
           "entro_build_codebook_limited")
    return cb


def entro_codebook_from_lengths(lengths: np.ndarray, bits: int) -> Codebook:
    lengths = np.ascontiguousarray(lengths, dtype=np.uint8)
    assert lengths.size == 1 << bits
    cb = Codebook()
    _check(lib().entro_codebook_from_lengths(_ptr(lengths, C.c_uint8), bits, C.byref(cb)),
           "entro_codebook_from_lengths")
    return cb


def entro_num_chunks(n: int, chunk_symbols: int) -> int:
    return int(lib().entro_num_chunks(n, chunk_symbols))


def entro_encode_bound(n: int, cb: Codebook) -> int:
    return int(lib().entro_encode_bound(n, C.byref(cb)))


def entro_encode(q: np.ndarray, cb: Codebook, chunk_symbols: int):
    """-> (stream uint8[stream_bytes], offsets uint64[n_chunks + 1])."""
    q = np.ascontiguousarray(q, dtype=np.uint8).ravel()
    n = q.size
    # worst-case capacity; untouched pages of it are never committed
    stream = np.empty(max(entro_encode_bound(n, cb), 32), np.uint8)
    offsets = np.empty(entro_num_chunks(n, chunk_symbols) + 1, np.uint64)
    nbytes = C.c_uint64(0)
    _check(lib().entro_encode(_ptr(q, C.c_uint8), n, C.byref(cb), chunk_symbols, _ptr(stream, C.c_uint8),
                              stream.size, C.byref(nbytes), _ptr(offsets, C.c_uint64)), "entro_encode")
    return stream[: nbytes.value].copy(), offsets


def entro_sub_index(q: np.ndarray, cb: Codebook, chunk_symbols: int, sub_symbols: int) -> np.ndarray:
    """-> uint16[ceil(n / sub_symbols)]: stream bits of every piece of sub_symbols symbols."""
    q = np.ascontiguousarray(q, dtype=np.uint8).ravel()
    sub = np.empty(entro_num_chunks(q.size, sub_symbols), np.uint16)
    _check(lib().entro_sub_index(_ptr(q, C.c_uint8), q.size, C.byref(cb), chunk_symbols, sub_symbols,
                                 _ptr(sub, C.c_uint16)), "entro_sub_index")
    return sub


def entro_check_offsets(offsets: np.ndarray, n: int, chunk_symbols: int, stream_bytes: int, cb: Codebook) -> int:
    offsets = np.ascontiguousarray(offsets, dtype=np.uint64)
    return int(lib().entro_check_offsets(_ptr(offsets, C.c_uint64), n, chunk_symbols, stream_bytes, C.byref(cb)))


def entro_bits_saved(bits: int, mean_code_len: float) -> float:
    return float(lib().entro_bits_saved(bits, mean_code_len))


def entro_theoretical_speedup(bits: int, mean_code_len: float) -> float:
    return float(lib().entro_theoretical_speedup(bits, mean_code_len))


# ------------------------------------------------------------- tensor holders
@dataclass
class EncodedTensor:
    """Host-side result of quantize -> codebook -> encode for one tensor."""
    stream: np.ndarray
    offsets: np.ndarray
    n: int
    chunk_symbols: int
    cb: Codebook
    qp: QParams
    rows: int = 0
    cols: int = 0
    name: str = ""
    sub_symbols: int = 0                   # spacing of the entry points inside the segments (0: none)
    sub_bits: Optional[np.ndarray] = None  # uint16 piece lengths (entro_sub_index)

    @property
    def total_bits(self) -> int:
        return int(self.offsets[-1])

    @property
    def mean_code_len(self) -> float:
        return self.total_bits / self.n


def encode_tensor(w: np.ndarray, bits: int, scheme: int, chunk_symbols: int, rows: int = 0, cols: int = 0,
                  name: str = "", return_q: bool = False, max_len: int = 0, sub_symbols: int = 0):
    """entro_quantize -> entro_build_codebook (length-limited if max_len is given) -> entro_encode
    (-> entro_sub_index if sub_symbols is given)."""
    q, qp = entro_quantize(w, bits, scheme)
    cb = entro_build_codebook_limited(q, bits, max_len) if max_len else entro_build_codebook(q, bits)
    stream, offsets = entro_encode(q, cb, chunk_symbols)
    enc = EncodedTensor(stream, offsets, q.size, chunk_symbols, cb, qp, rows, cols, name)
    if sub_symbols:
        enc.sub_symbols, enc.sub_bits = sub_symbols, entro_sub_index(q, cb, chunk_symbols, sub_symbols)
    return (enc, q) if return_q else enc


class DeviceTensor:
    """Device copies of one encoded tensor plus its output buffer (torch owns the memory)."""

    def __init__(self, enc: EncodedTensor, device="cuda", stream=None, offsets=None):
        import torch
        self.enc = enc
        # stream / offsets given: the tensor was encoded on the device and enc holds no host copy of them
        self.stream = torch.from_numpy(enc.stream).to(device) if stream is None else stream
        self.offsets = torch.from_numpy(enc.offsets.view(np.int64)).to(device) if offsets is None else offsets
        self.sub_bits = torch.from_numpy(enc.sub_bits.view(np.int16)).to(device) if enc.sub_symbols else None
        self.x = None
        self.out = None

    def ctensor(self, out, x=None, entry_points: bool = True) -> CTensor:
        """The tensor as the device entry points take it; entry_points=False leaves the entry points inside
        the segments out (every lane then takes a whole segment)."""
        e = self.enc
        t = CTensor()
        t.stream = self.stream.data_ptr()
        t.stream_bytes = self.stream.numel()
        t.offsets = self.offsets.data_ptr()
        t.n = e.n
        t.chunk_symbols = e.chunk_symbols
        t.sub_symbols = e.sub_symbols if entry_points else 0
        t.sub_bits = self.sub_bits.data_ptr() if (self.sub_bits is not None and entry_points) else None
        t.rows, t.cols = e.rows, e.cols
        t.cb = C.pointer(e.cb)
        t.qp = e.qp
        t.x = x.data_ptr() if x is not None else None
        t.out = out.data_ptr()
        self.out, self.x = out, x
        return t


def to_device(enc: EncodedTensor, device="cuda") -> DeviceTensor:
    return DeviceTensor(enc, device)


def _stream_ptr(stream) -> Optional[int]:
    if stream is None:
        import torch
        return torch.cuda.current_stream(torch.cuda.current_device()).cuda_stream          # (by its number: without one torch takes longer to find it)
    return getattr(stream, "cuda_stream", stream)


def _tensor_array(ts: Sequence[CTensor]):
    arr = (CTensor * len(ts))(*ts)
    return arr


# --------------------------------------------------------------- device calls
def entro_decode(t: CTensor, out_type: int, stream=None):
    _check(lib().entro_decode(C.byref(t), out_type, _stream_ptr(stream)), "entro_decode")


def entro_decode_dequant(t: CTensor, out_type: int, stream=None):
    _check(lib().entro_decode_dequant(C.byref(t), out_type, _stream_ptr(stream)), "entro_decode_dequant")


def entro_gemv_workspace_bytes(t: CTensor) -> int:
    return int(lib().entro_gemv_workspace_bytes(C.byref(t)))


def entro_decode_gemv(t: CTensor, y_type: int, workspace=None, stream=None):
    ws_ptr = workspace.data_ptr() if workspace is not None else None
    ws_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    _check(lib().entro_decode_gemv(C.byref(t), y_type, ws_ptr, ws_bytes, _stream_ptr(stream)), "entro_decode_gemv")


def entro_decode_gemv_static(t: CTensor, y_type: int, stream=None):
    _check(lib().entro_decode_gemv_static(C.byref(t), y_type, _stream_ptr(stream)), "entro_decode_gemv_static")


def entro_workspace_bytes(ts: Sequence[CTensor], op: int) -> int:
    arr = _tensor_array(ts)
    return int(lib().entro_workspace_bytes(arr, len(ts), op))


def entro_plan_init(ts: Sequence[CTensor], op: int, out_type: int, workspace, stream=None) -> Plan:
    arr = _tensor_array(ts)
    plan = Plan()
    _check(lib().entro_plan_init(C.byref(plan), arr, len(ts), op, out_type, workspace.data_ptr(),
                                 workspace.numel() * workspace.element_size(), _stream_ptr(stream)),
           "entro_plan_init")
    return plan


def entro_plan_staging_bytes(ts: Sequence[CTensor], op: int) -> int:
    arr = _tensor_array(ts)
    return int(lib().entro_plan_staging_bytes(arr, len(ts), op))


def entro_plan_init_staged(ts: Sequence[CTensor], op: int, out_type: int, workspace, staging, stream=None) -> Plan:
    """Non-blocking entro_plan_init: `staging` is a pinned host tensor (torch, uint8) that the caller keeps alive
    until the copy enqueued here has completed."""
    arr = _tensor_array(ts)
    plan = Plan()
    _check(lib().entro_plan_init_staged(C.byref(plan), arr, len(ts), op, out_type, workspace.data_ptr(),
                                        workspace.numel() * workspace.element_size(), staging.data_ptr(),
                                        staging.numel() * staging.element_size(), _stream_ptr(stream)),
           "entro_plan_init_staged")
    return plan


def entro_plan_run(plan: Plan, stream=None):
    _check(lib().entro_plan_run(C.byref(plan), _stream_ptr(stream)), "entro_plan_run")


def _batch(fn_name: str, ts, out_type, workspace, stream):
    arr = _tensor_array(ts)
    fn = getattr(lib(), fn_name)
    _check(fn(arr, len(ts), out_type, workspace.data_ptr(), workspace.numel() * workspace.element_size(),
              _stream_ptr(stream)), fn_name)


# ------------------------------------------------------- device-side compression
def entro_range_device(w, range16, stream=None):
    """min / max / non-finite flag of w (torch float32 device tensor) into range16 (16 bytes of device memory)."""
    _check(lib().entro_range_device(w.data_ptr(), w.numel(), range16.data_ptr(), _stream_ptr(stream)), "entro_range_device")


def entro_qparams_from_range(mn: float, mx: float, nonfinite: int, bits: int, scheme: int) -> QParams:
    qp = QParams()
    _check(lib().entro_qparams_from_range(mn, mx, nonfinite, bits, scheme, C.byref(qp)), "entro_qparams_from_range")
    return qp


def entro_scheme_for_range(mn: float, mx: float) -> int:
    return int(lib().entro_scheme_for_range(mn, mx))


def entro_quantize_device(w, qp: QParams, q, counts, stream=None):
    """q (uint8 device tensor, w.numel() bytes) and counts (int64 device tensor of 256) from w and qp."""
    _check(lib().entro_quantize_device(w.data_ptr(), w.numel(), C.byref(qp), q.data_ptr(), counts.data_ptr(),
                                       _stream_ptr(stream)), "entro_quantize_device")


def entro_encoded_bytes(counts: np.ndarray, cb: Codebook) -> int:
    counts = np.ascontiguousarray(counts, dtype=np.uint64)
    return int(lib().entro_encoded_bytes(_ptr(counts, C.c_uint64), C.byref(cb)))


def entro_encode_device(q, cb: Codebook, chunk_symbols: int, stream_out, offsets, status, stream=None):
    """Encode q (uint8 device tensor) into stream_out / offsets (device tensors); status: 4 bytes of device memory."""
    _check(lib().entro_encode_device(q.data_ptr(), q.numel(), C.byref(cb), chunk_symbols, stream_out.data_ptr(),
                                     stream_out.numel() * stream_out.element_size(), offsets.data_ptr(), status.data_ptr(),
                                     _stream_ptr(stream)), "entro_encode_device")


def entro_encode_device_status(word: int) -> int:
    return int(lib().entro_encode_device_status(int(word) & 0xFFFFFFFF))


def compress_on_device(w, bits: int, scheme: Optional[int], chunk_symbols: int, rows: int = 0, cols: int = 0, name: str = "",
                       max_len: int = 0, return_q: bool = False):
    """Range -> (s, z) -> quantise + count -> codebook -> encode for a float32 tensor that lives on the GPU.

    The three passes over the weights are kernels; the two small steps between them run in the host
    library on the 16 and 2048 bytes copied back.  scheme None: entro_scheme_for_range picks the grid.
    Returns a DeviceTensor ready for the decode calls.
    """
    import torch
    w = w.reshape(-1)
    dev = w.device
    small = torch.empty(4 + 1, dtype=torch.int32, device=dev)          # range (16 bytes) and the encoder's status word
    counts = torch.empty(256, dtype=torch.int64, device=dev)
    entro_range_device(w, small)
    r = small[:4].cpu().numpy()
    mn, mx = r[:2].view(np.float32)
    if scheme is None:
        scheme = entro_scheme_for_range(float(mn), float(mx))
    qp = entro_qparams_from_range(float(mn), float(mx), int(r[2]), bits, scheme)
    q = torch.empty(w.numel(), dtype=torch.uint8, device=dev)
    entro_quantize_device(w, qp, q, counts)
    cnt = counts.cpu().numpy().view(np.uint64)
    cb = (entro_codebook_from_counts_limited(cnt[: 1 << bits], bits, max_len) if max_len
          else entro_codebook_from_counts(cnt[: 1 << bits], bits))
    nbytes = entro_encoded_bytes(cnt, cb)
    stream_out = torch.empty(nbytes, dtype=torch.uint8, device=dev)
    offsets = torch.empty(entro_num_chunks(w.numel(), chunk_symbols) + 1, dtype=torch.int64, device=dev)
    status = small[4:]
    entro_encode_device(q, cb, chunk_symbols, stream_out, offsets, status)
    _check(entro_encode_device_status(int(status.cpu()[0])), "entro_encode_device (status word)")
    enc = EncodedTensor(None, None, w.numel(), chunk_symbols, cb, qp, rows, cols, name)
    dt = DeviceTensor(enc, dev, stream=stream_out, offsets=offsets)
    return (dt, q) if return_q else dt


def entro_decode_batch(ts, out_type, workspace, stream=None):
    _batch("entro_decode_batch", ts, out_type, workspace, stream)


def entro_decode_dequant_batch(ts, out_type, workspace, stream=None):
    _batch("entro_decode_dequant_batch", ts, out_type, workspace, stream)


def entro_decode_gemv_batch(ts, y_type, workspace, stream=None):
    _batch("entro_decode_gemv_batch", ts, y_type, workspace, stream)


# ------------------------------------------------------------------- the token cache
def entro_cache_width(head_dim: int) -> int:
    return int(lib().entro_cache_width(head_dim))


def _need(ok: bool, what: str):
    """The C side sees addresses only: shapes and types of tensors are looked at here."""
    if not ok:
        raise ValueError(what)


def _rows_type(x, what: str) -> int:
    import torch
    _need(x.dtype in (torch.float32, torch.bfloat16), f"{what} is float32 or bfloat16")
    return ENTRO_F32 if x.dtype == torch.float32 else ENTRO_BF16


def _ints(x, n: Optional[int], what: str):
    import torch
    if x.dtype != torch.int32 or not x.is_contiguous() or (n is not None and x.numel() != n):
        raise ValueError(f"{what} is a contiguous int32 tensor" + ("" if n is None else f" of {n}"))
    return x.data_ptr()


def _device_of(*tensors):
    """The device of all tensors (None: left out), or None where they lie on several."""
    devices = {x.device for x in tensors if x is not None}
    return devices.pop() if len(devices) == 1 else None


class Cache:
    """A pool of pages (include/entro.h has the layouts): the tensors, and the descriptor that the calls take."""

    def __init__(self, k, v, k_scale, v_scale, page_tokens: int, head_dim: int):
        import torch
        width = entro_cache_width(head_dim)
        _need(width > 0, "head_dim is 1..256")
        _need(k.dim() == 5 and k.dtype == torch.uint8 and k.is_contiguous(), "k is uint8 [layers][pages][kv_heads][page_tokens][width]")
        layers, pages, heads = k.shape[:3]
        _need(tuple(k.shape[3:]) == (page_tokens, width), f"k's pages are [{page_tokens}][{width}]")
        _need(tuple(v.shape) == (layers, pages, heads, width, page_tokens) and v.dtype == torch.uint8 and v.is_contiguous(),
              "v is uint8 [layers][pages][kv_heads][width][page_tokens]")
        for x in (k_scale, v_scale):
            _need(tuple(x.shape) == (layers, pages, heads) and x.dtype == torch.float32 and x.is_contiguous(),
                  "scales are float32 [layers][pages][kv_heads]")
        self.k, self.v, self.k_scale, self.v_scale, self.device = k, v, k_scale, v_scale, _device_of(k, v, k_scale, v_scale)
        self.layers, self.pages, self.kv_heads, self.page_tokens, self.head_dim, self.width = layers, pages, heads, page_tokens, head_dim, width
        self.c = CCache(k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), layers, pages, page_tokens, heads, head_dim, 0)

    @classmethod
    def empty(cls, layers: int, pages: int, kv_heads: int, page_tokens: int, head_dim: int, device="cuda") -> "Cache":
        """A pool in newly allocated memory (which needs no clearing)."""
        import torch
        width = entro_cache_width(head_dim)
        _need(width > 0, "head_dim is 1..256")
        k = torch.empty(layers, pages, kv_heads, page_tokens, width, dtype=torch.uint8, device=device)
        v = torch.empty(layers, pages, kv_heads, width, page_tokens, dtype=torch.uint8, device=device)
        ks, vs = (torch.empty(layers, pages, kv_heads, dtype=torch.float32, device=device) for _ in "kv")
        return cls(k, v, ks, vs, page_tokens, head_dim)


class CacheTable:
    """Page numbers int32 [seqs][slots] and lengths int32 [seqs] of sequences."""

    def __init__(self, slots, lengths):
        _need(slots.dim() == 2, "slots is [seqs][slots]")
        self.slots, self.lengths, self.device = slots, lengths, _device_of(slots, lengths)
        self.c = CCacheTable(_ints(slots, None, "slots"), _ints(lengths, slots.shape[0], "lengths"), slots.shape[0], slots.shape[1])

    @classmethod
    def empty(cls, seqs: int, slots: int, device="cuda") -> "CacheTable":
        """A table of empty sequences."""
        import torch
        return cls(torch.full((seqs, slots), -1, dtype=torch.int32, device=device), torch.zeros(seqs, dtype=torch.int32, device=device))


def _row_strides(x, what: str):
    _need(x.dim() == 3 and (x.shape[2] == 1 or x.stride(2) == 1), f"{what} is [tokens][heads][head_dim], its dimensions side by side")
    return x.stride(0), x.stride(1)


def _own_places(x) -> bool:
    """Whether a tensor that a call writes is none that was expanded."""
    return not any(n > 1 and s == 0 for n, s in zip(x.shape, x.stride()))


class CacheRows:
    """Keys and values [tokens][kv_heads][head_dim] of the last tokens of sequences; start: int32 [seqs + 1]."""

    def __init__(self, k, v, start, max_new: int, layer: int = 0):
        _need(k.shape == v.shape and k.dtype == v.dtype, "k and v have one shape and type")
        self.k, self.v, self.start, self.device = k, v, start, _device_of(k, v, start)
        self.c = CCacheRows(k.data_ptr(), v.data_ptr(), *_row_strides(k, "k"), *_row_strides(v, "v"), _ints(start, None, "start"),
                            k.shape[0], max_new, _rows_type(k, "k"), layer)


class CacheQuery:
    """Queries and results [tokens][q_heads][head_dim] of the last tokens of sequences; start: int32 [seqs + 1]; lse: float32
    [tokens][q_heads] or None; scale None: 1 / sqrt(head_dim)."""

    def __init__(self, q, out, start, max_new: int, max_len: int, lse=None, scale: Optional[float] = None, window: int = 0,
                 sinks: int = 0, layer: int = 0):
        import torch
        _need(q.shape == out.shape and q.dtype == out.dtype, "q and out have one shape and type")
        _need(lse is None or (lse.dtype == torch.float32 and lse.is_contiguous() and tuple(lse.shape) == tuple(q.shape[:2])),
              "lse is float32 [tokens][q_heads]")
        _need(q.dim() == 3 and _own_places(out), "out's elements have places of their own")
        self.q, self.out, self.start, self.lse, self.device = q, out, start, lse, _device_of(q, out, start, lse)
        self.c = CCacheQuery(q.data_ptr(), out.data_ptr(), None if lse is None else lse.data_ptr(), *_row_strides(q, "q"),
                             *_row_strides(out, "out"), _ints(start, None, "start"), q.shape[0], max_new, max_len, q.shape[1],
                             _rows_type(q, "q"), layer, window, sinks, q.shape[2] ** -0.5 if scale is None else scale, 0)


def _on_gpu(cache: Cache, *given):
    """Every tensor whose address a call takes lies on the pool's GPU; given: descriptors, tensors, None for what is left out."""
    device = cache.device
    _need(device is not None and device.type == "cuda" and all(x is None or x.device == device for x in given), "all tensors of a call lie on one GPU")


def _same_heads(cache: Cache, table: CacheTable, x, start):
    _need(x.shape[2] == cache.head_dim, f"rows have {cache.head_dim} dimensions")
    _need(start.numel() == table.c.seqs + 1, f"start is [{table.c.seqs} + 1]")


def entro_cache_append(cache: Cache, table: CacheTable, rows: CacheRows, stream=None):
    _same_heads(cache, table, rows.k, rows.start)
    _need(rows.k.shape[1] == cache.kv_heads, f"rows have {cache.kv_heads} heads")
    _on_gpu(cache, table, rows)
    _check(lib().entro_cache_append(C.byref(cache.c), C.byref(table.c), C.byref(rows.c), _stream_ptr(stream)), "entro_cache_append")


def entro_cache_read(cache: Cache, table: CacheTable, rows: CacheRows, stream=None):
    _same_heads(cache, table, rows.k, rows.start)
    _need(_own_places(rows.k) and _own_places(rows.v), "the elements of k and v that are written have places of their own")
    _need(rows.k.shape[1] == cache.kv_heads, f"rows have {cache.kv_heads} heads")
    _on_gpu(cache, table, rows)
    _check(lib().entro_cache_read(C.byref(cache.c), C.byref(table.c), C.byref(rows.c), _stream_ptr(stream)), "entro_cache_read")


def entro_cache_attend_workspace_bytes(cache: Cache, table: CacheTable, query: CacheQuery) -> int:
    return int(lib().entro_cache_attend_workspace_bytes(C.byref(cache.c), C.byref(table.c), C.byref(query.c)))


def _workspace(ws):
    """(address, bytes) of a workspace tensor."""
    return (None, 0) if ws is None else (ws.data_ptr(), ws.numel() * ws.element_size())


def entro_cache_attend(cache: Cache, table: CacheTable, query: CacheQuery, workspace=None, stream=None):
    _same_heads(cache, table, query.q, query.start)
    _on_gpu(cache, table, query, workspace)
    _check(lib().entro_cache_attend(C.byref(cache.c), C.byref(table.c), C.byref(query.c), *_workspace(workspace), _stream_ptr(stream)),
           "entro_cache_attend")


def entro_cache_pages_workspace_bytes(cache: Cache, table: CacheTable, following: CacheTable) -> int:
    return int(lib().entro_cache_pages_workspace_bytes(C.byref(cache.c), C.byref(table.c), C.byref(following.c)))


def entro_cache_regroup(cache: Cache, table: CacheTable, following: CacheTable, status, workspace, parent=None, grow=None,
                        window: int = 0, sinks: int = 0, stream=None):
    """`following` receives the table of the next step; status: int32 device tensor of 4 (entro_cache_status reads its first word)."""
    n = following.c.seqs
    _on_gpu(cache, table, following, status, workspace, parent, grow)
    _check(lib().entro_cache_regroup(C.byref(cache.c), C.byref(table.c), None if parent is None else _ints(parent, n, "parent"),
                                     None if grow is None else _ints(grow, n, "grow"), window, sinks, C.byref(following.c),
                                     _ints(status, 4, "status"), *_workspace(workspace), _stream_ptr(stream)), "entro_cache_regroup")


def entro_cache_compact(cache: Cache, table: CacheTable, following: CacheTable, status, workspace, stream=None):
    _on_gpu(cache, table, following, status, workspace)
    _check(lib().entro_cache_compact(C.byref(cache.c), C.byref(table.c), C.byref(following.c), _ints(status, 4, "status"),
                                     *_workspace(workspace), _stream_ptr(stream)), "entro_cache_compact")


def entro_cache_status(word: int) -> int:
    return int(lib().entro_cache_status(int(word)))


# ------------------------------------------------------------------------ positions
def entro_rotary_turns(dims: int, base: float = 10000.0, context: int = ENTRO_CONTEXT_AS_TRAINED, factor: float = 1.0, trained: float = 1.0,
                       low: float = 1.0, high: float = 32.0) -> np.ndarray:
    """uint64[dims / 2]: what a position turns each pair by, in 2^-64 of a turn."""
    turns = np.zeros(dims // 2, np.uint64)
    _check(lib().entro_rotary_turns(dims, base, context, factor, trained, low, high, _ptr(turns, C.c_uint64)), "entro_rotary_turns")
    return turns


class Rotary:
    """How heads are normed and rotated. turns: int64 device tensor [dims / 2] (entro_rotary_turns' numbers), None for no dims; gains: float32
    [head_dim], or [heads][head_dim] for one set a head, or None."""

    def __init__(self, turns, dims: int, layout: int = ENTRO_ROTARY_HALVES, amplitude: float = 1.0, norm: int = ENTRO_NORM_NONE, eps: float = 1e-6,
                 q_gain=None, k_gain=None):
        import torch
        _need(dims == 0 if turns is None else (turns.dtype in (torch.int64, torch.uint64) and turns.is_contiguous() and 2 * turns.numel() == dims),
              "turns is a contiguous int64 tensor of dims / 2")
        for g in (q_gain, k_gain):
            _need(g is None or (g.dtype == torch.float32 and g.dim() in (1, 2) and g.is_contiguous()), "gains are float32 [head_dim] or [heads][head_dim]")
        self.turns, self.q_gain, self.k_gain = turns, q_gain, k_gain
        given = [x for x in (turns, q_gain, k_gain) if x is not None]
        self.device = _device_of(*given) if given else True              # True: there is nothing that lies anywhere
        at, stride = (lambda x: None if x is None else x.data_ptr()), (lambda g: 0 if g is None or g.dim() == 1 else g.stride(0))
        self.c = CRotary(at(turns), at(q_gain), at(k_gain), stride(q_gain), stride(k_gain), dims, layout, norm, eps, amplitude, 0)
        self.q_shape, self.k_shape = (None if g is None else tuple(g.shape) for g in (q_gain, k_gain))

    def fits(self, shape, heads: int, head_dim: int):
        _need(shape is None or shape == (head_dim,) or shape == (heads, head_dim), "gains are [head_dim] or [heads][head_dim]")


class RotaryRows:
    """Rows [tokens][heads][head_dim] that are read (x) and written (y: x itself, or a tensor apart from it; None: x)."""

    def __init__(self, x, y=None):
        y = x if y is None else y
        _need(x.shape == y.shape and x.dtype == y.dtype, "x and y have one shape and type")
        self.x, self.y, self.device, self.type, self.shape = x, y, _device_of(x, y), _rows_type(x, "x"), tuple(x.shape)
        self.c = CRotaryRows(x.data_ptr(), y.data_ptr(), *_row_strides(x, "x"), *_row_strides(y, "y"), x.shape[1], 0)
        _need(_own_places(y), "y's elements have places of their own")


def _run_on(device, call):
    """call() with `device` as the current one, which is where the library launches."""
    import torch
    if device.index in (None, torch.cuda.current_device()):
        return call()
    with torch.cuda.device(device):
        return call()


def entro_rotate(rotary: Rotary, q: Optional[RotaryRows], k: Optional[RotaryRows], positions, stream=None):
    """Norms and rotations of q and k (either may be None) at positions, int32 [tokens]."""
    side = q if k is None else k
    _need(side is not None, "q or k is given")
    tokens, heads, dim = side.shape
    if q is not None:
        rows, q_heads, q_dim = q.shape
        _need(rows == tokens and q_dim == dim and q.type == side.type, "q and k have one type, as many tokens and dimensions")
        rotary.fits(rotary.q_shape, q_heads, dim)
    if k is not None:
        rotary.fits(rotary.k_shape, heads, dim)
    at, device = _ints(positions, tokens, "positions"), positions.device
    _need(device.type == "cuda" and (q is None or q.device == device) and (k is None or k.device == device) and (rotary.device is True or rotary.device == device),
          "all tensors of a call lie on one GPU")
    _run_on(device, lambda: _check(lib().entro_rotate(C.byref(rotary.c), None if q is None else C.byref(q.c), None if k is None else C.byref(k.c), at, tokens, dim,
                                                      side.type, _stream_ptr(stream)), "entro_rotate"))


def entro_cache_append_rotated(cache: Cache, table: CacheTable, rows: CacheRows, rotary: Rotary, queries: Optional[RotaryRows] = None, stream=None):
    """entro_cache_append of keys that are normed and rotated on their way, and `queries` normed and rotated beside them."""
    _same_heads(cache, table, rows.k, rows.start)
    _need(rows.k.shape[1] == cache.kv_heads, f"rows have {cache.kv_heads} heads")
    rotary.fits(rotary.k_shape, cache.kv_heads, cache.head_dim)
    if queries is not None:
        tokens, heads, dim = queries.shape
        _need(queries.type == rows.c.type and tokens == rows.c.tokens and dim == cache.head_dim, "queries have the type, tokens and dimensions of the rows")
        rotary.fits(rotary.q_shape, heads, dim)
    _on_gpu(cache, table, rows, queries, None if rotary.device is True else rotary)
    q = None if queries is None else C.byref(queries.c)
    _run_on(cache.device, lambda: _check(lib().entro_cache_append_rotated(C.byref(cache.c), C.byref(table.c), C.byref(rows.c), C.byref(rotary.c), q,
                                                                          _stream_ptr(stream)), "entro_cache_append_rotated"))


# ---------------------------------------------------------------------------------------------------- groups behind a prefix
class CacheGroups:
    """Groups of sequences that begin with the same pages. first: int32 [groups + 1], ascending; shared: int32 [groups], tokens in shared pages
    (entro_cache_shared writes it); max_own: most tokens that a sequence has behind those (0: max_len less max_shared)."""

    def __init__(self, first, shared, max_seqs: int, max_shared: int, max_own: int = 0):
        n = first.numel() - 1
        _need(n > 0, "first is [groups + 1]")
        self.first, self.shared, self.device = first, shared, _device_of(first, shared)
        self.c = CCacheGroups(_ints(first, None, "first"), _ints(shared, n, "shared"), n, max_seqs, max_shared, max_own)


def entro_cache_shared(cache: Cache, table: CacheTable, groups: CacheGroups, stream=None):
    """Writes groups.shared from the table."""
    _on_gpu(cache, table, groups)
    _run_on(cache.device, lambda: _check(lib().entro_cache_shared(C.byref(cache.c), C.byref(table.c), C.byref(groups.c), _stream_ptr(stream)),
                                         "entro_cache_shared"))


def entro_cache_attend_shared_workspace_bytes(cache: Cache, table: CacheTable, query: CacheQuery, groups: CacheGroups) -> int:
    return int(lib().entro_cache_attend_shared_workspace_bytes(C.byref(cache.c), C.byref(table.c), C.byref(query.c), C.byref(groups.c)))


def entro_cache_attend_shared(cache: Cache, table: CacheTable, query: CacheQuery, groups: CacheGroups, workspace, stream=None):
    _same_heads(cache, table, query.q, query.start)
    _on_gpu(cache, table, query, groups, workspace)
    _run_on(cache.device, lambda: _check(lib().entro_cache_attend_shared(C.byref(cache.c), C.byref(table.c), C.byref(query.c), C.byref(groups.c),
                                                                         *_workspace(workspace), _stream_ptr(stream)), "entro_cache_attend_shared"))
