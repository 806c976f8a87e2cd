"""ctypes binding of libalora (include/alora.h).  Argument marshalling only: torch supplies
device memory and streams, every step of the path runs in the library's HIP kernels.
There is no fallback: if the shared library is missing, importing this module raises."""
from __future__ import annotations

import ctypes as C
import os
from typing import Dict, List, Optional, Sequence

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
# ALORA_LIB: another build of the same library (kernel experiments); the default is the in-tree one
LIB_PATH = os.environ.get("ALORA_LIB") or os.path.join(_HERE, "libalora.so")

ALORA_OK, ALORA_EINVAL, ALORA_ESHAPE, ALORA_ECAPACITY, ALORA_EADAPTER, ALORA_EDTYPE, ALORA_EHIP = range(7)
ALORA_F32, ALORA_BF16 = 0, 1

EXPORTS = ["alora_create", "alora_destroy", "alora_last_error", "alora_status_string", "alora_set_option",
           "alora_profile_read", "alora_profile_reset", "alora_prefill", "alora_decode", "alora_decode_static", "alora_decode_steps", "alora_stack_prefill", "alora_stack_decode", "alora_lm_head",
           "alora_cache_copy", "alora_qcache_copy", "alora_qcache_store", "alora_qcache_load", "alora_qcache_attend", "alora_qcache_prefill",
           "alora_qcache_decode", "alora_qcache_stack_prefill", "alora_qcache_stack_decode"]
KERNELS = ["lm_head", "lm_argmax", "prep_rows", "qkv_gemm", "rope_append", "attn_prefill", "attn_decode", "attn_merge", "o_proj",
           "mlp_norm", "gate_up", "silu_mul", "down_proj", "row_move"]
Q_BLOCK = 32                 # channels of a row of 4 bits that share an exponent


class LayerDesc(C.Structure):
    _fields_ = [("d", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("rank", C.c_int32), ("n_adapters", C.c_int32), ("dtype", C.c_int32), ("intermediate", C.c_int32),
                ("W_qkv", C.c_void_p), ("A", C.c_void_p), ("B_q", C.c_void_p), ("B_k", C.c_void_p),
                ("B_v", C.c_void_p), ("scale", C.POINTER(C.c_float)), ("rms_gain", C.c_void_p),
                ("rms_eps", C.c_float), ("rope_theta", C.c_float),
                ("W_o", C.c_void_p), ("rms2_gain", C.c_void_p), ("W_gate", C.c_void_p), ("W_up", C.c_void_p),
                ("W_down", C.c_void_p),
                ("A_o", C.c_void_p), ("B_o", C.c_void_p), ("A_gu", C.c_void_p), ("B_gate", C.c_void_p),
                ("B_up", C.c_void_p), ("A_down", C.c_void_p), ("B_down", C.c_void_p)]


class KVCacheDesc(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("pool_tokens", C.c_int64),
                ("seq_offset", C.POINTER(C.c_int64)), ("seq_capacity", C.POINTER(C.c_int32)),
                ("seq_len", C.POINTER(C.c_int32)),
                ("prefix_offset", C.POINTER(C.c_int64)), ("prefix_len", C.POINTER(C.c_int32))]


class QCacheDesc(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p), ("pool_tokens", C.c_int64),
                ("seq_offset", C.POINTER(C.c_int64)), ("seq_capacity", C.POINTER(C.c_int32)), ("seq_len", C.POINTER(C.c_int32)),
                ("prefix_offset", C.POINTER(C.c_int64)), ("prefix_len", C.POINTER(C.c_int32))]


class RowRange(C.Structure):
    _fields_ = [("src", C.c_int64), ("dst", C.c_int64), ("n", C.c_int64)]


def load_library() -> C.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2504_12397_amd.build` "
                          "(there is no CPU or PyTorch fallback)")
    lib = C.CDLL(LIB_PATH)
    lib.alora_create.restype = C.c_int
    lib.alora_create.argtypes = [C.POINTER(C.c_void_p), C.c_int]
    lib.alora_destroy.restype = None
    lib.alora_destroy.argtypes = [C.c_void_p]
    lib.alora_last_error.restype = C.c_char_p
    lib.alora_last_error.argtypes = [C.c_void_p]
    lib.alora_status_string.restype = C.c_char_p
    lib.alora_status_string.argtypes = [C.c_int]
    lib.alora_set_option.restype = C.c_int
    lib.alora_set_option.argtypes = [C.c_void_p, C.c_char_p, C.c_int]
    lib.alora_profile_read.restype = C.c_int
    lib.alora_profile_read.argtypes = [C.c_void_p, C.c_char_p, C.POINTER(C.c_double), C.POINTER(C.c_int64)]
    lib.alora_profile_reset.restype = C.c_int
    lib.alora_profile_reset.argtypes = [C.c_void_p]
    i32p = C.POINTER(C.c_int32)
    lib.alora_prefill.restype = C.c_int
    lib.alora_prefill.argtypes = [C.c_void_p, C.POINTER(LayerDesc), C.POINTER(KVCacheDesc), C.c_void_p, i32p, i32p,
                                  i32p, C.c_int32, C.c_void_p, C.c_void_p]
    lib.alora_decode.restype = C.c_int
    lib.alora_decode.argtypes = [C.c_void_p, C.POINTER(LayerDesc), C.POINTER(KVCacheDesc), C.c_void_p, i32p, i32p,
                                 C.c_int32, C.c_void_p, C.c_void_p]
    lib.alora_decode_static.restype = C.c_int
    lib.alora_decode_static.argtypes = lib.alora_decode.argtypes
    lib.alora_decode_steps.restype = C.c_int
    lib.alora_decode_steps.argtypes = [C.c_void_p, C.POINTER(LayerDesc), C.POINTER(KVCacheDesc), C.c_void_p, i32p, i32p,
                                       C.c_int32, C.c_int32, C.c_void_p, C.c_void_p]
    lib.alora_lm_head.restype = C.c_int
    lib.alora_lm_head.argtypes = [C.c_void_p, C.c_int, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_float, C.c_void_p,
                                  C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p]
    lib.alora_stack_prefill.restype = C.c_int
    lib.alora_stack_prefill.argtypes = [C.c_void_p, C.POINTER(LayerDesc), C.c_int32, C.POINTER(KVCacheDesc),
                                        C.c_void_p, i32p, i32p, i32p, C.c_int32, C.c_void_p, C.c_void_p]
    lib.alora_stack_decode.restype = C.c_int
    lib.alora_stack_decode.argtypes = [C.c_void_p, C.POINTER(LayerDesc), C.c_int32, C.POINTER(KVCacheDesc), C.c_void_p,
                                       C.POINTER(C.c_int32), C.POINTER(C.c_int32), C.c_int32, C.c_void_p, C.c_void_p]
    # (arrays of descriptors, ranges and lengths go as addresses: the calls are short, and ctypes' typed pointers are not)
    i32, vp = C.c_int32, C.c_void_p
    kvp = qp = rp = vp
    lib.alora_cache_copy.argtypes = [vp, i32, i32, i32, kvp, kvp, i32, rp, i32, vp]
    lib.alora_qcache_copy.argtypes = [vp, i32, i32, qp, qp, i32, rp, i32, vp]
    lib.alora_qcache_store.argtypes = [vp, i32, i32, i32, qp, kvp, i32, rp, i32, vp]
    lib.alora_qcache_load.argtypes = [vp, i32, i32, i32, kvp, qp, i32, rp, i32, vp]
    lib.alora_qcache_attend.argtypes = [vp, i32, i32, i32, i32, qp, vp, vp, i32, vp, vp]
    lib.alora_qcache_prefill.argtypes = [vp, C.POINTER(LayerDesc), qp, vp, i32p, i32p, i32p, i32, vp, vp]
    lib.alora_qcache_decode.argtypes = [vp, C.POINTER(LayerDesc), qp, vp, i32p, i32p, i32, vp, vp]
    lib.alora_qcache_stack_prefill.argtypes = [vp, C.POINTER(LayerDesc), i32, qp, vp, i32p, i32p, i32p, i32, vp, vp]
    lib.alora_qcache_stack_decode.argtypes = [vp, C.POINTER(LayerDesc), i32, qp, vp, i32p, i32p, i32, vp, vp]
    for name in ("cache_copy", "qcache_copy", "qcache_store", "qcache_load", "qcache_attend", "qcache_prefill", "qcache_decode",
                 "qcache_stack_prefill", "qcache_stack_decode"):
        getattr(lib, "alora_" + name).restype = C.c_int
    return lib


_lib = load_library()


class AloraError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{_lib.alora_status_string(status).decode()}: {message}")
        self.status = status
        self.message = message


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    if t is None:
        return None
    assert t.is_contiguous(), "libalora takes contiguous row-major buffers"
    return t.data_ptr()


def _i32(a: Sequence[int]) -> np.ndarray:
    return np.ascontiguousarray(np.asarray(a, dtype=np.int32))


class Layer:
    """Holds the device tensors of one decoder layer and the C descriptor that points at them."""

    def __init__(self, tensors: Dict[str, Optional[torch.Tensor]], n_q_heads: int, n_kv_heads: int, head_dim: int,
                 rms_eps: float = 1e-5, rope_theta: float = 10000.0, intermediate: int = 0):
        self.t = tensors
        W = tensors["W_qkv"]
        dt = {torch.float32: ALORA_F32, torch.bfloat16: ALORA_BF16}[W.dtype]
        A = tensors.get("A")
        n_ad = int(A.shape[0]) if A is not None else 0
        rank = int(A.shape[2]) if A is not None else 0
        self.scale = np.ascontiguousarray(np.asarray(tensors.get("scale") or [], dtype=np.float32))
        g = tensors.get
        self.desc = LayerDesc(int(W.shape[1]), n_q_heads, n_kv_heads, head_dim, rank, n_ad, dt, int(intermediate),
                              _ptr(W), _ptr(A), _ptr(g("B_q")), _ptr(g("B_k")), _ptr(g("B_v")),
                              self.scale.ctypes.data_as(C.POINTER(C.c_float)) if n_ad else None,
                              _ptr(g("rms_gain")), float(rms_eps), float(rope_theta),
                              _ptr(g("W_o")), _ptr(g("rms2_gain")), _ptr(g("W_gate")), _ptr(g("W_up")),
                              _ptr(g("W_down")), _ptr(g("A_o")), _ptr(g("B_o")), _ptr(g("A_gu")), _ptr(g("B_gate")),
                              _ptr(g("B_up")), _ptr(g("A_down")), _ptr(g("B_down")))
        self.n_q = n_q_heads * head_dim
        self.d = int(W.shape[1])
        self.dtype = W.dtype
        self.device = W.device
        self.on = W.get_device()


def _table(x, dtype):
    return None if x is None else np.ascontiguousarray(np.asarray(x, dtype=dtype))


def _one_device(*arrays) -> int:
    on = arrays[0].get_device()
    if any([a.get_device() != on for a in arrays]):
        raise ValueError(f"arrays of one cache on {[str(a.device) for a in arrays]}")
    return on


class _Pool:
    """The host-side table of a pool of token rows: which rows belong to which sequence, and how many are valid."""

    def _regions(self, capacities: Sequence[int], guard_rows: int):
        caps = [int(c) for c in capacities]
        self.seq_capacity = _i32(caps)
        offs, o = [], guard_rows
        for c in caps:
            offs.append(o)
            o += c + guard_rows
        self.seq_offset = np.ascontiguousarray(np.asarray(offs, dtype=np.int64))
        self.pool_tokens = int(o)
        self.seq_len = np.zeros(len(caps), dtype=np.int32)
        self.prefix_offset = None        # set by share_prefix
        self.prefix_len = None

    def _wrap(self, pool_tokens, seq_offset, seq_capacity, seq_len, prefix_offset, prefix_len):
        self.pool_tokens = int(pool_tokens)
        self.seq_offset, self.seq_capacity = _table(seq_offset, np.int64), _table(seq_capacity, np.int32)
        self.seq_len = _table(seq_len, np.int32)
        self.prefix_offset, self.prefix_len = _table(prefix_offset, np.int64), _table(prefix_len, np.int32)
        tables = [self.seq_offset, self.seq_capacity, self.seq_len] + ([] if self.prefix_len is None else [self.prefix_offset, self.prefix_len])
        lengths = [len(t) for t in tables if t is not None]
        if lengths and (lengths != lengths[:1] * len(lengths) or (self.prefix_len is not None and self.prefix_offset is None)):
            raise ValueError(f"tables of {[None if t is None else len(t) for t in tables]} sequences")
        self._refresh()
        return self

    def _holds(self, n: int) -> bool:
        """Every table that a call of n sequences reads is there and as long as that: the library reads them on the host, as far as the call says."""
        need = (self.seq_offset, self.seq_capacity, self.seq_len) + (() if self.prefix_len is None else (self.prefix_offset, self.prefix_len))
        return all([t is not None and len(t) >= n for t in need])

    def _tables(self):
        def of(a, t):
            if a is None:
                return None
            if a.dtype != t or not a.flags.c_contiguous:
                raise ValueError(f"a table of {a.dtype} (contiguous: {a.flags.c_contiguous}) where the library reads {t.__name__} side by side")
            return a.ctypes.data_as(C.POINTER(t))
        shared = self.prefix_len is not None
        return (of(self.seq_offset, C.c_int64), of(self.seq_capacity, C.c_int32), of(self.seq_len, C.c_int32),
                of(self.prefix_offset, C.c_int64) if shared else None, of(self.prefix_len, C.c_int32))

    def share_prefix(self, b: int, pool_row: int, n: int):
        """Positions 0..n-1 of sequence b are read from pool rows pool_row.. (one copy that several sequences
        may name); its own rows then start at position n.  seq_len[b] becomes n if it was smaller."""
        if self.prefix_len is None:
            self.prefix_offset = np.zeros(len(self.seq_len), dtype=np.int64)
            self.prefix_len = np.zeros(len(self.seq_len), dtype=np.int32)
        self.prefix_offset[b] = int(pool_row)
        self.prefix_len[b] = int(n)
        self.seq_len[b] = max(int(self.seq_len[b]), int(n))
        self._refresh()


class KVCache(_Pool):
    """A flat pool of token rows [pool_tokens, n_kv_heads, head_dim] for keys and for values, plus the
    host-side table that says which rows belong to which sequence and how many are valid."""

    def __init__(self, capacities: Sequence[int], n_kv_heads: int, head_dim: int, dtype: torch.dtype, device,
                 fill: Optional[float] = None, guard_rows: int = 0):
        self._regions(capacities, guard_rows)
        shape = (self.pool_tokens, n_kv_heads, head_dim)
        if fill is None:
            self.k = torch.zeros(shape, dtype=dtype, device=device)
            self.v = torch.zeros(shape, dtype=dtype, device=device)
        else:
            self.k = torch.full(shape, fill, dtype=dtype, device=device)
            self.v = torch.full(shape, -fill, dtype=dtype, device=device)
        self._refresh()

    @classmethod
    def from_tensors(cls, k: torch.Tensor, v: torch.Tensor, seq_offset=None, seq_capacity=None, seq_len=None, prefix_offset=None,
                     prefix_len=None) -> "KVCache":
        """A cache over tensors that exist, k and v [pool_tokens, n_kv_heads, head_dim]; the table only where a call needs it."""
        assert k.shape == v.shape and k.dtype == v.dtype and k.dim() == 3, "k and v are of one shape and type"
        self = cls.__new__(cls)
        self.k, self.v = k, v
        return self._wrap(k.shape[0], seq_offset, seq_capacity, seq_len, prefix_offset, prefix_len)

    @property
    def head_dim(self) -> int:
        return int(self.k.shape[2])

    def _refresh(self):
        self.desc = KVCacheDesc(_ptr(self.k), _ptr(self.v), self.pool_tokens, *self._tables())
        self.kind = (int(self.k.shape[1]), self.head_dim, self.k.dtype, _one_device(self.k, self.v))

    def rows(self, b: int, lo: int, hi: int):
        o = int(self.seq_offset[b])
        return self.k[o + lo:o + hi], self.v[o + lo:o + hi]

    def load_prefix(self, b: int, K: torch.Tensor, V: torch.Tensor):
        """Copy already-computed cache rows (e.g. the base model's) for positions 0..n-1 of sequence b."""
        n = K.shape[0]
        o = int(self.seq_offset[b])
        self.k[o:o + n] = K.to(self.k.dtype).view(n, *self.k.shape[1:]).to(self.k.device)
        self.v[o:o + n] = V.to(self.v.dtype).view(n, *self.v.shape[1:]).to(self.v.device)
        self.seq_len[b] = n


class QCache(_Pool):
    """A pool of token rows in 4 bits: codes [pool_tokens, n_kv_heads, head_dim / 2] and exponents
    [pool_tokens, n_kv_heads, ceil(head_dim / 32)], uint8, for keys and for values, and the table of a KVCache."""

    def __init__(self, capacities: Sequence[int], n_kv_heads: int, head_dim: int, device, guard_rows: int = 0):
        self._regions(capacities, guard_rows)
        self.head_dim = int(head_dim)
        codes = (self.pool_tokens, n_kv_heads, head_dim // 2)
        scales = (self.pool_tokens, n_kv_heads, (head_dim + Q_BLOCK - 1) // Q_BLOCK)
        self.k, self.v = (torch.zeros(codes, dtype=torch.uint8, device=device) for _ in range(2))
        self.k_scale, self.v_scale = (torch.full(scales, 127, dtype=torch.uint8, device=device) for _ in range(2))
        self._refresh()

    @classmethod
    def from_tensors(cls, k: torch.Tensor, v: torch.Tensor, k_scale: torch.Tensor, v_scale: torch.Tensor, seq_offset=None,
                     seq_capacity=None, seq_len=None, prefix_offset=None, prefix_len=None) -> "QCache":
        """A cache over tensors that exist; the table only where a call needs it."""
        h = 2 * int(k.shape[-1])
        assert k.dim() == 3 and k.shape == v.shape and k_scale.shape == v_scale.shape == (*k.shape[:2], (h + Q_BLOCK - 1) // Q_BLOCK), "codes and exponents of one cache"
        assert all(t.dtype == torch.uint8 for t in (k, v, k_scale, v_scale)), "codes and exponents are uint8"
        self = cls.__new__(cls)
        self.head_dim = h
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        return self._wrap(k.shape[0], seq_offset, seq_capacity, seq_len, prefix_offset, prefix_len)

    def _refresh(self):
        self.desc = QCacheDesc(_ptr(self.k), _ptr(self.v), _ptr(self.k_scale), _ptr(self.v_scale), self.pool_tokens, *self._tables())
        self.kind = (int(self.k.shape[1]), self.head_dim, self.k.dtype, _one_device(self.k, self.v, self.k_scale, self.v_scale))


class Context:
    def __init__(self, device: int = 0):
        h = C.c_void_p()
        st = _lib.alora_create(C.byref(h), int(device))
        if st != ALORA_OK:
            raise AloraError(st, f"alora_create on device {device} failed")
        self._h = h
        self.device = int(device)

    def close(self):
        if getattr(self, "_h", None):
            _lib.alora_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, st: int):
        if st != ALORA_OK:
            raise AloraError(st, _lib.alora_last_error(self._h).decode())

    def set_option(self, key: str, value: int):
        self._check(_lib.alora_set_option(self._h, key.encode(), int(value)))

    def profile_reset(self):
        self._check(_lib.alora_profile_reset(self._h))

    def profile_read(self) -> Dict[str, Dict[str, float]]:
        """{kernel: {"ms": total, "launches": n}} for every kernel family that ran."""
        out = {}
        for name in KERNELS:
            ms, n = C.c_double(), C.c_int64()
            self._check(_lib.alora_profile_read(self._h, name.encode(), C.byref(ms), C.byref(n)))
            if n.value:
                out[name] = {"ms": ms.value, "launches": int(n.value)}
        return out


# (the current stream's handle without an object around it: 2.6 us less of a call that takes 9)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream_ptr(stream) -> Optional[int]:
    if stream is None:
        if _raw_stream is not None:
            return _raw_stream(torch.cuda.current_device())
        stream = torch.cuda.current_stream()
    return stream.cuda_stream


def alora_prefill(ctx: Context, layer: Layer, cache: KVCache, x_suffix: torch.Tensor, cu_seqlens: Sequence[int],
                  k_per_seq: Sequence[int], adapter_per_seq: Sequence[int], attn_out: Optional[torch.Tensor] = None,
                  stream=None) -> torch.Tensor:
    cu, kk, ad = _i32(cu_seqlens), _i32(k_per_seq), _i32(adapter_per_seq)
    B = len(kk)
    if attn_out is None:
        attn_out = torch.empty((x_suffix.shape[0], layer.n_q), dtype=layer.dtype, device=layer.device)
    p = C.POINTER(C.c_int32)
    st = _lib.alora_prefill(ctx._h, C.byref(layer.desc), C.byref(cache.desc), _ptr(x_suffix),
                            cu.ctypes.data_as(p), kk.ctypes.data_as(p), ad.ctypes.data_as(p), B,
                            _ptr(attn_out), _stream_ptr(stream))
    ctx._check(st)
    return attn_out


def alora_decode(ctx: Context, layer: Layer, cache: KVCache, x_tok: torch.Tensor, k_per_seq: Sequence[int],
                 adapter_per_seq: Sequence[int], attn_out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    kk, ad = _i32(k_per_seq), _i32(adapter_per_seq)
    B = len(kk)
    if attn_out is None:
        attn_out = torch.empty((B, layer.n_q), dtype=layer.dtype, device=layer.device)
    p = C.POINTER(C.c_int32)
    st = _lib.alora_decode(ctx._h, C.byref(layer.desc), C.byref(cache.desc), _ptr(x_tok), kk.ctypes.data_as(p),
                           ad.ctypes.data_as(p), B, _ptr(attn_out), _stream_ptr(stream))
    ctx._check(st)
    return attn_out


def alora_decode_static(ctx: Context, layer: Layer, cache: KVCache, x_tok: torch.Tensor, k_per_seq: Sequence[int],
                        adapter_per_seq: Sequence[int], attn_out: torch.Tensor, stream=None) -> torch.Tensor:
    """alora_decode through the entry point that allocates nothing; the caller brings the output buffer."""
    kk, ad = _i32(k_per_seq), _i32(adapter_per_seq)
    p = C.POINTER(C.c_int32)
    st = _lib.alora_decode_static(ctx._h, C.byref(layer.desc), C.byref(cache.desc), _ptr(x_tok), kk.ctypes.data_as(p),
                                  ad.ctypes.data_as(p), len(kk), _ptr(attn_out), _stream_ptr(stream))
    ctx._check(st)
    return attn_out


def alora_decode_steps(ctx: Context, layer: Layer, cache: KVCache, x_steps: torch.Tensor, k_per_seq: Sequence[int],
                       adapter_per_seq: Sequence[int], attn_out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """x_steps [n_steps, B, d] -> attn_out [n_steps, B, N_q]: n_steps decode steps staged once."""
    kk, ad = _i32(k_per_seq), _i32(adapter_per_seq)
    B = len(kk)
    n_steps = int(x_steps.shape[0])
    if attn_out is None:
        attn_out = torch.empty((n_steps, B, layer.n_q), dtype=layer.dtype, device=layer.device)
    p = C.POINTER(C.c_int32)
    st = _lib.alora_decode_steps(ctx._h, C.byref(layer.desc), C.byref(cache.desc), _ptr(x_steps), kk.ctypes.data_as(p),
                                 ad.ctypes.data_as(p), B, n_steps, _ptr(attn_out), _stream_ptr(stream))
    ctx._check(st)
    return attn_out


def alora_lm_head(ctx: Context, x_last: torch.Tensor, final_gain: Optional[torch.Tensor], rms_eps: float,
                  W_vocab: torch.Tensor, want_logits: bool = False, stream=None):
    """x_last [B, d], W_vocab [V, d] -> greedy token ids [B] (int32), and the fp32 logits [B, V] if asked for."""
    B, d = int(x_last.shape[0]), int(x_last.shape[1])
    V = int(W_vocab.shape[0])
    dt = ALORA_BF16 if x_last.dtype == torch.bfloat16 else ALORA_F32
    token = torch.empty((B,), dtype=torch.int32, device=x_last.device)
    logits = torch.empty((B, V), dtype=torch.float32, device=x_last.device) if want_logits else None
    st = _lib.alora_lm_head(ctx._h, dt, d, V, _ptr(x_last), _ptr(final_gain) if final_gain is not None else None,
                            float(rms_eps), _ptr(W_vocab), B, _ptr(logits) if logits is not None else None, _ptr(token),
                            _stream_ptr(stream))
    ctx._check(st)
    return (token, logits) if want_logits else token


def alora_stack_prefill(ctx: Context, layers: List[Layer], caches: List[KVCache], x: torch.Tensor,
                        cu_seqlens: Sequence[int], k_per_seq: Sequence[int], adapter_per_seq: Sequence[int],
                        out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    cu, kk, ad = _i32(cu_seqlens), _i32(k_per_seq), _i32(adapter_per_seq)
    B = len(kk)
    n = len(layers)
    descs = (LayerDesc * n)(*[l.desc for l in layers])
    cdescs = (KVCacheDesc * n)(*[c.desc for c in caches])
    if out is None:
        out = torch.empty_like(x)
    p = C.POINTER(C.c_int32)
    st = _lib.alora_stack_prefill(ctx._h, descs, n, cdescs, _ptr(x), cu.ctypes.data_as(p), kk.ctypes.data_as(p),
                                  ad.ctypes.data_as(p), B, _ptr(out), _stream_ptr(stream))
    ctx._check(st)
    # the library updated the seq_len array that caches[0] points at; mirror it to the others
    for c in caches[1:]:
        if c.seq_len is not caches[0].seq_len:
            c.seq_len[:] = caches[0].seq_len
    return out


def alora_stack_decode(ctx: Context, layers: List[Layer], caches: List[KVCache], x_tok: torch.Tensor,
                       k_per_seq: Sequence[int], adapter_per_seq: Sequence[int], out: Optional[torch.Tensor] = None,
                       stream=None) -> torch.Tensor:
    kk, ad = _i32(k_per_seq), _i32(adapter_per_seq)
    B = len(kk)
    n = len(layers)
    descs = (LayerDesc * n)(*[l.desc for l in layers])
    cdescs = (KVCacheDesc * n)(*[c.desc for c in caches])
    if out is None:
        out = torch.empty_like(x_tok)
    p = C.POINTER(C.c_int32)
    st = _lib.alora_stack_decode(ctx._h, descs, n, cdescs, _ptr(x_tok), kk.ctypes.data_as(p), ad.ctypes.data_as(p), B,
                                 _ptr(out), _stream_ptr(stream))
    ctx._check(st)
    for c in caches[1:]:
        if c.seq_len is not caches[0].seq_len:
            c.seq_len[:] = caches[0].seq_len
    return out


# ---- rows of a cache: copying them, and holding them in 4 bits ---------------------------------------------------
_DTYPES = {torch.float32: ALORA_F32, torch.bfloat16: ALORA_BF16}


def _address(a: np.ndarray) -> int:
    return a.__array_interface__["data"][0]


def _reach(ctx: Context, on: Sequence[int], tensors):
    """The GPU of the context reaches what is on these devices (-1: the host, where it reaches pinned memory); tensors() lists it all."""
    if ctx.device >= 0 and any([n != ctx.device for n in on]):
        for t in tensors():
            if t is not None and t.get_device() != ctx.device and not (t.get_device() < 0 and t.is_pinned()):
                raise ValueError(f"a tensor on {t.device}, which the context's GPU {ctx.device} does not reach")


def _arrays(c: _Pool):
    return [c.k, c.v] + ([c.k_scale, c.v_scale] if isinstance(c, QCache) else [])


def _move(name: str, ctx: Context, dst, src, ranges, stream, typed=None):
    """The four calls that move rows: caches are one, or a list of them, one per layer; typed: the side whose type the call is told."""
    d, s = ([dst] if isinstance(dst, _Pool) else dst), ([src] if isinstance(src, _Pool) else src)
    if len(d) != len(s) or len(d) == 0:
        raise ValueError(f"{len(d)} destination and {len(s)} source layers")
    to, of = d[0].kind, s[0].kind
    if any([c.kind != to for c in d]) or any([c.kind != of for c in s]) or to[:2] != of[:2] or (typed is None and to[2] != of[2]):
        raise ValueError(f"caches of different shapes or types: {[c.kind for c in d]} and {[c.kind for c in s]}")
    _reach(ctx, (to[3], of[3]), lambda: [t for c in (*d, *s) for t in _arrays(c)])
    r = np.ascontiguousarray(np.asarray(ranges, dtype=np.int64).reshape(-1, 3))
    kind = () if name == "alora_qcache_copy" else (_DTYPES[(to if typed == "dst" else of)[2]],)
    ctx._check(getattr(_lib, name)(ctx._h, *kind, *to[:2], b"".join([bytes(c.desc) for c in d]), b"".join([bytes(c.desc) for c in s]), len(d),
                                   _address(r), len(r), _stream_ptr(stream)))


def alora_cache_copy(ctx: Context, dst, src, ranges, stream=None):
    """ranges [n, 3] of (source row, destination row, rows): pool rows of `src` to pool rows of `dst` (a KVCache, or a list of them, one per
    layer), as if every row had been read before any is written; dst and src may be the same caches."""
    _move("alora_cache_copy", ctx, dst, src, ranges, stream)


def alora_qcache_copy(ctx: Context, dst, src, ranges, stream=None):
    """alora_cache_copy for QCaches."""
    _move("alora_qcache_copy", ctx, dst, src, ranges, stream)


def alora_qcache_store(ctx: Context, dst, src, ranges, stream=None):
    """Rows of KVCaches (src) into rows of 4 bits (dst): ranges as in alora_cache_copy."""
    _move("alora_qcache_store", ctx, dst, src, ranges, stream, typed="src")


def alora_qcache_load(ctx: Context, dst, src, ranges, stream=None):
    """Rows of 4 bits (src) into rows of KVCaches (dst), exactly."""
    _move("alora_qcache_load", ctx, dst, src, ranges, stream, typed="dst")


def alora_qcache_attend(ctx: Context, cache: QCache, q: torch.Tensor, cu_seqlens: Sequence[int], n_q_heads: int,
                        out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """q [T, n_q_heads * head_dim], rotated queries of the last rows of every sequence -> attention over the cache."""
    cu = _i32(cu_seqlens)
    h = cache.head_dim
    if out is None:
        out = torch.empty_like(q)
    if q.dtype not in _DTYPES or q.shape != (int(cu[-1]), n_q_heads * h) or out.shape != q.shape or out.dtype != q.dtype:
        raise ValueError(f"q {tuple(q.shape)} and out {tuple(out.shape)} have to be [{int(cu[-1])}, {n_q_heads * h}], fp32 or bf16")
    if not cache._holds(len(cu) - 1):
        raise ValueError(f"{len(cu) - 1} sequences are more than the tables of the cache hold")
    _reach(ctx, (cache.kind[3], q.get_device(), out.get_device()), lambda: [*_arrays(cache), q, out])
    ctx._check(_lib.alora_qcache_attend(ctx._h, _DTYPES[q.dtype], n_q_heads, int(cache.k.shape[1]), h, C.byref(cache.desc), _ptr(q), _address(cu),
                                        len(cu) - 1, _ptr(out), _stream_ptr(stream)))
    return out


def _q_call(name, ctx, layers, caches, x, cu, k_per_seq, adapter_per_seq, out, width, stream):
    """The four calls on QCaches that run layers; cu = None: one row per sequence; width: columns of the output."""
    kk, ad = _i32(k_per_seq), _i32(adapter_per_seq)
    stack = "stack" in name
    T = len(kk) if cu is None else int(cu[-1])
    if len(layers) != len(caches) or any([c.kind[:2] != (l.desc.n_kv_heads, l.desc.head_dim) for l, c in zip(layers, caches)]):
        raise ValueError(f"{len(layers)} layers and {len(caches)} caches, which have to be of the layers' heads")
    lengths = [0 if c.seq_len is None else len(c.seq_len) for c in caches]
    if any([n != lengths[0] for n in lengths]) or not caches[0]._holds(len(kk)) or len(ad) != len(kk) or (cu is not None and len(cu) != len(kk) + 1):
        raise ValueError(f"{len(kk)} sequences, {len(ad)} adapters and caches of {lengths}, which have to be as many in every layer and in every table")
    if x.shape != (T, layers[0].d) or x.dtype != layers[0].dtype or (out is not None and (out.shape != (T, width) or out.dtype != x.dtype)):
        raise ValueError(f"x {tuple(x.shape)} has to be [{T}, {layers[0].d}] and out [{T}, {width}], both of the layers' type")
    if out is None:
        out = torch.empty((x.shape[0], width), dtype=layers[0].dtype, device=layers[0].device)
    _reach(ctx, (x.get_device(), out.get_device(), *[c.kind[3] for c in caches], *[l.on for l in layers]),
           lambda: [x, out] + [t for c in caches for t in _arrays(c)] + [l.t["W_qkv"] for l in layers])
    p = C.POINTER(C.c_int32)
    descs = b"".join([bytes(c.desc) for c in caches])
    args = [ctx._h, (LayerDesc * len(layers))(*[l.desc for l in layers])] + ([len(layers)] if stack else []) + [descs, _ptr(x)]
    if cu is not None:
        cu = _i32(cu)
        args.append(cu.ctypes.data_as(p))
    st = getattr(_lib, name)(*args, kk.ctypes.data_as(p), ad.ctypes.data_as(p), len(kk), _ptr(out), _stream_ptr(stream))
    ctx._check(st)
    # the library updated the seq_len array that caches[0] points at; mirror it to the others
    for c in caches[1:]:
        if c.seq_len is not caches[0].seq_len:
            c.seq_len[:] = caches[0].seq_len
    return out


def alora_qcache_prefill(ctx: Context, layer: Layer, cache: QCache, x_suffix: torch.Tensor, cu_seqlens: Sequence[int], k_per_seq: Sequence[int],
                         adapter_per_seq: Sequence[int], attn_out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    return _q_call("alora_qcache_prefill", ctx, [layer], [cache], x_suffix, cu_seqlens, k_per_seq, adapter_per_seq, attn_out, layer.n_q, stream)


def alora_qcache_decode(ctx: Context, layer: Layer, cache: QCache, x_tok: torch.Tensor, k_per_seq: Sequence[int],
                        adapter_per_seq: Sequence[int], attn_out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    return _q_call("alora_qcache_decode", ctx, [layer], [cache], x_tok, None, k_per_seq, adapter_per_seq, attn_out, layer.n_q, stream)


def alora_qcache_stack_prefill(ctx: Context, layers: List[Layer], caches: List[QCache], x: torch.Tensor, cu_seqlens: Sequence[int],
                               k_per_seq: Sequence[int], adapter_per_seq: Sequence[int], out: Optional[torch.Tensor] = None,
                               stream=None) -> torch.Tensor:
    return _q_call("alora_qcache_stack_prefill", ctx, layers, caches, x, cu_seqlens, k_per_seq, adapter_per_seq, out, layers[0].d, stream)


def alora_qcache_stack_decode(ctx: Context, layers: List[Layer], caches: List[QCache], x_tok: torch.Tensor, k_per_seq: Sequence[int],
                              adapter_per_seq: Sequence[int], out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    return _q_call("alora_qcache_stack_decode", ctx, layers, caches, x_tok, None, k_per_seq, adapter_per_seq, out, layers[0].d, stream)
