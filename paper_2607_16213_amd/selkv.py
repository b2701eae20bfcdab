"""Thin ctypes binding of libselkv.so (C ABI in include/selkv.h).

Argument marshalling only: every step runs in the HIP kernels of the
library.  Tensors are torch device tensors (PyTorch provides device memory
and the current stream); the functions check dtype, shape, device and
contiguity, then pass raw pointers.  Importing this module raises if the
built library is missing -- there is no fallback path.
"""
from __future__ import annotations

import ctypes
import os

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libselkv.so")

F32, BF16 = 0, 1
GATE_COSINE, GATE_DROP, GATE_MERGE_ALL = 0, 1, 2
ROUTE_BUCKET, ROUTE_FULL_COSINE, ROUTE_BUCKET_NEAREST, ROUTE_COATTN = 0, 1, 2, 3
SELECT_PER_HEAD, SELECT_UNION = 0, 1
ABI_VERSION = 6
CALL_SCORE, CALL_SELECT, CALL_MERGE, CALL_BIAS, CALL_DECODE, CALL_ROUTE, CALL_MERGE_BIAS = range(7)
STATUS = {0: "SELKV_OK", 1: "SELKV_EINVAL", 2: "SELKV_EDTYPE", 3: "SELKV_EUNSUPPORTED", 4: "SELKV_EALIGN",
          5: "SELKV_EWORKSPACE", 6: "SELKV_EHIP"}
GATE_MODES = {"cosine": GATE_COSINE, "drop": GATE_DROP, "merge_all": GATE_MERGE_ALL}
ROUTE_MODES = {"bucket": ROUTE_BUCKET, "full_cosine": ROUTE_FULL_COSINE, "bucket_nearest": ROUTE_BUCKET_NEAREST,
               "coattn": ROUTE_COATTN}
SELECT_MODES = {"per_head": SELECT_PER_HEAD, "union": SELECT_UNION}
CODE_I8, CODE_E4M3 = 0, 1
CODES8 = {"int8": CODE_I8, "e4m3": CODE_E4M3}


class SelkvError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {STATUS.get(status, status)}")


class Params(ctypes.Structure):
    _fields_ = [
        ("struct_size", ctypes.c_uint32),
        ("batch", ctypes.c_int32),
        ("n_heads_kv", ctypes.c_int32),
        ("group", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("seq_len", ctypes.c_int32),
        ("window", ctypes.c_int32),
        ("pool_kernel", ctypes.c_int32),
        ("recent", ctypes.c_int32),
        ("bucket", ctypes.c_int32),
        ("kv_dtype", ctypes.c_int32),
        ("gate_mode", ctypes.c_int32),
        ("route_mode", ctypes.c_int32),
        ("scale", ctypes.c_float),
        ("alpha", ctypes.c_float),
        ("gate_threshold", ctypes.c_float),
        ("gate_temperature", ctypes.c_float),
        ("budget_ratio", ctypes.c_double),
        ("select_mode", ctypes.c_int32),
        ("merge_keys", ctypes.c_int32),
    ]


class Cache8Struct(ctypes.Structure):
    """selkv_cache8."""
    _fields_ = [
        ("struct_size", ctypes.c_uint32),
        ("code", ctypes.c_int32),
        ("block", ctypes.c_int32),
        ("capacity", ctypes.c_int32),
        ("K", ctypes.c_void_p),
        ("V", ctypes.c_void_p),
        ("k_scale", ctypes.c_void_p),
        ("v_scale", ctypes.c_void_p),
        ("k_tail", ctypes.c_void_p),
        ("v_tail", ctypes.c_void_p),
    ]


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is not built; run paper_2607_16213_amd.build.build() first")
    lib = ctypes.CDLL(LIB_PATH)
    vp, sz, i32, fp, ip = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p
    P = ctypes.POINTER(Params)
    C8 = ctypes.POINTER(Cache8Struct)
    sigs = {
        "selkv_params_init": (None, [P]),
        "selkv_budget": (ctypes.c_int, [P, ctypes.POINTER(i32), ctypes.POINTER(i32), ctypes.POINTER(i32)]),
        "selkv_workspace_size": (ctypes.c_int, [P, i32, i32, ctypes.POINTER(sz)]),
        "selkv_score": (ctypes.c_int, [P, vp, vp, vp, fp, fp, fp, vp, sz, vp]),
        "selkv_select": (ctypes.c_int, [P, fp, ip, ip, vp, sz, vp]),
        "selkv_route_coattn": (ctypes.c_int, [P, vp, vp, ip, ip, ip, vp, sz, vp]),
        "selkv_merge": (ctypes.c_int, [P, vp, vp, fp, fp, ip, ip, vp, vp, ip, fp, vp, sz, vp]),
        "selkv_bias": (ctypes.c_int, [P, fp, ip, ip, ip, fp, fp, vp, sz, vp]),
        "selkv_merge_bias": (ctypes.c_int, [P, vp, vp, fp, fp, ip, ip, vp, vp, ip, fp, fp, vp, sz, vp]),
        "selkv_decode_attn": (ctypes.c_int, [P, vp, vp, vp, fp, i32, fp, vp, sz, vp]),
        "selkv_decode_attn_noalloc": (ctypes.c_int, [P, vp, vp, vp, fp, i32, fp, vp]),
        "selkv_rope_reposition": (ctypes.c_int, [P, ip, vp, ctypes.c_double, vp]),
        "selkv_decode_append": (ctypes.c_int, [P, vp, vp, vp, vp, vp, fp, i32, i32, fp, vp, sz, vp]),
        "selkv_cache8_init": (None, [C8]),
        "selkv_cache8_write": (ctypes.c_int, [P, C8, vp, vp, i32, i32, ip, ip, vp]),
        "selkv_cache8_read": (ctypes.c_int, [P, C8, vp, vp, i32, i32, i32, ip, vp]),
        "selkv_decode8_workspace_size": (ctypes.c_int, [P, C8, ctypes.POINTER(sz)]),
        "selkv_decode8_attn": (ctypes.c_int, [P, C8, vp, fp, i32, ip, fp, vp, sz, vp]),
        "selkv_decode8_append": (ctypes.c_int, [P, C8, vp, vp, vp, fp, i32, ip, fp, vp, sz, vp]),
        "selkv_status_string": (ctypes.c_char_p, [ctypes.c_int]),
        "selkv_abi_version": (ctypes.c_int32, []),
    }
    for name, (res, args) in sigs.items():
        f = getattr(lib, name)
        f.restype = res
        f.argtypes = args
    return lib


lib = _load()
if lib.selkv_abi_version() != ABI_VERSION:
    raise ImportError(f"{LIB_PATH} has ABI version {lib.selkv_abi_version()}, this binding expects {ABI_VERSION}")


def params(**kw) -> Params:
    """selkv_params with the paper's defaults, overridden by keyword."""
    p = Params()
    lib.selkv_params_init(ctypes.byref(p))
    for k, v in kw.items():
        if k == "gate_mode" and isinstance(v, str):
            v = GATE_MODES[v]
        if k == "route_mode" and isinstance(v, str):
            v = ROUTE_MODES[v]
        if k == "select_mode" and isinstance(v, str):
            v = SELECT_MODES[v]
        if k == "kv_dtype" and isinstance(v, (str, torch.dtype)):
            v = BF16 if v in ("bf16", torch.bfloat16) else F32
        if not hasattr(p, k):
            raise AttributeError(k)
        setattr(p, k, v)
    return p


def _check(status: int, where: str):
    if status != 0:
        raise SelkvError(status, where)


def budget(p: Params):
    m, mr, ms = ctypes.c_int32(), ctypes.c_int32(), ctypes.c_int32()
    _check(lib.selkv_budget(ctypes.byref(p), ctypes.byref(m), ctypes.byref(mr), ctypes.byref(ms)), "selkv_budget")
    return m.value, mr.value, ms.value


def workspace_bytes(p: Params, call: int, cache_len: int = 0) -> int:
    b = ctypes.c_size_t()
    _check(lib.selkv_workspace_size(ctypes.byref(p), call, cache_len, ctypes.byref(b)), "selkv_workspace_size")
    return b.value


def workspace(p: Params, call: int, device, cache_len: int = 0) -> torch.Tensor:
    """Scratch for `call` (zero-filled for tidiness; no call needs it initialised)."""
    nbytes = workspace_bytes(p, call, cache_len)
    return torch.zeros(max(nbytes, 1), dtype=torch.uint8, device=device)


def _ptr(t):
    return None if t is None else t.data_ptr()


# Handle of the current device's current stream (0 is the null stream), without
# building a torch Stream object per call.  A torch without GPU support has no
# such entry, and no call here gets as far as asking for a stream.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream):
    return _raw_stream(torch.cuda.current_device()) if stream is None else stream.cuda_stream


def _dev(t: torch.Tensor, shape, dtype, name):
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} has dtype {t.dtype}, expected {dtype}")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    return t


def _ok(t, shape, dtype):
    """Whether t passes _dev; the calls test this first and say what is wrong only when something is."""
    return t.is_cuda and t.dtype == dtype and t.shape == shape and t.is_contiguous()


def _sizes(p):
    """(m, m_r') of a valid problem, as selkv_budget gives them: m = floor(rho n) in IEEE double.  The library
    validates p itself, so a call on an invalid p fails there (or on a shape) and _refuse says why."""
    try:
        m = int(p.budget_ratio * p.seq_len)
    except (ValueError, OverflowError):   # rho is not a number
        budget(p)
        raise
    return m, min(p.recent, m)


def _refuse(p, status, where):
    budget(p)                             # an invalid problem is reported as such
    raise SelkvError(status, where)


def _nbytes(ws):
    """Size in bytes of a workspace tensor (any dtype), 0 for none."""
    if ws is None:
        return 0
    if not ws.is_cuda or not ws.is_contiguous():
        raise ValueError("workspace must be a contiguous device tensor")
    return ws.numel() * ws.element_size()


def _kvdt(p: Params):
    return torch.bfloat16 if p.kv_dtype == BF16 else torch.float32


_F32, _I32 = torch.float32, torch.int32


def score(p, K, V, Qwin, score_out, attn, vnorm, ws, stream=None):
    B, H, n, d = p.batch, p.n_heads_kv, p.seq_len, p.head_dim
    m, mr = _sizes(p)
    dt = _kvdt(p)
    kv, q, sc, per_key = (B, H, n, d), (B, H * p.group, p.window, d), (B, H, n - mr), (B, H, n)
    if not (_ok(K, kv, dt) and _ok(V, kv, dt) and _ok(Qwin, q, dt) and _ok(score_out, sc, _F32)
            and _ok(attn, per_key, _F32) and _ok(vnorm, per_key, _F32)):
        budget(p)
        _dev(K, kv, dt, "K"); _dev(V, kv, dt, "V"); _dev(Qwin, q, dt, "Qwin"); _dev(score_out, sc, _F32, "score")
        _dev(attn, per_key, _F32, "attn"); _dev(vnorm, per_key, _F32, "vnorm")
    st = lib.selkv_score(p, K.data_ptr(), V.data_ptr(), Qwin.data_ptr(), score_out.data_ptr(), attn.data_ptr(),
                         vnorm.data_ptr(), _ptr(ws), _nbytes(ws), _stream(stream))
    if st:
        _refuse(p, st, "selkv_score")


def select(p, score_in, kept, evicted, ws=None, stream=None):
    B, H, n = p.batch, p.n_heads_kv, p.seq_len
    m, mr = _sizes(p)
    sc, k, e = (B, H, n - mr), (B, H, m), (B, H, n - m)
    if not (_ok(score_in, sc, _F32) and _ok(kept, k, _I32) and _ok(evicted, e, _I32)):
        budget(p)
        _dev(score_in, sc, _F32, "score"); _dev(kept, k, _I32, "kept_idx"); _dev(evicted, e, _I32, "evicted_idx")
    st = lib.selkv_select(p, score_in.data_ptr(), kept.data_ptr(), evicted.data_ptr(), _ptr(ws), _nbytes(ws),
                          _stream(stream))
    if st:
        _refuse(p, st, "selkv_select")


def route_coattn(p, K, Qwin, kept, evicted, target, ws, stream=None):
    """Co-attention routing (route_mode COATTN): target slots for selkv_merge / selkv_bias."""
    B, H, n, d = p.batch, p.n_heads_kv, p.seq_len, p.head_dim
    m, mr = _sizes(p)
    dt = _kvdt(p)
    kv, q, k, e = (B, H, n, d), (B, H * p.group, p.window, d), (B, H, m), (B, H, n - m)
    if not (_ok(K, kv, dt) and _ok(Qwin, q, dt) and _ok(kept, k, _I32) and _ok(evicted, e, _I32)
            and _ok(target, e, _I32)):
        budget(p)
        _dev(K, kv, dt, "K"); _dev(Qwin, q, dt, "Qwin"); _dev(kept, k, _I32, "kept_idx")
        _dev(evicted, e, _I32, "evicted_idx"); _dev(target, e, _I32, "target")
    st = lib.selkv_route_coattn(p, K.data_ptr(), Qwin.data_ptr(), kept.data_ptr(), evicted.data_ptr(),
                                target.data_ptr(), _ptr(ws), _nbytes(ws), _stream(stream))
    if st:
        _refuse(p, st, "selkv_route_coattn")


def _check_merge(p, K, V, attn, vnorm, kept, evicted, K_out, V_out, target, gate, bias_out=None):
    B, H, n, d = p.batch, p.n_heads_kv, p.seq_len, p.head_dim
    m, mr = _sizes(p)
    dt = _kvdt(p)
    kv, per_key, k, e, out = (B, H, n, d), (B, H, n), (B, H, m), (B, H, n - m), (B, H, m, d)
    if not (_ok(K, kv, dt) and _ok(V, kv, dt) and _ok(attn, per_key, _F32) and _ok(vnorm, per_key, _F32)
            and _ok(kept, k, _I32) and _ok(evicted, e, _I32) and _ok(K_out, out, dt) and _ok(V_out, out, dt)
            and _ok(target, e, _I32) and _ok(gate, e, _F32) and (bias_out is None or _ok(bias_out, k, _F32))):
        budget(p)
        _dev(K, kv, dt, "K"); _dev(V, kv, dt, "V")
        _dev(attn, per_key, _F32, "attn"); _dev(vnorm, per_key, _F32, "vnorm")
        _dev(kept, k, _I32, "kept_idx"); _dev(evicted, e, _I32, "evicted_idx")
        _dev(K_out, out, dt, "K_out"); _dev(V_out, out, dt, "V_out")
        _dev(target, e, _I32, "target"); _dev(gate, e, _F32, "gate")
        if bias_out is not None:
            _dev(bias_out, k, _F32, "bias")


def merge(p, K, V, attn, vnorm, kept, evicted, K_out, V_out, target, gate, ws, stream=None):
    _check_merge(p, K, V, attn, vnorm, kept, evicted, K_out, V_out, target, gate)
    st = lib.selkv_merge(p, K.data_ptr(), V.data_ptr(), attn.data_ptr(), vnorm.data_ptr(), kept.data_ptr(),
                         evicted.data_ptr(), K_out.data_ptr(), V_out.data_ptr(), target.data_ptr(), gate.data_ptr(),
                         _ptr(ws), _nbytes(ws), _stream(stream))
    if st:
        _refuse(p, st, "selkv_merge")


def merge_bias(p, K, V, attn, vnorm, kept, evicted, K_out, V_out, target, gate, bias_out, ws, stream=None):
    """selkv_merge and selkv_bias in one pass (the bias from the merge's own sums)."""
    if bias_out is None:
        raise AttributeError("bias_out must be a device tensor")
    _check_merge(p, K, V, attn, vnorm, kept, evicted, K_out, V_out, target, gate, bias_out)
    st = lib.selkv_merge_bias(p, K.data_ptr(), V.data_ptr(), attn.data_ptr(), vnorm.data_ptr(), kept.data_ptr(),
                              evicted.data_ptr(), K_out.data_ptr(), V_out.data_ptr(), target.data_ptr(),
                              gate.data_ptr(), bias_out.data_ptr(), _ptr(ws), _nbytes(ws), _stream(stream))
    if st:
        _refuse(p, st, "selkv_merge_bias")


def bias(p, attn, kept, evicted, target, gate, bias_out, ws, stream=None):
    B, H, n = p.batch, p.n_heads_kv, p.seq_len
    m, mr = _sizes(p)
    per_key, k, e = (B, H, n), (B, H, m), (B, H, n - m)
    if not (_ok(attn, per_key, _F32) and _ok(kept, k, _I32) and _ok(evicted, e, _I32) and _ok(target, e, _I32)
            and _ok(gate, e, _F32) and _ok(bias_out, k, _F32)):
        budget(p)
        _dev(attn, per_key, _F32, "attn")
        _dev(kept, k, _I32, "kept_idx"); _dev(evicted, e, _I32, "evicted_idx")
        _dev(target, e, _I32, "target"); _dev(gate, e, _F32, "gate")
        _dev(bias_out, k, _F32, "bias")
    st = lib.selkv_bias(p, attn.data_ptr(), kept.data_ptr(), evicted.data_ptr(), target.data_ptr(), gate.data_ptr(),
                        bias_out.data_ptr(), _ptr(ws), _nbytes(ws), _stream(stream))
    if st:
        _refuse(p, st, "selkv_bias")


def rope_reposition(p, kept, K_out, rope_theta, stream=None):
    B, H, d = p.batch, p.n_heads_kv, p.head_dim
    m, mr, ms = budget(p)
    _dev(kept, (B, H, m), _I32, "kept_idx")
    _dev(K_out, (B, H, m, d), _kvdt(p), "K_out")
    _check(lib.selkv_rope_reposition(p, _ptr(kept), _ptr(K_out), float(rope_theta), _stream(stream)),
           "selkv_rope_reposition")


def _check_decode(p, q, K, V, bias_in, out):
    B, H, d = p.batch, p.n_heads_kv, p.head_dim
    L = K.shape[2]
    dt = _kvdt(p)
    qs, kv = (B, H * p.group, d), (B, H, L, d)
    if not (_ok(q, qs, dt) and _ok(K, kv, dt) and _ok(V, kv, dt) and _ok(out, qs, _F32)
            and (bias_in is None or _ok(bias_in, (B, H, L), _F32))):
        _dev(q, qs, dt, "q")
        _dev(K, kv, dt, "K"); _dev(V, kv, dt, "V")
        if bias_in is not None:
            _dev(bias_in, (B, H, L), _F32, "bias")
        _dev(out, qs, _F32, "out")
    return L


def decode_attn(p, q, K, V, bias_in, out, ws, stream=None):
    L = _check_decode(p, q, K, V, bias_in, out)
    st = lib.selkv_decode_attn(p, q.data_ptr(), K.data_ptr(), V.data_ptr(), _ptr(bias_in), L, out.data_ptr(),
                               _ptr(ws), _nbytes(ws), _stream(stream))
    if st:
        raise SelkvError(st, "selkv_decode_attn")


def decode_attn_noalloc(p, q, K, V, bias_in, out, stream=None):
    """selkv_decode_attn with the library's fixed per-GPU scratch instead of a
    workspace (nothing is allocated; calls overlapping on one GPU race)."""
    L = _check_decode(p, q, K, V, bias_in, out)
    st = lib.selkv_decode_attn_noalloc(p, q.data_ptr(), K.data_ptr(), V.data_ptr(), _ptr(bias_in), L, out.data_ptr(),
                                       _stream(stream))
    if st:
        raise SelkvError(st, "selkv_decode_attn_noalloc")


def decode_append(p, q, k_new, v_new, K, V, bias_io, cache_len, out, ws, stream=None):
    """Append (k_new, v_new) at entry cache_len (bias 0 there) and attend over
    cache_len + 1 entries; K, V [B, H, capacity, d] and bias [B, H, capacity]."""
    B, H, d = p.batch, p.n_heads_kv, p.head_dim
    cap = K.shape[2]
    dt = _kvdt(p)
    qs, new, kv = (B, H * p.group, d), (B, H, d), (B, H, cap, d)
    if not (_ok(q, qs, dt) and _ok(k_new, new, dt) and _ok(v_new, new, dt) and _ok(K, kv, dt) and _ok(V, kv, dt)
            and _ok(out, qs, _F32) and (bias_io is None or _ok(bias_io, (B, H, cap), _F32))):
        _dev(q, qs, dt, "q")
        _dev(k_new, new, dt, "k_new"); _dev(v_new, new, dt, "v_new")
        _dev(K, kv, dt, "K"); _dev(V, kv, dt, "V")
        if bias_io is not None:
            _dev(bias_io, (B, H, cap), _F32, "bias")
        _dev(out, qs, _F32, "out")
    st = lib.selkv_decode_append(p, q.data_ptr(), k_new.data_ptr(), v_new.data_ptr(), K.data_ptr(), V.data_ptr(),
                                 _ptr(bias_io), int(cache_len), cap, out.data_ptr(), _ptr(ws), _nbytes(ws),
                                 _stream(stream))
    if st:
        raise SelkvError(st, "selkv_decode_append")


class Cache8:
    """A KV cache held in 8 bits: its buffers and the selkv_cache8 that names them.

    `capacity` entries per KV head (rounded up to whole blocks) as `code`
    ("int8" or "e4m3") with one scale per `block` tokens; the rows of the last,
    incomplete block stay in the storage type.  `over` takes existing buffers.
    The lengths are the caller's: every call is given them."""

    def __init__(self, p: Params, capacity: int, device, code: str = "int8", block: int = 64):
        if block not in (16, 32, 64, 128):
            raise ValueError("block must be 16, 32, 64 or 128")
        B, H, d, dt = p.batch, p.n_heads_kv, p.head_dim, _kvdt(p)
        cap = -(-capacity // block) * block
        ct = torch.int8 if CODES8[code] == CODE_I8 else torch.float8_e4m3fn
        zeros = lambda shape, t: torch.zeros(shape, dtype=t, device=device)
        self._take(p, torch.zeros((B, H, cap, d), dtype=torch.int8, device=device).view(ct),
                   torch.zeros((B, H, cap // 16, d, 16), dtype=torch.int8, device=device).view(ct),
                   zeros((B, H, cap // block), _F32), zeros((B, H, cap // block), _F32), zeros((B, H, block, d), dt),
                   zeros((B, H, block, d), dt))

    @classmethod
    def over(cls, p: Params, K, V, k_scale, v_scale, k_tail, v_tail) -> "Cache8":
        """A cache in buffers that the caller owns (the layouts of include/selkv.h): the type of the codes is that of
        K, the block the rows of k_tail, the capacity K.shape[2]."""
        c = cls.__new__(cls)
        c._take(p, K, V, k_scale, v_scale, k_tail, v_tail)
        return c

    def _take(self, p, K, V, k_scale, v_scale, k_tail, v_tail):
        B, H, d, dt = p.batch, p.n_heads_kv, p.head_dim, _kvdt(p)
        if K.dtype not in (torch.int8, torch.float8_e4m3fn):
            raise ValueError(f"K has dtype {K.dtype}, expected torch.int8 or torch.float8_e4m3fn")
        if K.dim() != 4 or k_tail.dim() != 4:
            raise ValueError("K and k_tail must have four dimensions")
        cap, block = K.shape[2], k_tail.shape[2]
        if block not in (16, 32, 64, 128) or cap < block or cap % block:
            raise ValueError(f"a cache of {cap} entries and a tail of {block} rows: the tail must have 16, 32, 64 or 128 "
                             "rows and the capacity be whole blocks of them")
        _dev(K, (B, H, cap, d), K.dtype, "K"); _dev(V, (B, H, cap // 16, d, 16), K.dtype, "V")
        _dev(k_scale, (B, H, cap // block), _F32, "k_scale"); _dev(v_scale, (B, H, cap // block), _F32, "v_scale")
        _dev(k_tail, (B, H, block, d), dt, "k_tail"); _dev(v_tail, (B, H, block, d), dt, "v_tail")
        self.K, self.V, self.k_scale, self.v_scale, self.k_tail, self.v_tail = K, V, k_scale, v_scale, k_tail, v_tail
        self.device = K.device
        if any(t.device != K.device for t in (V, k_scale, v_scale, k_tail, v_tail)):
            raise ValueError("the buffers of a cache must be on one device")
        self.capacity, self.block = cap, block
        self._of = (B, H, d, p.kv_dtype)
        self.c = Cache8Struct()
        lib.selkv_cache8_init(self.c)
        self.c.code = CODE_I8 if K.dtype == torch.int8 else CODE_E4M3
        self.c.block, self.c.capacity = block, cap
        self.c.K, self.c.V, self.c.k_scale, self.c.v_scale = (t.data_ptr() for t in (K, V, k_scale, v_scale))
        self.c.k_tail, self.c.v_tail = k_tail.data_ptr(), v_tail.data_ptr()


def _check_cache8(p, cache, tensors, lens, counts, stream):
    """Checks the cache against p and the current device, and (tensor, shape, dtype, name) of every tensor; returns the
    stream's handle.  The launch goes to the current device, so all of them have to be there."""
    if cache._of != (p.batch, p.n_heads_kv, p.head_dim, p.kv_dtype):
        raise ValueError(f"the cache was made for (batch, n_heads_kv, head_dim, kv_dtype) = {cache._of}")
    dev = cache.device
    if dev.index != torch.cuda.current_device() or (stream is not None and stream.device != dev):
        raise ValueError(f"the cache is on {dev}: it must be the current device, and that of the stream")
    if lens is not None:
        tensors += ((lens, (p.batch,), _I32, "lens"),)
    if counts is not None:
        tensors += ((counts, (p.batch,), _I32, "counts"),)
    for t, shape, dtype, name in tensors:
        if not (t.device == dev and t.dtype == dtype and t.shape == shape and t.is_contiguous()):
            _dev(t, shape, dtype, name)
            raise ValueError(f"{name} is on {t.device}, the cache on {dev}")
    return _raw_stream(dev.index) if stream is None else stream.cuda_stream


def cache8_write(p, cache, K_new, V_new, cache_len, lens=None, counts=None, stream=None):
    """Append rows K_new, V_new [B, H, n_new, d] behind the cache_len (or lens[b]) entries of every sequence;
    counts [B] says how many of them each sequence gets (all n_new without it).  The biases of the new entries are the
    caller's to set (0 for plain rows)."""
    if K_new.dim() != 4:
        raise ValueError("K_new must have four dimensions")
    n_new = K_new.shape[2]
    new, dt = (p.batch, p.n_heads_kv, n_new, p.head_dim), _kvdt(p)
    on = _check_cache8(p, cache, ((K_new, new, dt, "K_new"), (V_new, new, dt, "V_new")), lens, counts, stream)
    if n_new == 0:
        return
    st = lib.selkv_cache8_write(p, cache.c, K_new.data_ptr(), V_new.data_ptr(), n_new, int(cache_len), _ptr(lens),
                                _ptr(counts), on)
    if st:
        raise SelkvError(st, "selkv_cache8_write")


def cache8_read(p, cache, K_out, V_out, cache_len, first=0, lens=None, stream=None):
    """Entries first .. first + K_out.shape[2] - 1 as rows in the storage type; rows of entries that a sequence does
    not hold are left as they were."""
    if K_out.dim() != 4:
        raise ValueError("K_out must have four dimensions")
    count = K_out.shape[2]
    out, dt = (p.batch, p.n_heads_kv, count, p.head_dim), _kvdt(p)
    on = _check_cache8(p, cache, ((K_out, out, dt, "K_out"), (V_out, out, dt, "V_out")), lens, None, stream)
    if count == 0:
        return
    st = lib.selkv_cache8_read(p, cache.c, K_out.data_ptr(), V_out.data_ptr(), int(first), count, int(cache_len),
                               _ptr(lens), on)
    if st:
        raise SelkvError(st, "selkv_cache8_read")


def decode8_workspace_bytes(p: Params, cache: Cache8) -> int:
    b = ctypes.c_size_t()
    _check(lib.selkv_decode8_workspace_size(p, cache.c, ctypes.byref(b)), "selkv_decode8_workspace_size")
    return b.value


def decode8_workspace(p: Params, cache: Cache8) -> torch.Tensor:
    """Scratch for decode8_attn and decode8_append at every length up to the capacity (needs no initialisation)."""
    return torch.zeros(max(decode8_workspace_bytes(p, cache), 1), dtype=torch.uint8, device=cache.device)


def decode8_attn(p, cache, q, bias_in, cache_len, out, ws, lens=None, stream=None):
    """Biased decode over the 8-bit cache; bias_in [B, H, capacity] or None."""
    B, H = p.batch, p.n_heads_kv
    qs = (B, H * p.group, p.head_dim)
    ts = ((q, qs, _kvdt(p), "q"), (out, qs, _F32, "out"))
    if ws is not None and ws.device != cache.device:
        raise ValueError(f"the workspace is on {ws.device}, the cache on {cache.device}")
    if bias_in is not None:
        ts += ((bias_in, (B, H, cache.capacity), _F32, "bias"),)
    on = _check_cache8(p, cache, ts, lens, None, stream)
    st = lib.selkv_decode8_attn(p, cache.c, q.data_ptr(), _ptr(bias_in), int(cache_len), _ptr(lens), out.data_ptr(),
                                _ptr(ws), _nbytes(ws), on)
    if st:
        raise SelkvError(st, "selkv_decode8_attn")


def decode8_append(p, cache, q, k_new, v_new, bias_io, cache_len, out, ws, lens=None, stream=None):
    """Append (k_new, v_new) [B, H, d] at entry cache_len (or lens[b]; bias 0 there) and attend over the entries with
    it.  lens is read only: advance it after the call."""
    B, H, d = p.batch, p.n_heads_kv, p.head_dim
    dt, qs = _kvdt(p), (B, H * p.group, d)
    ts = ((q, qs, dt, "q"), (k_new, (B, H, d), dt, "k_new"), (v_new, (B, H, d), dt, "v_new"), (out, qs, _F32, "out"))
    if ws is not None and ws.device != cache.device:
        raise ValueError(f"the workspace is on {ws.device}, the cache on {cache.device}")
    if bias_io is not None:
        ts += ((bias_io, (B, H, cache.capacity), _F32, "bias"),)
    on = _check_cache8(p, cache, ts, lens, None, stream)
    st = lib.selkv_decode8_append(p, cache.c, q.data_ptr(), k_new.data_ptr(), v_new.data_ptr(), _ptr(bias_io),
                                  int(cache_len), _ptr(lens), out.data_ptr(), _ptr(ws), _nbytes(ws), on)
    if st:
        raise SelkvError(st, "selkv_decode8_append")


class Compressor:
    """Owns the output and scratch tensors of one problem size and runs the
    compression calls (score, select, [route_coattn,] merge_bias, or merge then
    bias with fused=False) on the current stream.  Allocation happens once, in
    the constructor."""

    def __init__(self, p: Params, device):
        self.p = p
        B, H, n, d = p.batch, p.n_heads_kv, p.seq_len, p.head_dim
        self.m, self.mr, self.ms = budget(p)
        m, mr = self.m, self.mr
        dt = _kvdt(p)
        f32, i32 = torch.float32, torch.int32
        self.score = torch.empty((B, H, n - mr), dtype=f32, device=device)
        self.attn = torch.empty((B, H, n), dtype=f32, device=device)
        self.vnorm = torch.empty((B, H, n), dtype=f32, device=device)
        self.kept = torch.empty((B, H, m), dtype=i32, device=device)
        self.evicted = torch.empty((B, H, n - m), dtype=i32, device=device)
        self.K_out = torch.empty((B, H, m, d), dtype=dt, device=device)
        self.V_out = torch.empty((B, H, m, d), dtype=dt, device=device)
        self.target = torch.empty((B, H, n - m), dtype=i32, device=device)
        self.gate = torch.empty((B, H, n - m), dtype=f32, device=device)
        self.bias = torch.empty((B, H, m), dtype=f32, device=device)
        self.ws_score = workspace(p, CALL_SCORE, device)
        self.ws_select = workspace(p, CALL_SELECT, device)
        self.ws_merge = workspace(p, CALL_MERGE_BIAS, device)   # covers merge and bias alone too
        self.ws_route = workspace(p, CALL_ROUTE, device) if p.route_mode == ROUTE_COATTN else None

    def run(self, K, V, Qwin, stream=None, fused=True):
        p = self.p
        score(p, K, V, Qwin, self.score, self.attn, self.vnorm, self.ws_score, stream)
        select(p, self.score, self.kept, self.evicted, self.ws_select, stream)
        if p.route_mode == ROUTE_COATTN:
            route_coattn(p, K, Qwin, self.kept, self.evicted, self.target, self.ws_route, stream)
        if fused:
            merge_bias(p, K, V, self.attn, self.vnorm, self.kept, self.evicted, self.K_out, self.V_out, self.target,
                       self.gate, self.bias, self.ws_merge, stream)
        else:
            merge(p, K, V, self.attn, self.vnorm, self.kept, self.evicted, self.K_out, self.V_out, self.target,
                  self.gate, self.ws_merge, stream)
            bias(p, self.attn, self.kept, self.evicted, self.target, self.gate, self.bias, self.ws_merge, stream)
        return self

    def store8(self, cache: Cache8, bias_out=None, stream=None):
        """Write the compressed cache of the last run into an 8-bit cache from its start (it then holds m entries);
        bias_out [B, H, capacity], if given, gets the biases of those entries."""
        p = self.p
        if bias_out is not None:
            _dev(bias_out, (p.batch, p.n_heads_kv, cache.capacity), _F32, "bias")
        cache8_write(p, cache, self.K_out, self.V_out, 0, stream=stream)
        if bias_out is not None:
            with torch.cuda.stream(stream):   # the current stream where none is given
                bias_out[:, :, :self.m].copy_(self.bias)
        return cache

    def outputs(self):
        return dict(score=self.score, attn=self.attn, vnorm=self.vnorm, kept=self.kept, evicted=self.evicted,
                    K_out=self.K_out, V_out=self.V_out, target=self.target, gate=self.gate, bias=self.bias)


class Decoder:
    """Owns the split-K workspace for decode over caches of `cache_len` entries."""

    def __init__(self, p: Params, cache_len: int, device):
        self.p = p
        self.cache_len = cache_len
        self.ws = workspace(p, CALL_DECODE, device, cache_len)
        self.out = torch.empty((p.batch, p.n_heads_kv * p.group, p.head_dim), dtype=torch.float32, device=device)

    def run(self, q, K, V, bias_in=None, out=None, stream=None):
        o = self.out if out is None else out
        decode_attn(self.p, q, K, V, bias_in, o, self.ws, stream)
        return o


class Decoder8:
    """Owns the split-K workspace and the output of decode over one 8-bit cache."""

    def __init__(self, p: Params, cache: Cache8):
        self.p, self.cache = p, cache
        self.ws = decode8_workspace(p, cache)
        self.out = torch.empty((p.batch, p.n_heads_kv * p.group, p.head_dim), dtype=torch.float32,
                               device=cache.device)

    def run(self, q, cache_len, bias_in=None, lens=None, out=None, stream=None):
        """Attend over the entries that are there."""
        o = self.out if out is None else out
        decode8_attn(self.p, self.cache, q, bias_in, cache_len, o, self.ws, lens, stream)
        return o

    def step(self, q, k_new, v_new, cache_len, bias_io=None, lens=None, out=None, stream=None):
        """Append the new token and attend over the entries with it."""
        o = self.out if out is None else out
        decode8_append(self.p, self.cache, q, k_new, v_new, bias_io, cache_len, o, self.ws, lens, stream)
        return o
