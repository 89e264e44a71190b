"""Urgency-Aware Denoising on GB300: Python binding of the C ABI in include/uad.h.

Argument marshalling only: every step of the denoising loop runs in the library's CUDA
kernels. There is no CPU fallback; importing this package fails if libuad.so is missing.
"""
from __future__ import annotations

import ctypes as C
import os
import struct

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libuad.so")
if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is missing: build it with `python paper_2609_37772_gb300/build.py` "
                      "(or __graft_entry__.build()); there is no fallback path")
_lib = C.CDLL(LIB_PATH)

UAD_OK, UAD_EINVAL, UAD_ESTATE, UAD_ENOMEM, UAD_ECUDA, UAD_ETIMEDOUT, UAD_ENONFINITE = 0, -22, -1, -12, -5, -110, -33
KIND = {"adarms": 0, "dit": 1, "concat": 2}
DTYPE = {"f32": 0, "bf16": 1}
MAX_STEPS = 64

_I32, _P = C.c_int32, C.c_void_p


class uad_arch(C.Structure):
    _fields_ = [(n, _I32) for n in ("kind", "dtype", "n_layers", "width", "n_heads", "n_kv_heads",
                                    "head_dim", "mlp_dim", "action_dim", "chunk_len", "prefix_len",
                                    "prefix_width", "rope", "max_batch")]


class uad_schedule(C.Structure):
    _fields_ = [("budgets", C.POINTER(_I32)), ("batch", _I32), ("n_exec", _I32), ("tr", _I32),
                ("gac", _I32), ("chunk_relative", _I32), ("gac_mask", C.POINTER(C.c_uint8)),
                ("rot_dim", _I32)]


class uad_stats(C.Structure):
    _fields_ = [("evals", _I32), ("n_star", _I32), ("nonfinite", _I32), ("tr_extra_evals", _I32)]


class uad_kernel_stat(C.Structure):
    _fields_ = [("name", C.c_char * 32), ("launches", _I32), ("pad", _I32), ("total_ms", C.c_double),
                ("bytes", C.c_double), ("flops", C.c_double)]


class uad_kv_pages(C.Structure):
    _fields_ = [("k", _P), ("v", _P), ("page_stride", C.c_int64), ("slot_stride", C.c_int64), ("head_stride", C.c_int64)] + \
               [(n, _I32) for n in ("dtype", "n_pages", "page_size", "n_kv_heads", "head_dim", "pad")]


class uad_kv_seqs(C.Structure):
    _fields_ = [("table", _P), ("len", _P), ("start", _P), ("table_stride", C.c_int64)] + \
               [(n, _I32) for n in ("n_seqs", "table_width", "max_new", "max_len")]


class uad_rope(C.Structure):
    _fields_ = [("dim", _I32), ("pad", _I32), ("turn", C.c_uint64 * 128)]


class uad_kv_rows(C.Structure):
    _fields_ = [("q", _P), ("k", _P), ("v", _P), ("q_stride", C.c_int64), ("k_stride", C.c_int64), ("v_stride", C.c_int64),
                ("q_out", _P), ("q_out_stride", C.c_int64), ("dtype", _I32), ("n_heads", _I32), ("n_rows", _I32), ("pad", _I32)]


class uad_attn(C.Structure):
    _fields_ = [("q", _P), ("out", _P), ("lse", _P), ("key_mask", _P), ("q_stride", C.c_int64), ("out_stride", C.c_int64),
                ("mask_stride", C.c_int64), ("scale", C.c_float), ("n_heads", _I32), ("n_rows", _I32), ("causal", _I32),
                ("window", _I32), ("pad", _I32)]


def _fn(name, res, *args):
    f = getattr(_lib, name)
    f.restype = res
    f.argtypes = list(args)
    return f


uad_version = _fn("uad_version", C.c_char_p)
uad_last_error = _fn("uad_last_error", C.c_char_p, _P)
uad_init = _fn("uad_init", C.c_int, C.POINTER(uad_arch), _P, C.c_size_t, C.POINTER(_P))
uad_set_prefix_kv = _fn("uad_set_prefix_kv", C.c_int, _P, _I32, _P, _P, _I32, _I32)
uad_prepare_times = _fn("uad_prepare_times", C.c_int, _P, _I32)
uad_denoise = _fn("uad_denoise", C.c_int, _P, _P, C.POINTER(uad_schedule), _I32, _P)
uad_poll_released = _fn("uad_poll_released", C.c_int, _P, _I32, _I32, C.c_int64, _P, _P, _P)
uad_finish = _fn("uad_finish", C.c_int, _P, _P, _P, _P, C.POINTER(uad_stats), C.c_int64)
uad_step_times = _fn("uad_step_times", C.c_int, _P, _P, _I32)
uad_launches_per_chunk = _fn("uad_launches_per_chunk", C.c_int, _P, _I32, _I32)
uad_destroy = _fn("uad_destroy", None, _P)
uad_plan_step = _fn("uad_plan_step", C.c_int, _P, _I32, _I32, _I32, _P, _P, _P)
uad_profile_chunk = _fn("uad_profile_chunk", C.c_int, _P, _P, C.POINTER(uad_schedule), _P, _I32, C.c_int64)
uad_tile_weight = _fn("uad_tile_weight", C.c_int, _P, _I32, _I32, _P)
uad_linear = _fn("uad_linear", C.c_int, _P, _P, _P, _P, _I32, _I32, _I32, _P)
uad_linear_static_scratch = _fn("uad_linear_static_scratch", C.c_int, _P, _P, _P, _P, _I32, _I32, _I32, _P)
uad_linear_status = _fn("uad_linear_status", C.c_int)
uad_linear_check = _fn("uad_linear_check", C.c_int, _P, _P, _P, _P, _I32, _I32, _I32, _P)
uad_set_wait_limit = _fn("uad_set_wait_limit", C.c_int, _P, C.c_int64, _I32)
uad_so3_check = _fn("uad_so3_check", C.c_int, _P, _I32, _P, _P)
uad_rope_init = _fn("uad_rope_init", C.c_int, C.c_double, _I32, C.POINTER(uad_rope))
_PAGES, _SEQS = C.POINTER(uad_kv_pages), C.POINTER(uad_kv_seqs)
uad_kv_append = _fn("uad_kv_append", C.c_int, _PAGES, _SEQS, C.POINTER(uad_kv_rows), C.POINTER(uad_rope), _P, _P)
uad_paged_attention_workspace = _fn("uad_paged_attention_workspace", C.c_int64, _PAGES, _SEQS, C.POINTER(uad_attn))
uad_paged_attention = _fn("uad_paged_attention", C.c_int, _PAGES, _SEQS, C.POINTER(uad_attn), _P, C.c_size_t, _P, _P)
uad_set_prefix_paged = _fn("uad_set_prefix_paged", C.c_int, _P, _I32, _PAGES, _I32, _P, _I32)
uad_linear_w4 = _fn("uad_linear_w4", C.c_int, _P, _P, _P, _P, _P, _P, _I32, _I32, _I32, _I32, _P)
uad_quantize_w4 = _fn("uad_quantize_w4", C.c_int, _P, _I32, _I32, _I32, _P, _P, _P)
# The same entries for the wrappers below, with structures as addresses or packed bytes: a decoding step makes several such
# calls a layer, whose time on the host is longer than the kernels'.
_append, _attention, _w4 = _lib["uad_kv_append"], _lib["uad_paged_attention"], _lib["uad_linear_w4"]
_append.restype = _attention.restype = _w4.restype = C.c_int
_append.argtypes = [_P] * 6
_attention.argtypes = [_P] * 4 + [C.c_size_t, _P, _P]
_w4.argtypes = uad_linear_w4.argtypes
_pack_rows = struct.Struct("@3P3qPq4i").pack   # uad_kv_rows
_pack_attn = struct.Struct("@4P3qf5i").pack    # uad_attn
_LEAST = 2.0 ** -149   # fp32's least number above 0
UAD_ETOOBIG = -7
UAD_KV_BAD_PAGE, UAD_KV_BAD_SEQ = 1, 2
UAD_W4_MAX_ROWS = 64

EXPORTS = ["uad_version", "uad_last_error", "uad_init", "uad_set_prefix_kv", "uad_prepare_times",
           "uad_denoise", "uad_poll_released", "uad_finish", "uad_step_times",
           "uad_launches_per_chunk", "uad_destroy", "uad_plan_step", "uad_profile_chunk",
           "uad_tile_weight", "uad_linear", "uad_linear_static_scratch", "uad_set_wait_limit",
           "uad_linear_status", "uad_linear_check", "uad_so3_check", "uad_rope_init", "uad_kv_append",
           "uad_paged_attention_workspace", "uad_paged_attention", "uad_set_prefix_paged", "uad_linear_w4", "uad_quantize_w4"]


def tile_weight(w):
    """fp32 [K][N] -> uint16 bf16 bits in the tensor-core projection layout (host only)."""
    w = np.ascontiguousarray(w, dtype=np.float32)
    K, N = w.shape
    out = np.empty(N * K, dtype=np.uint16)
    rc = uad_tile_weight(_ptr(w), K, N, _ptr(out))
    if rc:
        raise UADError(rc, "tile_weight: needs N % 128 == 0 and K % 64 == 0")
    return out


class UADError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"UAD error {code}: {msg}")
        self.code = code


def _ptr(a):
    """Raw address of a numpy array or torch tensor (contiguous), or None."""
    if a is None:
        return None
    if isinstance(a, np.ndarray):
        if not a.flags["C_CONTIGUOUS"]:
            raise ValueError("buffer must be C-contiguous")
        return a.ctypes.data
    if not a.is_contiguous():
        raise ValueError("buffer must be contiguous")
    return a.data_ptr()


def _buf(a, n, dtype, what, host=False):
    """Address of a buffer the library reads or writes n elements of: a C-contiguous numpy
    array or torch tensor of `dtype` ("float32", "int32", "uint8"; "bfloat16" = np.uint16 bit
    patterns or a torch bfloat16 tensor) holding exactly n elements (host memory only when
    `host`). The C ABI takes bare pointers and cannot check sizes, so a short buffer is
    refused here, before the call, with ValueError; None passes through."""
    if a is None:
        return None
    if isinstance(a, np.ndarray):
        ok = a.dtype == (np.dtype(np.uint16) if dtype == "bfloat16" else np.dtype(dtype))
        size, on_host = a.size, True
    else:
        ok = str(a.dtype) == "torch." + dtype
        size, on_host = a.numel(), a.device.type == "cpu"
    if not ok:
        raise ValueError(f"{what}: expected {dtype} elements, got {a.dtype}")
    if size != n:
        raise ValueError(f"{what}: expected {n} elements, got {size}")
    if host and not on_host:
        raise ValueError(f"{what}: must be host memory")
    return _ptr(a)


def _stream_handle(stream):
    if stream is None:
        return None
    return getattr(stream, "cuda_stream", stream)


def arch_struct(arch, max_batch=1):
    """uad_arch from any object with the architecture's attribute names."""
    g = (lambda k: arch[k]) if isinstance(arch, dict) else (lambda k: getattr(arch, k))
    kind, dt = g("kind"), g("dtype")
    return uad_arch(kind=KIND.get(kind, kind), dtype=DTYPE.get(dt, dt), n_layers=g("n_layers"),
                    width=g("width"), n_heads=g("n_heads"), n_kv_heads=g("n_kv_heads"),
                    head_dim=g("head_dim"), mlp_dim=g("mlp_dim"), action_dim=g("action_dim"),
                    chunk_len=g("chunk_len"), prefix_len=g("prefix_len"),
                    prefix_width=g("prefix_width"), rope=int(bool(g("rope"))), max_batch=max_batch)


def plan_step(budgets, k, tr=True):
    """Host-only plan of step k: (n_star, flags[H], tau_num[H], tau_den[H])."""
    b = np.ascontiguousarray(budgets, dtype=np.int32)
    H = b.size
    f, tn, td = (np.zeros(H, np.int32) for _ in range(3))
    ns = uad_plan_step(_ptr(b), H, k, int(tr), _ptr(f), _ptr(tn), _ptr(td))
    if ns < 0:
        raise UADError(ns, "invalid plan arguments")
    return ns, f, tn, td


_row_types = {}   # 0 or 1 by the type of a row tensor, once seen
_dtypes = {}   # torch's types by name, once a tensor has been seen: the binding itself does not import torch


def _tensor(t, what, dtype, shape, device=None, rows=False):
    """The address of a torch tensor that a kernel reads or writes: element type, shape (None: any size), contiguous
    (rows: its rows alone, which may be apart) and on `device` (the GPU of the tensors beside it)."""
    if not _dtypes:
        import torch
        _dtypes.update({n: getattr(torch, n) for n in ("float32", "bfloat16", "int32", "uint8")})
    if t.dtype is not _dtypes[dtype]:
        raise ValueError(f"{what}: expected {dtype} elements, got {t.dtype}")
    if t.shape != shape and (t.dim() != len(shape) or any(a is not None and a != b for a, b in zip(shape, t.shape))):
        raise ValueError(f"{what}: expected shape {list(shape)}, got {list(t.shape)}")
    if not t.is_contiguous() and not (rows and t.dim() == 2 and t.stride(1) == 1 and t.stride(0) >= t.shape[1]):
        raise ValueError(f"{what}: buffer must be contiguous" + (" along its rows" if rows else ""))
    if t.get_device() < 0 or (device is not None and t.get_device() != device):
        raise ValueError(f"{what}: must be on {'the GPU' if device is None else 'cuda:%d' % device}, is on {t.device}")
    return t.data_ptr()


def rope(theta, dim):
    """Rotation of a head's first `dim` dimensions by its token's position: pair (i, i + dim / 2) by the angle
    position * theta^(-2 i / dim). To be kept by the caller and given to PagedCache.append."""
    r = uad_rope()
    rc = uad_rope_init(theta, dim, C.byref(r))
    if rc:
        raise UADError(rc, "rope: dim must be a multiple of 16 up to 256, theta positive and finite")
    return r


class Sequences:
    """A batch of sequences in a paged cache, as GPU tensors that the kernels read when they run: table int32
    [n][pages of the longest], length int32 [n] (tokens in the cache, new ones included), start int32 [n + 1] (rows
    start[b] .. start[b + 1] - 1 of the token tensors are the newest tokens of sequence b; None: row b is). max_new: at
    least the largest number of new tokens of a sequence; max_len: about the longest length, from which attention splits
    its work (0: what the table holds)."""

    def __init__(self, table, length, start=None, max_len=0, max_new=1):
        n = length.shape[0] if length.dim() else -1
        self.n = n
        tp = _tensor(table, "table", "int32", (n, None), rows=True)
        self._gpu = table.get_device()
        lp = _tensor(length, "length", "int32", (n,), self._gpu)
        sp = None if start is None else _tensor(start, "start", "int32", (n + 1,), self._gpu)
        self.device = table.device
        self._keep = table, length, start
        self.seqs = uad_kv_seqs(table=tp, len=lp, start=sp, table_stride=table.stride(0) if n > 1 else max(1, table.shape[1]), n_seqs=n,
                                table_width=table.shape[1], max_new=max_new, max_len=max_len)
        self._at = C.addressof(self.seqs)


class PagedCache:
    """One layer's paged key-value cache on the GPU: k and v [n_pages][page_size][n_kv_heads][head_dim], float32 or
    bfloat16, the last dimension contiguous, the others in any order (a view of [pages][heads][slots][dim], or of keys and
    values in one tensor), both with the same strides. The tensors stay the caller's. Calls are asynchronous on `stream`
    (None: the legacy default stream); `status`: an int32 tensor of one element that device-side findings
    (UAD_KV_BAD_PAGE, UAD_KV_BAD_SEQ) are added to. On a stream of their own, the caller keeps the tensors until the work is done."""

    def __init__(self, k, v):
        if k.dim() != 4 or k.shape != v.shape or k.dtype != v.dtype or k.stride() != v.stride() or k.device != v.device:
            raise ValueError("pages: k and v must be [n_pages][page_size][n_kv_heads][head_dim] of one type, device and strides")
        name = str(k.dtype)[6:]
        if name not in ("float32", "bfloat16"):
            raise ValueError(f"pages: expected float32 or bfloat16 elements, got {k.dtype}")
        if k.stride(3) != 1 or min(k.stride()) < 1:
            raise ValueError("pages: the last dimension must be contiguous")
        if k.device.type != "cuda":
            raise ValueError(f"pages: must be on the GPU, is on {k.device}")
        self.k, self.v, self.device, self.dtype = k, v, k.device, k.dtype
        self._gpu = k.get_device()
        self.page_size, self.n_kv_heads, self.head_dim = k.shape[1], k.shape[2], k.shape[3]
        self.pages = uad_kv_pages(k=k.data_ptr(), v=v.data_ptr(), page_stride=k.stride(0), slot_stride=k.stride(1),
                                  head_stride=k.stride(2), dtype=DTYPE["f32" if name == "float32" else "bf16"],
                                  n_pages=k.shape[0], page_size=k.shape[1], n_kv_heads=k.shape[2], head_dim=k.shape[3])
        self._at = C.addressof(self.pages)

    def _rows(self, t, what, dtype, n, width):
        """Address and row stride of a [n][width] tensor of `dtype` whose rows may be apart."""
        if t.dtype is dtype and t.get_device() == self._gpu and t.shape == (n, width):
            ld, one = t.stride()
            if one == 1 and ld >= width:
                return t.data_ptr(), ld
            if n == 1 and (one == 1 or width == 1):   # the stride of a single row says nothing
                return t.data_ptr(), width
        _tensor(t, what, str(dtype)[6:], (n, width), self._gpu, True)
        return t.data_ptr(), width   # contiguous in spite of its strides: no rows

    def _status(self, status):
        return None if status is None else _tensor(status, "status", "int32", (1,), self._gpu)

    def _heads(self, t):
        if t.dim() != 2:
            raise ValueError(f"q: expected rows of heads, got shape {list(t.shape)}")
        heads, rest = divmod(t.shape[1], self.head_dim)
        if rest:
            raise ValueError(f"q: expected a multiple of {self.head_dim} columns, got {t.shape[1]}")
        return heads

    def _refused(self, rc, what):
        raise UADError(rc, f"{what}: the arguments break a rule of include/uad.h, or the pages are not on the current device"
                       if rc == UAD_EINVAL else what)

    def append(self, seqs, k=None, v=None, q=None, q_out=None, rope=None, status=None, stream=None):
        """Write the new tokens' keys and values [rows][n_kv_heads * head_dim] into their pages and their queries
        [rows][n_heads * head_dim] into q_out, keys and queries rotated by `rope` (None: not). float32 or bfloat16 rows,
        which may be parts of a fused projection; q_out in the cache's type (q itself only where that is the rows')."""
        g = self._gpu
        if seqs._gpu != g:
            raise ValueError(f"sequences: must be on {self.device}, are on {seqs.device}")
        kp = vp = qp = op = kl = vl = ql = ol = heads = 0
        if k is not None and v is not None:
            kind, shape = k.dtype, k.shape
        elif q is not None and k is v:
            kind, shape = q.dtype, q.shape
        else:
            raise ValueError("append: k goes with v, q with q_out, and one of the two is needed")
        if (q is None) != (q_out is None):
            raise ValueError("append: k goes with v, q with q_out, and one of the two is needed")
        n = shape[0] if len(shape) else 0
        code = _row_types.get(kind)
        if code is None:
            if str(kind) not in ("torch.float32", "torch.bfloat16"):
                raise ValueError(f"append: expected float32 or bfloat16 rows, got {kind}")
            code = _row_types[kind] = int(str(kind) == "torch.bfloat16")
        # the usual rows checked at once; where a check fails, _rows says which or finds them sound
        if k is not None:
            width = self.n_kv_heads * self.head_dim
            (kl, one), (vl, uno) = (k.stride(), v.stride()) if len(shape) == 2 == v.dim() else ((0, 0), (0, 0))
            if (v.dtype is kind and shape == (n, width) == v.shape and one == 1 == uno and kl >= width <= vl and
                    k.get_device() == g == v.get_device()):
                kp, vp = k.data_ptr(), v.data_ptr()
            else:
                kp, kl = self._rows(k, "k", kind, n, width)
                vp, vl = self._rows(v, "v", kind, n, width)
        if q is not None:
            wide = q.shape
            heads = wide[1] // self.head_dim if len(wide) == 2 else 0
            (ql, one), (ol, uno) = (q.stride(), q_out.stride()) if len(wide) == 2 == q_out.dim() else ((0, 0), (0, 0))
            if (q.dtype is kind and q_out.dtype is self.dtype and wide == (n, heads * self.head_dim) == q_out.shape and one == 1 == uno and
                    ql >= wide[1] <= ol and q.get_device() == g == q_out.get_device()):
                qp, op = q.data_ptr(), q_out.data_ptr()
            else:
                heads = self._heads(q)
                qp, ql = self._rows(q, "q", kind, n, wide[1])
                op, ol = self._rows(q_out, "q_out", self.dtype, n, wide[1])
        rc = _append(self._at, seqs._at, _pack_rows(qp, kp, vp, ql, kl, vl, op, ol, code, heads, n, 0),
                     None if rope is None else C.addressof(rope), self._status(status), _stream_handle(stream))
        if rc:
            self._refused(rc, "append")

    def attention_workspace(self, seqs, rows, n_heads, window=0):
        """Bytes of the workspace that attention of these sizes needs (0 is possible). Without a window: enough for every window."""
        n = uad_paged_attention_workspace(self.pages, seqs.seqs, uad_attn(n_heads=n_heads, n_rows=rows, window=window))
        if n < 0:
            self._refused(n, "attention_workspace")
        return n

    def attention(self, seqs, q, out, workspace=None, scale=None, causal=True, window=0, key_mask=None, lse=None, status=None,
                  stream=None):
        """out = softmax(scale q k) v of the new tokens' queries [rows][n_heads * head_dim] over their sequences' pages
        (scale None: 1 / sqrt(head_dim); 0: all keys alike). causal: a token sees the keys up to its own; window > 0: no more than so many; key_mask
        uint8 [sequences][tokens that the table holds]: only where it is not 0. Where a token sees nothing, out is 0 and lse
        (float32 [rows][n_heads]) -inf. workspace: a uint8 tensor of attention_workspace bytes, not shared by calls that may
        run at the same time."""
        g = self._gpu
        if seqs._gpu != g:
            raise ValueError(f"sequences: must be on {self.device}, are on {seqs.device}")
        lp = mp = ml = wn = 0
        wp = None
        # the usual rows checked at once; where a check fails, _rows says which or finds them sound
        wide = q.shape
        heads = wide[1] // self.head_dim if len(wide) == 2 else 0
        n = wide[0] if len(wide) else 0
        (ql, one), (ol, uno) = (q.stride(), out.stride()) if len(wide) == 2 == out.dim() else ((0, 0), (0, 0))
        if (q.dtype is self.dtype is out.dtype and wide == (n, heads * self.head_dim) == out.shape and one == 1 == uno and ql >= wide[1] <= ol and
                q.get_device() == g == out.get_device()):
            qp, op = q.data_ptr(), out.data_ptr()
        else:
            heads = self._heads(q)
            qp, ql = self._rows(q, "q", self.dtype, n, wide[1])
            op, ol = self._rows(out, "out", self.dtype, n, wide[1])
        if lse is not None:
            if lse.dtype is _dtypes.get("float32") and lse.shape == (n, heads) and lse.is_contiguous() and lse.get_device() == g:
                lp = lse.data_ptr()
            else:
                lp = _tensor(lse, "lse", "float32", (n, heads), g)
        if key_mask is not None:
            mp, ml = _tensor(key_mask, "key_mask", "uint8", (seqs.n, None), self._gpu, True), key_mask.stride(0)
            if key_mask.shape[1] < seqs.seqs.table_width * self.page_size:
                raise ValueError(f"key_mask: expected {seqs.seqs.table_width * self.page_size} columns, what the table holds")
        if workspace is not None:
            wn = workspace.numel()
            if workspace.dtype is _dtypes.get("uint8") and workspace.dim() == 1 and workspace.is_contiguous() and workspace.get_device() == g:
                wp = workspace.data_ptr()
            else:
                wp = _tensor(workspace, "workspace", "uint8", (None,), g)
        # uad_attn takes 0 for the default: a scale of 0, or one that fp32 does not hold, is the least that it does
        factor = 0.0 if scale is None else _LEAST if abs(scale) < _LEAST else scale
        rc = _attention(self._at, seqs._at, _pack_attn(qp, op, lp, mp, ql, ol, ml, factor, heads, n, 1 if causal else 0, window, 0),
                        wp, wn, self._status(status), _stream_handle(stream))
        if rc:
            self._refused(rc, "attention")


def quantize_w4(w, group=64, symmetric=False):
    """fp32 [K][N] -> (q uint8 [N][K / 2], scale [N][K / group] as uint16 bf16 bits, zero uint8 [N][K / group] or None) for
    linear_w4 (host only)."""
    w = np.ascontiguousarray(w, dtype=np.float32)
    K, N = w.shape
    g = K // group if group > 0 else 0
    q, scale = np.empty((N, K // 2), np.uint8), np.empty((N, g), np.uint16)
    zero = None if symmetric else np.empty((N, g), np.uint8)
    rc = uad_quantize_w4(_ptr(w), K, N, group, _ptr(q), _ptr(scale), _ptr(zero))
    if rc:
        raise UADError(rc, "quantize_w4: needs finite weights, group 32, 64 or 128 and K % group == 0")
    return q, scale, zero


def linear_w4(x, q, scale, out, zero=None, bias=None, stream=None):
    """out [M][N] = x [M][K] w^T + bias with w = (q - zero) * scale, 4 bits a weight (zero None: 8): x bfloat16, q uint8
    [N][K / 2] (the even k in the low bits), scale bfloat16 and zero uint8 [N][K / group], bias and out float32; group 32, 64 or
    128, M up to UAD_W4_MAX_ROWS. Asynchronous on `stream` (None: the legacy default stream)."""
    M, K = x.shape if x.dim() == 2 else (0, 0)
    N, groups = scale.shape if scale.dim() == 2 else (0, 0)
    d, half, byte, full = x.get_device(), _dtypes.get("bfloat16"), _dtypes.get("uint8"), _dtypes.get("float32")
    # all checks at once, which takes half of what one by one does; where one fails, they say which
    if not (x.dtype is half and scale.dtype is half and q.dtype is byte and out.dtype is full and q.shape == (N, K // 2) and out.shape == (M, N) and
            x.is_contiguous() and scale.is_contiguous() and q.is_contiguous() and out.is_contiguous() and
            d >= 0 and d == scale.get_device() == q.get_device() == out.get_device()):
        _tensor(x, "x", "bfloat16", (M, K))
        _tensor(q, "q", "uint8", (N, K // 2), d)
        _tensor(scale, "scale", "bfloat16", (N, groups), d)
        _tensor(out, "out", "float32", (M, N), d)
    zp = bp = None
    if zero is not None:
        if not (zero.dtype is byte and zero.shape == scale.shape and zero.is_contiguous() and zero.get_device() == d):
            _tensor(zero, "zero", "uint8", (N, groups), d)
        zp = zero.data_ptr()
    if bias is not None:
        if not (bias.dtype is full and bias.shape == (N,) and bias.is_contiguous() and bias.get_device() == d):
            _tensor(bias, "bias", "float32", (N,), d)
        bp = bias.data_ptr()
    if groups < 1 or K % groups:
        raise ValueError(f"scale: {groups} groups do not divide {K} columns")
    rc = _w4(x.data_ptr(), q.data_ptr(), scale.data_ptr(), zp, bp, out.data_ptr(), M, N, K, K // groups, _stream_handle(stream))
    if rc:
        raise UADError(rc, "linear_w4: group must be 32, 64 or 128, x and q 16-byte aligned and on the current device, at most "
                       f"{UAD_W4_MAX_ROWS} rows")


class Expert:
    """One library context: an action expert's weights, prefixes and denoising state."""

    def __init__(self, arch, weights, max_batch=1):
        self.arch = arch_struct(arch, max_batch)
        self.H, self.D = self.arch.chunk_len, self.arch.action_dim
        h = _P()
        w = weights if not isinstance(weights, np.ndarray) else np.ascontiguousarray(weights, np.float32)
        n = w.size if isinstance(w, np.ndarray) else w.numel()
        rc = uad_init(C.byref(self.arch), _buf(w, n, "float32", "weights"), n, C.byref(h))
        if rc != UAD_OK:
            raise UADError(rc, "uad_init failed (see stderr)")
        self.h = h
        self._keep = None
        self._B = 1

    def _check(self, rc, what):
        if rc < 0:
            raise UADError(rc, f"{what}: {uad_last_error(self.h).decode()}")
        return rc

    def set_prefix(self, robot, k, v=None, dtype="f32"):
        """Attention-prefix experts: k, v [L][P][Hkv][dh]; DiT: k = prefix tokens
        [P][prefix_width], v = None. dtype "f32" (float32) or "bf16" (bfloat16 tensors or
        np.uint16 bit patterns); host or device."""
        code = DTYPE.get(dtype, dtype)
        el = "bfloat16" if code == DTYPE["bf16"] else "float32"
        a = self.arch
        if a.kind == KIND["dit"]:
            n = a.prefix_len * a.prefix_width
        else:
            n = a.n_layers * a.prefix_len * a.n_kv_heads * a.head_dim
        if isinstance(k, np.ndarray):
            k = np.ascontiguousarray(k, np.float32 if el == "float32" else None)
        if isinstance(v, np.ndarray):
            v = np.ascontiguousarray(v, np.float32 if el == "float32" else None)
        return self._check(uad_set_prefix_kv(self.h, robot, _buf(k, n, el, "prefix k"),
                                             _buf(v, n, el, "prefix v"), a.prefix_len, code),
                           "set_prefix")

    def set_prefix_paged(self, robot, caches, table):
        """set_prefix from pages: the first arch.prefix_len tokens of a sequence. caches: a PagedCache for each layer; table: int32
        [pages], a tensor or array on the host or the GPU, one for all layers. Synchronous and behind the legacy default stream: what
        other streams write has to be finished first."""
        t = np.ascontiguousarray(table, np.int32) if isinstance(table, (list, tuple)) else table
        if len(t.shape) != 1:
            raise ValueError(f"table: expected the pages of one sequence, got shape {list(t.shape)}")
        layers = (uad_kv_pages * len(caches))(*[c.pages for c in caches])
        return self._check(uad_set_prefix_paged(self.h, robot, layers, len(caches), _buf(t, t.shape[0], "int32", "table"), t.shape[0]),
                           "set_prefix_paged")

    def prepare_times(self, max_budget):
        return self._check(uad_prepare_times(self.h, max_budget), "prepare_times")

    def _schedule(self, budgets, n_exec, tr, gac, chunk_relative, gac_mask, rot_dim=None):
        b = np.ascontiguousarray(budgets, dtype=np.int32).reshape(-1, self.H)
        m = None if gac_mask is None else np.ascontiguousarray(gac_mask, dtype=np.uint8)
        if m is not None and m.size != self.D:
            raise ValueError(f"gac_mask: expected {self.D} entries, got {m.size}")
        sc = uad_schedule(budgets=b.ctypes.data_as(C.POINTER(_I32)), batch=b.shape[0], n_exec=n_exec,
                          tr=int(tr), gac=int(gac), chunk_relative=int(chunk_relative),
                          gac_mask=None if m is None else m.ctypes.data_as(C.POINTER(C.c_uint8)),
                          rot_dim=-1 if rot_dim is None else int(rot_dim))
        return sc, (b, m)

    def denoise(self, noise, budgets, n_exec=0, tr=True, gac=True, chunk_relative=False,
                gac_mask=None, n_star=0, stream=None, rot_dim=None):
        """rot_dim: first of three rotation-vector dimensions corrected on SO(3) (None: none)."""
        sc, keep = self._schedule(budgets, n_exec, tr, gac, chunk_relative, gac_mask, rot_dim)
        if isinstance(noise, np.ndarray):
            noise = np.ascontiguousarray(noise, dtype=np.float32)
        B = keep[0].shape[0]
        p = _buf(noise, B * self.H * self.D, "float32", "noise")
        self._keep = noise
        self._B = B
        return self._check(uad_denoise(self.h, p, C.byref(sc), n_star, _stream_handle(stream)), "denoise")

    def profile(self, noise, budgets, n_exec=0, tr=True, gac=True, chunk_relative=False, gac_mask=None,
                timeout_us=120_000_000):
        """Per-kernel-class CUDA-event times of one eagerly launched chunk."""
        sc, keep = self._schedule(budgets, n_exec, tr, gac, chunk_relative, gac_mask)
        if isinstance(noise, np.ndarray):
            noise = np.ascontiguousarray(noise, dtype=np.float32)
        B = keep[0].shape[0]
        p = _buf(noise, B * self.H * self.D, "float32", "noise")
        self._B = B
        stats = (uad_kernel_stat * 64)()
        n = self._check(uad_profile_chunk(self.h, p, C.byref(sc), stats, 64, int(timeout_us)), "profile")
        return [dict(name=st.name.decode(), launches=st.launches, total_ms=st.total_ms, bytes=st.bytes,
                     flops=st.flops) for st in stats[:n]]

    def poll(self, robot, min_ready=1, timeout_us=0, out=None):
        out = np.zeros((self.H, self.D), np.float32) if out is None else out
        ready = np.zeros(self.H, np.int32)
        step = np.zeros(self.H, np.int32)
        p = _buf(out, self.H * self.D, "float32", "out", host=True)
        rc = uad_poll_released(self.h, robot, min_ready, int(timeout_us), p, _ptr(ready), _ptr(step))
        if rc < 0 and rc != UAD_ETIMEDOUT:
            self._check(rc, "poll")
        return rc, out, ready, step

    def finish(self, timeout_us=-1, final=None, ghost=None, gac_error=None, check=True):
        B = self._B
        final = np.zeros((B, self.H, self.D), np.float32) if final is None else final
        ghost = np.zeros((B, self.H, self.D), np.float32) if ghost is None else ghost
        gac_error = np.zeros((B, self.D), np.float32) if gac_error is None else gac_error
        st = uad_stats()
        n = B * self.H * self.D
        pf, pg = _buf(final, n, "float32", "final"), _buf(ghost, n, "float32", "ghost")
        pe = _buf(gac_error, B * self.D, "float32", "gac_error")
        rc = uad_finish(self.h, pf, pg, pe, C.byref(st), int(timeout_us))
        if check and rc < 0:
            self._check(rc, "finish")
        return dict(rc=rc, final=final, ghost=ghost, E=gac_error, evals=st.evals, n_star=st.n_star,
                    nonfinite=st.nonfinite, tr_extra_evals=st.tr_extra_evals)

    def step_times(self, n=MAX_STEPS):
        out = np.zeros(n, np.float64)
        k = self._check(uad_step_times(self.h, _ptr(out), n), "step_times")
        return out[:k]

    def set_wait_limit(self, wait_ns=2_000_000_000, unreachable=0):
        """Testing aid: bound of every wait in the persistent kernel, and extra arrivals its
        first completion count waits for (> 0: the wait runs out and the chunk reports an
        error)."""
        return self._check(uad_set_wait_limit(self.h, int(wait_ns), int(unreachable)), "set_wait_limit")

    def launches_per_chunk(self, batch, n_star):
        return self._check(uad_launches_per_chunk(self.h, batch, n_star), "launches")

    def close(self):
        if getattr(self, "h", None):
            uad_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
