"""ctypes binding of ``libdma_b200.so`` (declared in ``include/dma.h``): argument marshalling only.

Every function here has the name of the C entry point it calls. Tensors are torch CUDA tensors used as
device memory; the current torch stream is passed as the CUDA stream. There is no fallback: if the library is
not built, or a call returns an error status, a ``DmaError`` is raised.
"""
import ctypes
import os
import struct

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libdma_b200.so")
_lib = None

DMA_BF16, DMA_FP32 = 0, 1
DMA_FLAG_IGNORE_BITMAP, DMA_FLAG_SIMT, DMA_FLAG_COMPACT_KV, DMA_FLAG_FULL_DELTA, DMA_FLAG_TILE_PATH = 1, 2, 4, 8, 16
DMA_FLAG_BLOCK_SKIP, DMA_FLAG_DETERMINISTIC = 32, 64

ENTRY_POINTS = ("dma_query_workspace", "dma_bitmap_words", "dma_mask_build", "dma_attn_fwd", "dma_attn_bwd",
                "dma_read_status", "dma_launch_count", "dma_strerror", "dma_step_host_arena", "dma_step_host", "dma_mask_build_static", "dma_selftest_wait_timeout",
                "dma_mask_bwd_workspace", "dma_mask_bwd", "dma_delta_range", "dma_decode_workspace", "dma_decode",
                "dma_mask_build_varlen", "dma_decode_state_bytes", "dma_decode_state_init", "dma_decode_step",
                "dma_attn_fwd_chunk", "dma_kernel_timing", "dma_kernel_timing_read",
                "dma_cache4_bytes", "dma_page_plan", "dma_cache4_append", "dma_cache4_read", "dma_cache4_decode_workspace", "dma_cache4_decode")


class DmaError(RuntimeError):
    def __init__(self, status, what):
        self.status = status
        super().__init__(f"{what}: status {status} ({dma_strerror(status)})")


class dma_problem_t(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("Hq", ctypes.c_int32), ("Hkv", ctypes.c_int32), ("L", ctypes.c_int32),
                ("d", ctypes.c_int32), ("w", ctypes.c_int32), ("causal", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("tile_m", ctypes.c_int32), ("tile_n", ctypes.c_int32), ("flags", ctypes.c_int32),
                ("softmax_scale", ctypes.c_float),
                ("q_stride", ctypes.c_int64 * 3), ("k_stride", ctypes.c_int64 * 3),
                ("v_stride", ctypes.c_int64 * 3), ("o_stride", ctypes.c_int64 * 3)]


class dma_cache_t(ctypes.Structure):
    _fields_ = [("Hq", ctypes.c_int32), ("Hkv", ctypes.c_int32), ("d", ctypes.c_int32), ("w", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("page_size", ctypes.c_int32), ("num_pages", ctypes.c_int32),
                ("max_blocks", ctypes.c_int32), ("nseq", ctypes.c_int32), ("rows", ctypes.c_int32), ("flags", ctypes.c_int32),
                ("softmax_scale", ctypes.c_float), ("table_ld", ctypes.c_int64),
                ("q_stride", ctypes.c_int64 * 2), ("k_stride", ctypes.c_int64 * 2),
                ("v_stride", ctypes.c_int64 * 2), ("o_stride", ctypes.c_int64 * 2)]


_KV_STRIDES, _KV_AT = struct.Struct("4q"), dma_cache_t.k_stride.offset       # k_stride and v_stride at once: a tenth of the time of two ctypes arrays


def lib():
    """Loads the shared library; raises if it has not been built (``python -m paper_2508_02124_b200.build``)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise DmaError(-6, f"{LIB_PATH} is missing: build it with `python -m paper_2508_02124_b200.build`")
        L = ctypes.CDLL(LIB_PATH)
        L.dma_strerror.restype = ctypes.c_char_p
        L.dma_launch_count.restype = ctypes.c_longlong
        _lib = L
    return _lib


def dma_strerror(status):
    try:
        return lib().dma_strerror(int(status)).decode()
    except Exception:
        return "?"


def _dtype_code(dtype):
    if dtype in (torch.bfloat16, torch.float32):
        return DMA_BF16 if dtype == torch.bfloat16 else DMA_FP32
    if type(dtype) is int and dtype in (DMA_BF16, DMA_FP32):
        return dtype
    raise TypeError(f"element type {dtype!r}: torch.bfloat16, torch.float32, DMA_BF16 or DMA_FP32")


def problem(B, Hq, Hkv, L, d, w, dtype=torch.bfloat16, causal=1, tile_m=0, tile_n=0, flags=0, softmax_scale=0.0):
    p = dma_problem_t()
    p.B, p.Hq, p.Hkv, p.L, p.d, p.w, p.causal = B, Hq, Hkv, L, d, w, causal
    p.dtype = _dtype_code(dtype)
    p.tile_m, p.tile_n, p.flags, p.softmax_scale = tile_m, tile_n, flags, softmax_scale
    return p


def _ptr(t):
    return None if t is None else t.data_ptr()


def _elem(p, *tensors):
    """The library reads Q, K, V, ... as the problem's element type; a tensor of another type would be read out of bounds."""
    want = torch.bfloat16 if p.dtype == DMA_BF16 else torch.float32
    for t in tensors:
        if t is not None and t.dtype != want:
            raise TypeError(f"tensor of {t.dtype} passed for a problem whose element type is {want}")


# torch's own calls for the handle alone, where this release of it has them
_raw_stream, _raw_device = (getattr(torch._C, n, None) for n in ("_cuda_getCurrentRawStream", "_cuda_getDevice"))


def _stream():
    """The current stream of the current device, as torch.cuda.current_stream().cuda_stream says it. That call builds a Stream
    object, 5.7 us a time, which was 40 % of the host's share of a decoding token; asking for the handle alone is 0.3 us."""
    if _raw_stream is None or _raw_device is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_raw_device())


# Parameter types of the calls that take device pointers: P problem, v pointer, i int32, l int64, z size_t. ctypes then converts
# plain integers itself; an object per argument (ctypes.c_void_p and so on) is 0.3 us, ten of them per call. With _stream()'s part the
# host's share of a decoding token (dma_delta_range and dma_decode, three launches) goes from 27 to 18.5 us.
_SIGNATURES = {
    "dma_mask_build": "Pvvvvvvvzv", "dma_mask_build_varlen": "Pvvvvivvvvzv", "dma_mask_build_static": "Pvvvvvvv",
    "dma_mask_bwd": "Pvvvvvvvvvzv", "dma_attn_fwd": "Pvvvvvvvvvzv", "dma_attn_fwd_chunk": "Piivvvvvvvvzv",
    "dma_attn_bwd": "Pvvvvvvvvvvvvvvzv", "dma_delta_range": "Pvvvvliiv", "dma_decode": "Pvvvvlvvvvzv",
    "dma_decode_state_init": "Pvlvvzv", "dma_decode_step": "Pvvvvlvvvvzv", "dma_step_host": "Pivvvvvvvvvvvvvzv",
    "dma_page_plan": "vvvvvvvvvvvvv", "dma_cache4_append": "vvvvvvlvvvvv", "dma_cache4_read": "vvvvvvvvlv",
    "dma_cache4_decode": "vvvvvvvvvvvzv", "dma_read_status": "vv", "dma_selftest_wait_timeout": "vzv"}
_KINDS = {"P": ctypes.POINTER(dma_problem_t), "v": ctypes.c_void_p, "i": ctypes.c_int32, "l": ctypes.c_int64, "z": ctypes.c_size_t}
_typed = {}                  # name -> function object with typed parameters
_typed_lib = None            # a handle of its own: the function objects of lib() stay untyped


def _typed_fn(name):
    global _typed_lib
    f = _typed.get(name)
    if f is None:
        if _typed_lib is None:
            lib()                              # (raises where the library is missing)
            _typed_lib = ctypes.CDLL(LIB_PATH)
        f = _typed_lib[name]
        f.argtypes = [_KINDS[k] for k in _SIGNATURES[name]]
        _typed[name] = f
    return f


def _call(name, *args):
    """Calls an entry point; a status other than 0 is raised."""
    rc = _typed_fn(name)(*args)
    if rc != 0:
        raise DmaError(rc, name)


def _check(rc, what):
    if rc != 0:
        raise DmaError(rc, what)


def dma_query_workspace(p):
    m, f, b = ctypes.c_size_t(), ctypes.c_size_t(), ctypes.c_size_t()
    _check(lib().dma_query_workspace(ctypes.byref(p), ctypes.byref(m), ctypes.byref(f), ctypes.byref(b)), "dma_query_workspace")
    return m.value, f.value, b.value


def dma_bitmap_words(p):
    n = ctypes.c_size_t()
    _check(lib().dma_bitmap_words(ctypes.byref(p), ctypes.byref(n)), "dma_bitmap_words")
    return n.value


def _ws(nbytes, device):
    return torch.empty((nbytes + 255) // 256 * 256, dtype=torch.uint8, device=device)


def dma_mask_build(p, V, W_delta, A, bias=None, expiry=None, bitmap=None, ws=None):
    """Returns (bias [B,Hq,L] fp32, expiry [B,Hq,L] int32, bitmap [B,Hq,Tr,ceil(Tc/32)] int32-typed uint32 words)."""
    _elem(p, V)
    dev = V.device
    if bias is None:
        bias = torch.empty(p.B, p.Hq, p.L, dtype=torch.float32, device=dev)
    if expiry is None:
        expiry = torch.empty(p.B, p.Hq, p.L, dtype=torch.int32, device=dev)
    if bitmap is None:
        tm, tn = (p.tile_m or 128), (p.tile_n or 128)
        Tr, Tc = -(-p.L // tm), -(-p.L // tn)
        bitmap = torch.empty(p.B, p.Hq, Tr, (Tc + 31) // 32, dtype=torch.int32, device=dev)
    if ws is None:
        ws = _ws(dma_query_workspace(p)[0], dev)
    _call("dma_mask_build", p, _ptr(V), _ptr(W_delta), _ptr(A), _ptr(bias), _ptr(expiry), _ptr(bitmap), _ptr(ws), ws.numel(),
          _stream())
    return bias, expiry, bitmap


def dma_mask_build_varlen(p, V, W_delta, A, cu_seqlens, bias=None, expiry=None, bitmap=None, ws=None):
    """dma_mask_build for sequences packed along the sequence axis; cu_seqlens: int32 device tensor [nseq + 1]."""
    _elem(p, V)
    dev = V.device
    assert cu_seqlens.dtype == torch.int32 and cu_seqlens.is_cuda and cu_seqlens.is_contiguous()
    if bias is None:
        bias = torch.empty(p.B, p.Hq, p.L, dtype=torch.float32, device=dev)
    if expiry is None:
        expiry = torch.empty(p.B, p.Hq, p.L, dtype=torch.int32, device=dev)
    if bitmap is None:
        tm, tn = (p.tile_m or 128), (p.tile_n or 128)
        Tr, Tc = -(-p.L // tm), -(-p.L // tn)
        bitmap = torch.empty(p.B, p.Hq, Tr, (Tc + 31) // 32, dtype=torch.int32, device=dev)
    if ws is None:
        ws = _ws(dma_query_workspace(p)[0], dev)
    _call("dma_mask_build_varlen", p, _ptr(V), _ptr(W_delta), _ptr(A), _ptr(cu_seqlens), cu_seqlens.numel() - 1, _ptr(bias),
          _ptr(expiry), _ptr(bitmap), _ptr(ws), ws.numel(), _stream())
    return bias, expiry, bitmap


def dma_mask_bwd_workspace(p):
    n = ctypes.c_size_t()
    _check(lib().dma_mask_bwd_workspace(ctypes.byref(p), ctypes.byref(n)), "dma_mask_bwd_workspace")
    return n.value


def dma_mask_bwd(p, V, W_delta, A, bias, dM, dV, dW_delta=None, dA=None, ws=None):
    """Adds the mask path's contribution to dV in place; returns (dV, dW_delta fp32 shaped like W_delta, dA [Hq] fp32)."""
    _elem(p, V, dV)
    dev = V.device
    if dW_delta is None:
        dW_delta = torch.empty(p.Hq, p.Hkv * p.d if p.flags & DMA_FLAG_FULL_DELTA else p.d, dtype=torch.float32, device=dev)
    if dA is None:
        dA = torch.empty(p.Hq, dtype=torch.float32, device=dev)
    if ws is None:
        ws = _ws(dma_mask_bwd_workspace(p), dev)
    _call("dma_mask_bwd", p, _ptr(V), _ptr(W_delta), _ptr(A), _ptr(bias), _ptr(dM), _ptr(dV), _ptr(dW_delta), _ptr(dA),
          _ptr(ws), ws.numel(), _stream())
    return dV, dW_delta, dA


def dma_delta_range(p, V, W_delta, A, delta, j_begin, j_end):
    """delta[b,h,j] for the keys j in [j_begin, j_end) of the cache V, written into the delta cache [B,Hq,ld]."""
    _elem(p, V)
    _call("dma_delta_range", p, _ptr(V), _ptr(W_delta), _ptr(A), _ptr(delta), delta.stride(1), j_begin, j_end, _stream())
    return delta


def dma_decode_workspace(p):
    n = ctypes.c_size_t()
    _check(lib().dma_decode_workspace(ctypes.byref(p), ctypes.byref(n)), "dma_decode_workspace")
    return n.value


def dma_decode(p, q, K, V, delta, o=None, lse=None, sel_idx=None, want_idx=False, ws=None):
    """One decoding step over the cached keys; returns (o [B,Hq,d], lse [B,Hq], sel_idx or None)."""
    _elem(p, q, K, V, o)
    dev = q.device
    if o is None:
        o = torch.empty_like(q)
    if lse is None:
        lse = torch.empty(p.B, p.Hq, dtype=torch.float32, device=dev)
    if sel_idx is None and want_idx:
        sel_idx = torch.empty(p.B, p.Hq, min(p.w, p.L), dtype=torch.int32, device=dev)
    if ws is None:
        ws = _ws(dma_decode_workspace(p), dev)
    _call("dma_decode", p, _ptr(q), _ptr(K), _ptr(V), _ptr(delta), delta.stride(1), _ptr(o), _ptr(lse), _ptr(sel_idx),
          _ptr(ws), ws.numel(), _stream())
    return o, lse, sel_idx


def dma_decode_state(p, device):
    """Zero-filled incremental decoding state for (B, Hq, w): int32 [B*Hq, 8 + roundup(w, 4)] (count 0 everywhere)."""
    n = ctypes.c_size_t()
    _check(lib().dma_decode_state_bytes(ctypes.byref(p), ctypes.byref(n)), "dma_decode_state_bytes")
    return torch.zeros(p.B * p.Hq, n.value // 4 // (p.B * p.Hq), dtype=torch.int32, device=device)


def dma_decode_state_init(p, delta, state, ws=None):
    if ws is None:
        ws = _ws(dma_decode_workspace(p), delta.device)
    _call("dma_decode_state_init", p, _ptr(delta), delta.stride(1), _ptr(state), _ptr(ws), ws.numel(), _stream())
    return state


def dma_decode_step(p, q, K, V, delta, state, o=None, lse=None, ws=None):
    """One decoding step with the carried state (p.L counts the cached keys including the one just appended)."""
    _elem(p, q, K, V, o)
    dev = q.device
    if o is None:
        o = torch.empty_like(q)
    if lse is None:
        lse = torch.empty(p.B, p.Hq, dtype=torch.float32, device=dev)
    if ws is None:
        ws = _ws(dma_decode_workspace(p), dev)
    _call("dma_decode_step", p, _ptr(q), _ptr(K), _ptr(V), _ptr(delta), delta.stride(1), _ptr(state), _ptr(o), _ptr(lse),
          _ptr(ws), ws.numel(), _stream())
    return o, lse


def decode_state_sets(state, w):
    """The kept index sets of a state tensor: list over rows of sorted Python lists."""
    st = state.cpu()
    return [sorted(st[r, 8:8 + int(st[r, 0])].tolist()) for r in range(st.shape[0])]


def dma_attn_fwd(p, Q, K, V, bias, expiry, bitmap, O=None, lse=None, ws=None):
    """Returns (O like Q, lse [B,Hq,L] fp32)."""
    _elem(p, Q, K, V, O)
    if O is None:
        O = torch.empty_like(Q)
    if lse is None:
        lse = torch.empty(p.B, p.Hq, p.L, dtype=torch.float32, device=Q.device)
    if ws is None:
        ws = _ws(dma_query_workspace(p)[1], Q.device)
    _call("dma_attn_fwd", p, _ptr(Q), _ptr(K), _ptr(V), _ptr(bias), _ptr(expiry), _ptr(bitmap), _ptr(O), _ptr(lse), _ptr(ws),
          ws.numel(), _stream())
    return O, lse


def dma_attn_fwd_chunk(p, q_begin, Q, K, V, bias, expiry, O=None, lse=None, ws=None):
    """Forward for the query rows q_begin .. q_begin + Q.shape[1] - 1 of a sequence of p.L keys; returns (O like Q, lse [B,Hq,q_len])."""
    _elem(p, Q, K, V, O)
    q_len = Q.shape[1]
    if O is None:
        O = torch.empty_like(Q)
    if lse is None:
        lse = torch.empty(p.B, p.Hq, q_len, dtype=torch.float32, device=Q.device)
    if ws is None:
        pc = dma_problem_t.from_buffer_copy(bytes(p))
        pc.flags |= DMA_FLAG_COMPACT_KV
        ws = _ws(dma_query_workspace(pc)[1], Q.device)
    _call("dma_attn_fwd_chunk", p, q_begin, q_len, _ptr(Q), _ptr(K), _ptr(V), _ptr(bias), _ptr(expiry), _ptr(O), _ptr(lse),
          _ptr(ws), ws.numel(), _stream())
    return O, lse


def dma_attn_bwd(p, Q, K, V, O, dO, lse, bias, expiry, bitmap, dQ=None, dK=None, dV=None, dM=None, ws=None):
    """Returns (dQ like Q, dK like K, dV like V, dM [B,Hq,L] fp32)."""
    _elem(p, Q, K, V, O, dO, dQ, dK, dV)
    dQ = torch.empty_like(Q) if dQ is None else dQ
    dK = torch.empty_like(K) if dK is None else dK
    dV = torch.empty_like(V) if dV is None else dV
    if dM is None:
        dM = torch.empty(p.B, p.Hq, p.L, dtype=torch.float32, device=Q.device)
    if ws is None:
        ws = _ws(dma_query_workspace(p)[2], Q.device)
    _call("dma_attn_bwd", p, _ptr(Q), _ptr(K), _ptr(V), _ptr(O), _ptr(dO), _ptr(lse), _ptr(bias), _ptr(expiry), _ptr(bitmap),
          _ptr(dQ), _ptr(dK), _ptr(dV), _ptr(dM), _ptr(ws), ws.numel(), _stream())
    return dQ, dK, dV, dM


def cache(Hq=1, Hkv=1, d=64, w=1, dtype=torch.bfloat16, rows=1, nseq=1, page_size=64, num_pages=1, max_blocks=1, flags=0, softmax_scale=0.0):
    """Descriptor of a paged 4-bit cache and of one call's rows (contiguous q, K, V, o; strides are set on the result). dma_page_plan
    reads the rows, sequences and pages only."""
    c = dma_cache_t()
    c.Hq, c.Hkv, c.d, c.w, c.dtype = Hq, Hkv, d, w, _dtype_code(dtype)
    c.page_size, c.num_pages, c.max_blocks, c.nseq, c.rows = page_size, num_pages, max_blocks, nseq, rows
    c.flags, c.softmax_scale = flags, softmax_scale
    return c


# Checks of the paged calls: a tensor that the library would misread is refused before its address is passed on. They take the host's time of every token, so each
# tensor has one call that tests it and returns its address (0.3 us; the tests by keyword that these replace took half of a call's 14 us).
def _here():
    """The current device, whose stream and memory the library uses."""
    return torch.cuda.current_device() if _raw_device is None else _raw_device()


def _flat(name, t, dtype, n, dev):
    """Address of at least n contiguous entries of `dtype` on the device."""
    if t.dtype is not dtype:
        raise TypeError(f"{name}: {t.dtype} where {dtype} is read")
    if t.get_device() != dev:
        raise ValueError(f"{name} is on {t.device}, the call runs on cuda:{dev}")
    if t.numel() < n or not t.is_contiguous():
        raise ValueError(f"{name}: {n} contiguous entries are read or written, it is {tuple(t.shape)} with strides {t.stride()}")
    return t.data_ptr()


def _same_layout(shape, got, want):
    return got == want or all(n <= 1 or a == b for n, a, b in zip(shape, got, want))


def _row_major(name, t, dtype, rows, heads, d, stride, dev):
    """Address of [rows, heads, d] laid out as the descriptor's row and head strides say."""
    if t.dtype is not dtype:
        raise TypeError(f"{name}: {t.dtype} where {dtype} is read")
    if t.get_device() != dev:
        raise ValueError(f"{name} is on {t.device}, the call runs on cuda:{dev}")
    shape = t.shape
    if shape != (rows, heads, d) and (len(shape) != 3 or shape[0] < rows or shape[1] != heads or shape[2] != d):
        raise ValueError(f"{name}: shape {tuple(shape)} where [{rows}, {heads}, {d}] is read")
    row = stride[0]
    if not (t.is_contiguous() if row == 0 and stride[1] == 0 else _same_layout(shape, t.stride(), (row, stride[1], 1))):
        raise ValueError(f"{name}: strides {t.stride()} differ from the descriptor's")
    return t.data_ptr()


def _written(name, t, dtype, rows, heads, d, dev):
    """Address, row and head strides of [rows, heads, d] that is written in its own layout (0, 0: contiguous). A stride that no second row or head takes is the contiguous one."""
    if t.dtype is not dtype:
        raise TypeError(f"{name}: {t.dtype} where {dtype} is written")
    if t.get_device() != dev:
        raise ValueError(f"{name} is on {t.device}, the call runs on cuda:{dev}")
    shape = t.shape
    if shape != (rows, heads, d) and (len(shape) != 3 or shape[0] < rows or shape[1] != heads or shape[2] != d):
        raise ValueError(f"{name}: shape {tuple(shape)} where [{rows}, {heads}, {d}] is written")
    if t.is_contiguous():
        return t.data_ptr(), 0, 0
    row, head, one = t.stride()
    if one != 1:
        raise ValueError(f"{name}: strides {t.stride()}, the channels of a head lie side by side")
    return t.data_ptr(), row if shape[0] > 1 else heads * d, head if heads > 1 else d


def _table(c, t, dev):
    if t.dtype is not torch.int32:
        raise TypeError(f"block_table: {t.dtype} where {torch.int32} is read")
    if t.get_device() != dev:
        raise ValueError(f"block_table is on {t.device}, the call runs on cuda:{dev}")
    blocks, shape = c.max_blocks, t.shape
    ld = c.table_ld or blocks
    if len(shape) != 2 or shape[0] < c.nseq or shape[1] < blocks or not _same_layout(shape, t.stride(), (ld, 1)):
        raise ValueError(f"block_table: {tuple(shape)} with strides {t.stride()} where [{c.nseq}, {blocks}] with rows of {ld} is read")
    return t.data_ptr()


def _by_head(name, t, heads, rows, dev):
    """Address and row stride of [heads, >= rows] fp32."""
    if t.dtype is not torch.float32:
        raise TypeError(f"{name}: {t.dtype} where {torch.float32} is read")
    if t.get_device() != dev:
        raise ValueError(f"{name} is on {t.device}, the call runs on cuda:{dev}")
    shape, (ld, one) = t.shape, t.stride() if t.dim() == 2 else (0, 0)
    if len(shape) != 2 or shape[0] < heads or shape[1] < rows or (one != 1 and shape[1] > 1):
        raise ValueError(f"{name}: {tuple(shape)} with strides {t.stride()} where [{heads}, {rows}] is read")
    return t.data_ptr(), ld if shape[0] > 1 else max(rows, shape[1])


def _pool(c, codes, scales, delta, heads, kv_heads, d, dev):
    keys = c.num_pages * c.page_size
    return (_flat("codes", codes, torch.uint8, keys * kv_heads * d, dev), _flat("scales", scales, torch.bfloat16, keys * kv_heads * (d // 16), dev),
            _flat("delta", delta, torch.float32, keys * heads, dev))


def dma_cache4_bytes(c):
    """Bytes of (codes, scales, delta)."""
    n = [ctypes.c_size_t() for _ in range(3)]
    _check(lib().dma_cache4_bytes(ctypes.byref(c), *map(ctypes.byref, n)), "dma_cache4_bytes")
    return tuple(x.value for x in n)


def cache4(c, device):
    """Arrays of the descriptor's pool: (codes uint8, scales bf16, delta fp32), zero-filled."""
    return (torch.zeros(c.num_pages, c.Hkv, c.page_size, 2, c.d // 2, dtype=torch.uint8, device=device),
            torch.zeros(c.num_pages, c.Hkv, c.page_size, 2, c.d // 64, 2, dtype=torch.bfloat16, device=device),
            torch.zeros(c.num_pages, c.Hq, c.page_size, dtype=torch.float32, device=device))


def dma_page_plan(c, lens, want, block_table, free_pages, pool, lens_out=None, pool_out=None, cu_rows=None, row_seq=None, row_pos=None, slot=None):
    """Pages for the sequences' new lengths (int32 tensors; block_table and free_pages are updated in place). Returns (lens_out,
    pool_out, cu_rows, row_seq, row_pos, slot)."""
    dev, i32, nseq, rows = _here(), torch.int32, c.nseq, c.rows

    def new(t, n):
        return torch.empty(n, dtype=i32, device=lens.device) if t is None else t
    lens_out, pool_out, cu_rows = new(lens_out, nseq), new(pool_out, 4), new(cu_rows, nseq + 1)
    row_seq, row_pos, slot = new(row_seq, rows), new(row_pos, rows), new(slot, rows)
    _call("dma_page_plan", ctypes.byref(c), _flat("lens", lens, i32, nseq, dev), _flat("want", want, i32, nseq, dev), _table(c, block_table, dev),
          _flat("free_pages", free_pages, i32, c.num_pages, dev), _flat("pool", pool, i32, 4, dev), _flat("lens_out", lens_out, i32, nseq, dev),
          _flat("pool_out", pool_out, i32, 4, dev), _flat("cu_rows", cu_rows, i32, nseq + 1, dev), _flat("row_seq", row_seq, i32, rows, dev),
          _flat("row_pos", row_pos, i32, rows, dev), _flat("slot", slot, i32, rows, dev), _stream())
    return lens_out, pool_out, cu_rows, row_seq, row_pos, slot


def dma_cache4_append(c, K, V, slot, codes, scales, delta, W_delta=None, A=None, delta_new=None):
    """Writes the rows K, V [rows, Hkv, d] into their slots, with the dynamic weights of V (W_delta [Hq, d], A [Hq]) or those given
    as delta_new [Hq, >= rows]."""
    dev, rows, heads, kv_heads, d, dt = _here(), c.rows, c.Hq, c.Hkv, c.d, torch.bfloat16 if c.dtype == DMA_BF16 else torch.float32
    given, ld, w, a = None, 0, None, None
    if delta_new is not None:
        given, ld = _by_head("delta_new", delta_new, heads, rows, dev)
    elif W_delta is None or A is None:
        raise ValueError("either W_delta and A or delta_new")
    else:
        w, a = _flat("W_delta", W_delta, torch.float32, heads * d, dev), _flat("A", A, torch.float32, heads, dev)
    _call("dma_cache4_append", ctypes.byref(c), _row_major("K", K, dt, rows, kv_heads, d, c.k_stride, dev), _row_major("V", V, dt, rows, kv_heads, d, c.v_stride, dev),
          w, a, given, ld, _flat("slot", slot, torch.int32, rows, dev), *_pool(c, codes, scales, delta, heads, kv_heads, d, dev), _stream())


def dma_cache4_read(c, codes, scales, delta, slot, K=None, V=None, delta_out=None, want_delta=True):
    """The rows in the given slots: (K, V [rows, Hkv, d], delta_out [Hq, rows] or None). K and V that are given are written as they are laid out, new ones are contiguous:
    the descriptor's k_stride and v_stride, which may be those of the rows that dma_cache4_append took, are not asked."""
    dev, rows, heads, kv_heads, d, dt = _here(), c.rows, c.Hq, c.Hkv, c.d, torch.bfloat16 if c.dtype == DMA_BF16 else torch.float32
    K = torch.empty(rows, kv_heads, d, dtype=dt, device=slot.device) if K is None else K
    V = torch.empty(rows, kv_heads, d, dtype=dt, device=slot.device) if V is None else V
    if delta_out is None and want_delta:
        delta_out = torch.empty(heads, rows, dtype=torch.float32, device=slot.device)
    out, ld = (None, 0) if delta_out is None else _by_head("delta_out", delta_out, heads, rows, dev)
    k, k_row, k_head = _written("K", K, dt, rows, kv_heads, d, dev)
    v, v_row, v_head = _written("V", V, dt, rows, kv_heads, d, dev)
    if _KV_STRIDES.unpack_from(c, _KV_AT) != (k_row, k_head, v_row, v_head):
        c = dma_cache_t.from_buffer_copy(c)
        _KV_STRIDES.pack_into(c, _KV_AT, k_row, k_head, v_row, v_head)
    _call("dma_cache4_read", ctypes.byref(c), *_pool(c, codes, scales, delta, heads, kv_heads, d, dev), _flat("slot", slot, torch.int32, rows, dev), k, v, out, ld, _stream())
    return K, V, delta_out


def dma_cache4_decode_workspace(c):
    n = ctypes.c_size_t()
    _check(lib().dma_cache4_decode_workspace(ctypes.byref(c), ctypes.byref(n)), "dma_cache4_decode_workspace")
    return n.value


def dma_cache4_decode(c, q, codes, scales, delta, block_table, row_seq, row_pos, o=None, lse=None, ws=None):
    """One step over the pages for every row; returns (o [rows, Hq, d], lse [rows, Hq])."""
    dev, rows, heads, d, dt = _here(), c.rows, c.Hq, c.d, torch.bfloat16 if c.dtype == DMA_BF16 else torch.float32
    if o is None:
        o = torch.empty(rows, heads, d, dtype=q.dtype, device=q.device)
    if lse is None:
        lse = torch.empty(rows, heads, dtype=torch.float32, device=q.device)
    if ws is None:
        ws = _ws(dma_cache4_decode_workspace(c), q.device)
    _call("dma_cache4_decode", ctypes.byref(c), _row_major("q", q, dt, rows, heads, d, c.q_stride, dev), *_pool(c, codes, scales, delta, heads, c.Hkv, d, dev),
          _table(c, block_table, dev), _flat("row_seq", row_seq, torch.int32, rows, dev), _flat("row_pos", row_pos, torch.int32, rows, dev),
          _row_major("o", o, dt, rows, heads, d, c.o_stride, dev), _flat("lse", lse, torch.float32, rows * heads, dev), _flat("ws", ws, torch.uint8, 0, dev), ws.numel(), _stream())
    return o, lse


def dma_read_status(ws):
    return _typed_fn("dma_read_status")(_ptr(ws), _stream())


def dma_launch_count():
    return lib().dma_launch_count()


def dma_kernel_timing(enable):
    """Starts (discarding earlier records) or stops the recording of event pairs around each attention call's main kernel."""
    _check(lib().dma_kernel_timing(int(bool(enable))), "dma_kernel_timing")


def dma_kernel_timing_read(capacity=4096):
    """[(stage, ms), ...] of the launches recorded so far, in call order; stage is "fwd" or "bwd"."""
    ms = (ctypes.c_float * capacity)()
    which = (ctypes.c_int32 * capacity)()
    n = ctypes.c_int32()
    _check(lib().dma_kernel_timing_read(ms, which, capacity, ctypes.byref(n)), "dma_kernel_timing_read")
    return [("bwd" if which[i] else "fwd", float(ms[i])) for i in range(min(n.value, capacity))]


def dma_step_host_arena(p, backward):
    n = ctypes.c_size_t()
    _check(lib().dma_step_host_arena(ctypes.byref(p), int(backward), ctypes.byref(n)), "dma_step_host_arena")
    return n.value


def dma_step_host(p, backward, hQ, hK, hV, hdO, hW, hA, hO, hlse, hdQ, hdK, hdV, hdM, arena):
    """All h* are CPU tensors (ideally pinned); `arena` is a CUDA uint8 tensor of dma_step_host_arena() bytes."""
    _call("dma_step_host", p, int(backward), _ptr(hQ), _ptr(hK), _ptr(hV), _ptr(hdO), _ptr(hW), _ptr(hA), _ptr(hO), _ptr(hlse),
          _ptr(hdQ), _ptr(hdK), _ptr(hdV), _ptr(hdM), _ptr(arena), arena.numel(), _stream())


def dma_mask_build_static(p, V, W_delta, A, bias, expiry, bitmap):
    """dma_mask_build without a workspace: the scratch is a fixed array inside the library (see include/dma.h for
    the size limit and the sharing rules). Outputs must be preallocated by the caller; nothing is allocated here."""
    _elem(p, V)
    _call("dma_mask_build_static", p, _ptr(V), _ptr(W_delta), _ptr(A), _ptr(bias), _ptr(expiry), _ptr(bitmap), _stream())
    return bias, expiry, bitmap


def dma_selftest_wait_timeout(ws):
    """Launches the bounded-wait self test; afterwards dma_read_status(ws) reports DMA_ERR_DEVICE_TIMEOUT (-7)."""
    _call("dma_selftest_wait_timeout", _ptr(ws), ws.numel(), _stream())
