"""Python names for the C entry points (same names, argument marshalling only)."""
from __future__ import annotations

import ctypes as C
import struct
from typing import Optional, Sequence

from . import _cabi as K


class RgError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = K.load().rg_status_string(status).decode()
        super().__init__(f"{where}: {K.STATUS_NAMES.get(status, status)} ({msg})")


def _check(status: int, where: str):
    if status != K.RG_OK:
        raise RgError(status, where)


def rg_desc(*, cuts: Sequence[int] = (), tree: int = K.RG_TREE_BALANCED, fma: int = 0, BM: int = 0, BN: int = 0,
            BK: int = 0, stages: int = 0, cta_group: int = 0, raster: int = 0, split_merge: int = 0, **order_fields) -> K.rg_desc_t:
    """A descriptor with the library defaults (rg_desc_init), then the given fields."""
    d = K.rg_desc_t()
    K.load().rg_desc_init(C.byref(d))
    d.BM, d.BN, d.BK, d.stages, d.cta_group, d.raster, d.split_merge = BM, BN, BK, stages, cta_group, raster, split_merge
    d.tree, d.fma = tree, fma
    for k, v in order_fields.items():
        setattr(d, k, v)
    if "in_dtype" not in order_fields:
        d.in_dtype = K.RG_BF16
    if d.in_dtype == K.RG_F8E4M3 and "atom" not in order_fields:
        d.atom = K.RG_ATOM_TC_F8_K32           # the 8-bit operand type and the 32-wide step go together
    cuts = list(cuts)
    if len(cuts) > K.RG_MAX_CUTS:
        raise RgError(2, "rg_desc")
    d.n_cuts = len(cuts)
    for i, c in enumerate(cuts):
        d.cuts[i] = int(c)
    return d


def rg_desc_validate(d: K.rg_desc_t, M: int, N: int, Kdim: int) -> int:
    return int(K.load().rg_desc_validate(C.byref(d), M, N, Kdim))


def rg_desc_class(d: K.rg_desc_t) -> int:
    return int(K.load().rg_desc_class(C.byref(d)))


def rg_gemm_workspace_bytes(d: K.rg_desc_t, M: int, N: int) -> int:
    return int(K.load().rg_gemm_workspace_bytes(C.byref(d), M, N))


def rg_status_string(status: int) -> str:
    return K.load().rg_status_string(status).decode()


def rg_device_status() -> int:
    """Read and clear the device health word (synchronises).  0 = healthy."""
    code = C.c_uint32(0)
    K.load().rg_device_status(C.byref(code))
    return int(code.value)


def rg_selftest_exp(form: int, x, y):
    """y[i] = FORM(x[i]) by the device functions the kernels use (forms: see include/rg.h).  x, y: float32 CUDA tensors."""
    st = K.load().rg_selftest_exp(int(form), x.data_ptr(), y.data_ptr(), int(x.numel()), _stream(x))
    _check(st, "rg_selftest_exp")
    return y


def rg_selftest_bounded_wait(limit_ns: int, counter):
    """Launch the bounded-wait self-test (see include/rg.h).  `counter`: a zeroed CUDA int32/uint32
    tensor of one element; it holds 2 afterwards (both warps abandoned their wait)."""
    st = K.load().rg_selftest_bounded_wait(int(limit_ns), counter.data_ptr(), _stream(counter))
    _check(st, "rg_selftest_bounded_wait")


# ---------------------------------------------------------------- marshalling
def _dtype_code(t) -> int:
    import torch
    if t.dtype == torch.bfloat16:
        return K.RG_BF16
    if t.dtype == torch.float32:
        return K.RG_F32
    if t.dtype == torch.float16:
        return K.RG_F16
    if t.dtype == torch.float8_e4m3fn:
        return K.RG_F8E4M3
    raise TypeError(f"rg tensors are bfloat16, float16, float32 or float8_e4m3fn, got {t.dtype}")


def _tensor(t) -> K.rg_tensor_t:
    if t.dim() == 1:
        return K.rg_tensor_t(t.data_ptr(), _dtype_code(t), t.shape[0], 1, int(t.stride(0)) if t.shape[0] > 1 else 1)
    assert t.dim() == 2 and (t.shape[1] <= 1 or t.stride(1) == 1), "rows must be contiguous"
    ld = int(t.stride(0)) if t.shape[0] > 1 else max(int(t.stride(0)), int(t.shape[1]))      # rows that overlap are the library's to refuse
    return K.rg_tensor_t(t.data_ptr(), _dtype_code(t), t.shape[0], t.shape[1], ld)


def _workspace(ws):
    """Address of a workspace tensor and the bytes it has there: an expanded one has fewer than its elements say."""
    if ws is None:
        return None, 0
    n = ws.numel()
    if n and not ws.is_contiguous():
        n = min(n, 1 + sum((size - 1) * stride for size, stride in zip(ws.shape, ws.stride())))
    return ws.data_ptr(), n * ws.element_size()


def _epilogue(bias, act, residual) -> Optional[K.rg_epilogue_t]:
    if bias is None and residual is None and not act:
        return None
    e = K.rg_epilogue_t()
    e.act = int(act)
    if bias is not None:
        e.bias, e.bias_dtype = bias.data_ptr(), _dtype_code(bias)
    if residual is not None:
        e.residual, e.residual_dtype, e.ldr = residual.data_ptr(), _dtype_code(residual), int(residual.stride(0))
    return e


def _stream(t) -> int:
    import torch
    return torch.cuda.current_stream(t.device).cuda_stream if t.is_cuda else 0


def rg_gemm(d: K.rg_desc_t, A, B, C_out, *, bias=None, act: int = 0, residual=None, ws=None):
    """C_out[M,N] = epilogue(A[M,K] @ B[N,K]^T) with the bits the descriptor fixes.
    All tensors are CUDA tensors; `ws` is a CUDA byte/float tensor of at least
    rg_gemm_workspace_bytes(d, M, N) bytes when the descriptor has cuts."""
    L = K.load()
    a, b, c = _tensor(A), _tensor(B), _tensor(C_out)
    e = _epilogue(bias, act, residual)
    ws_ptr, ws_bytes = _workspace(ws)
    st = L.rg_gemm(C.byref(d), C.byref(a), C.byref(b), C.byref(c), C.byref(e) if e is not None else None,
                   ws_ptr, ws_bytes, _stream(A))
    _check(st, "rg_gemm")
    return C_out


def rg_gemm_noalloc(d: K.rg_desc_t, A, B, C_out, *, bias=None, act: int = 0, residual=None):
    """rg_gemm for callers that cannot allocate device memory: the split-K workspace is a fixed
    array inside the library (at most RG_NOALLOC_WS_BYTES; larger shapes raise RG_ERR_WORKSPACE).
    Calls on one device share that array, so do not let two of them overlap on the GPU."""
    L = K.load()
    a, b, c = _tensor(A), _tensor(B), _tensor(C_out)
    e = _epilogue(bias, act, residual)
    st = L.rg_gemm_noalloc(C.byref(d), C.byref(a), C.byref(b), C.byref(c), C.byref(e) if e is not None else None,
                           _stream(A))
    _check(st, "rg_gemm_noalloc")
    return C_out


def rg_reduce_rows(d: K.rg_desc_t, op: int, x, out, *, weight=None, eps: float = 0.0, aux_out=None):
    """Row reduction with the descriptor's tree (see include/rg.h for the three operations)."""
    L = K.load()
    xt, ot = _tensor(x), _tensor(out)
    args = K.rg_reduce_args_t()
    if weight is not None:
        args.weight, args.weight_dtype = weight.data_ptr(), _dtype_code(weight)
    args.eps = float(eps)
    if aux_out is not None:
        args.aux_out = aux_out.data_ptr()
    st = L.rg_reduce_rows(C.byref(d), int(op), C.byref(xt), C.byref(ot), C.byref(args), _stream(x))
    _check(st, "rg_reduce_rows")
    return out


def rg_attn_desc(*, block_n: int, scale: float, heads: int = 1, sum_tree: int = K.RG_TREE_BALANCED, p_dtype: int = K.RG_BF16,
                 mask: int = 0, div_place: int = 0, exp_base: int = 0, block_m: int = 0) -> K.rg_attn_desc_t:
    d = K.rg_attn_desc_t()
    d.size = C.sizeof(K.rg_attn_desc_t)
    d.heads, d.block_n, d.scale = heads, block_n, scale
    d.block_m = block_m if block_m else (128 if mask else 0)
    d.sum_tree, d.p_dtype, d.mask, d.div_place, d.exp_base = sum_tree, p_dtype, mask, div_place, exp_base
    return d


def rg_attention(d: K.rg_attn_desc_t, Q, Kt, Vt, O):
    """O = attention(Q, K, V) with the descriptor's key-block recurrence.  Q [heads*Nq, d],
    Kt [heads*Nk, d], Vt [heads*d, Nk] (V transposed), O [heads*Nq, d]: CUDA tensors."""
    L = K.load()
    q, k, v, o = _tensor(Q), _tensor(Kt), _tensor(Vt), _tensor(O)
    st = L.rg_attention(C.byref(d), C.byref(q), C.byref(k), C.byref(v), C.byref(o), _stream(Q))
    _check(st, "rg_attention")
    return O


def rg_reduce_cols_workspace_bytes(rows: int, cols: int) -> int:
    return int(K.load().rg_reduce_cols_workspace_bytes(rows, cols))


def rg_reduce_cols(d: K.rg_desc_t, op: int, x, out, *, y=None, ws=None):
    """Reduction along axis 0 with the descriptor's tree: out[c] = TREE_r x[r, c] (RG_COLOP_SUM) or
    TREE_r x[r, c] * y[r, c] (RG_COLOP_DOT).  `ws`: CUDA tensor of at least
    rg_reduce_cols_workspace_bytes(rows, cols) bytes when x has more than 256 rows."""
    L = K.load()
    xt, ot = _tensor(x), _tensor(out)
    yt = _tensor(y) if y is not None else None
    ws_ptr, ws_bytes = _workspace(ws)
    st = L.rg_reduce_cols(C.byref(d), int(op), C.byref(xt), C.byref(yt) if yt is not None else None, C.byref(ot),
                          ws_ptr, ws_bytes, _stream(x))
    _check(st, "rg_reduce_cols")
    return out


def rg_gemm_host(d: K.rg_desc_t, A, B, C_out, dev_scratch, *, bias=None, act: int = 0, residual=None):
    """Host-buffer form: A, B, C_out, bias, residual are CPU tensors (pinned for async copies);
    `dev_scratch` is a CUDA tensor.  Enqueues copies + kernels on the current stream."""
    L = K.load()
    a, b, c = _tensor(A), _tensor(B), _tensor(C_out)
    e = _epilogue(bias, act, residual)
    st = L.rg_gemm_host(C.byref(d), C.byref(a), C.byref(b), C.byref(c), C.byref(e) if e is not None else None,
                        *_workspace(dev_scratch), _stream(dev_scratch))
    _check(st, "rg_gemm_host")
    return C_out


def rg_gemm_host_scratch_bytes(d, M, N, Kdim, c_dtype, bias=None, act=0, residual=None) -> int:
    e = _epilogue(bias, act, residual)
    return int(K.load().rg_gemm_host_scratch_bytes(C.byref(d), M, N, Kdim, c_dtype, C.byref(e) if e is not None else None))


def rg_reduce_rows_host(d: K.rg_desc_t, op: int, x, out, dev_scratch, *, weight=None, eps: float = 0.0, aux_out=None):
    L = K.load()
    xt, ot = _tensor(x), _tensor(out)
    args = K.rg_reduce_args_t()
    if weight is not None:
        args.weight, args.weight_dtype = weight.data_ptr(), _dtype_code(weight)
    args.eps = float(eps)
    if aux_out is not None:
        args.aux_out = aux_out.data_ptr()
    st = L.rg_reduce_rows_host(C.byref(d), int(op), C.byref(xt), C.byref(ot), C.byref(args),
                               *_workspace(dev_scratch), _stream(dev_scratch))
    _check(st, "rg_reduce_rows_host")
    return out


def rg_reduce_rows_host_scratch_bytes(op, x, out) -> int:
    xt, ot = _tensor(x), _tensor(out)
    return int(K.load().rg_reduce_rows_host_scratch_bytes(int(op), C.byref(xt), C.byref(ot)))


# ---------------------------------------------------------------- positions, paged cache, attention over it
# These calls are a few microseconds of GPU work in a decode step: their C structures are packed in one go (a ctypes structure
# costs a microsecond more) and passed as bytes.
_ROWS, _CACHE, _TENSOR = struct.Struct("@Pi5q"), struct.Struct("@Pi7q"), struct.Struct("@Pi3q")
_CODES, _POSITION_CODES = {}, {}


def _code(t) -> int:
    c = _CODES.get(t.dtype)
    if c is None:
        c = _CODES[t.dtype] = _dtype_code(t)
    return c


def _rows(t) -> bytes:
    if t.dim() != 3:
        raise ValueError(f"rows are [tokens, heads, dim], got a tensor of {t.dim()} dimensions")
    n, h, d = t.shape
    st, sh, sd = t.stride()
    if sd != 1 and d > 1:
        raise ValueError("the elements of a head must be contiguous")
    return _ROWS.pack(t.data_ptr(), _code(t), n, h, d, st, sh)


def _cache(t) -> bytes:
    if t.dim() != 4:
        raise ValueError(f"a cache is [pages, page_size, heads, dim], got a tensor of {t.dim()} dimensions")
    n, page, h, d = t.shape
    sn, sp, sh, sd = t.stride()
    if sd != 1 and d > 1:
        raise ValueError("the elements of a head must be contiguous")
    return _CACHE.pack(t.data_ptr(), _code(t), n, page, h, d, sn, sp, sh)


def _positions(pos) -> bytes:
    code = _POSITION_CODES.get(pos.dtype)
    if code is None:
        import torch
        _POSITION_CODES.update({torch.int32: K.RG_I32, torch.int64: K.RG_I64})
        if pos.dtype not in _POSITION_CODES:
            raise TypeError(f"positions are int32 or int64, got {pos.dtype}")
        code = _POSITION_CODES[pos.dtype]
    shape, stride = pos.shape, pos.stride()
    n = shape[-1] if shape else 0
    if len(shape) not in (1, 2) or (n > 1 and stride[-1] != 1):
        raise ValueError("positions are [tokens] or [axes, tokens], contiguous along the tokens")
    if len(shape) == 1:
        return _TENSOR.pack(pos.data_ptr(), code, 1, n, n)
    return _TENSOR.pack(pos.data_ptr(), code, shape[0], n, stride[0])


def _frequencies(inv_freq, d) -> int:
    import torch
    if inv_freq.dtype != torch.float64 or not inv_freq.is_contiguous() or inv_freq.numel() != d.rot_dim // 2:
        raise ValueError(f"inv_freq is a contiguous float64 tensor of rot_dim / 2 = {d.rot_dim // 2} elements")
    return inv_freq.data_ptr()


_get_device = _raw_stream = None


def _call(where: str, fn, device: int, *args):
    """One C call with `device` current and on its current stream."""
    global _get_device, _raw_stream
    if _get_device is None:                              # what torch.cuda.current_device() and current_stream() come down to for initialised CUDA
        import torch
        _get_device, _raw_stream = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream
    if device == _get_device():
        st = fn(*args, _raw_stream(device))
    else:
        import torch
        with torch.cuda.device(device):
            st = fn(*args, _raw_stream(device))
    if st:
        raise RgError(st, where)


def _one_device(where: str, *tensors) -> int:
    device = tensors[0].get_device()
    for t in tensors:
        if t is not None and t.get_device() != device:
            raise ValueError(f"{where}: tensors on different devices")
    if device < 0:
        raise ValueError(f"{where}: tensors must be on a CUDA device")
    return device


def _fits(bits: int, *values) -> bool:
    """Whether unsigned fields of so many bits hold the values (ctypes drops what they do not)."""
    return all(0 <= v < 1 << bits for v in values)


def rg_rope_desc(*, rot_dim: int, style: int = K.RG_ROPE_HALF, sections: Sequence[int] = (), inverse: int = 0) -> K.rg_rope_desc_t:
    """Rotary positions (see include/rg.h): `sections` gives the pairs of each axis (default: one axis with all of them)."""
    d = K.rg_rope_desc_t()
    sections = tuple(sections) or (rot_dim // 2,)
    if len(sections) > 4 or not _fits(32, rot_dim, *sections) or not _fits(8, style, int(inverse)):
        raise RgError(2, "rg_rope_desc")
    d.size, d.rot_dim, d.style, d.n_axes, d.inverse = C.sizeof(K.rg_rope_desc_t), rot_dim, style, len(sections), int(inverse)
    for i, n in enumerate(sections):
        d.sections[i] = n
    return d


def rg_rope(d: K.rg_rope_desc_t, x, pos, inv_freq, out):
    """out = x [tokens, heads, dim] rotated by `pos` ([tokens] or [axes, tokens], int32 or int64); inv_freq: float64 [rot_dim / 2],
    radians per position.  out may be x."""
    device = _one_device("rg_rope", x, pos, inv_freq, out)
    _call("rg_rope", K.load().rg_rope, device, C.byref(d), _rows(x), _positions(pos), _frequencies(inv_freq, d), _rows(out))
    return out


class rg_paged_seqs:
    """The sequences of a batch (see include/rg.h): int32 CUDA tensors block_table [n, pages] (one row expanded to n is fine: all sequences
    read the same pages), seq_lens [n] and cu_q [n + 1], and the host's bounds of new tokens in one sequence and of seq_lens (0: none known).  The tensors are read when the kernels run."""
    __slots__ = ("block_table", "seq_lens", "cu_q", "device", "c")

    def get_device(self) -> int:
        return self.device

    def __init__(self, block_table, seq_lens, cu_q, *, max_q: int = 0, max_len: int = 0):
        import torch
        for name, t, dims in (("block_table", block_table, 2), ("seq_lens", seq_lens, 1), ("cu_q", cu_q, 1)):
            if t.dtype != torch.int32 or t.dim() != dims or (t.shape[-1] > 1 and t.stride(-1) != 1):
                raise ValueError(f"{name} is a contiguous int32 tensor of {dims} dimension(s)")
        n = seq_lens.shape[0]
        if block_table.shape[0] != n or cu_q.shape[0] != n + 1:
            raise ValueError(f"{n} sequences need block_table [{n}, pages] and cu_q [{n + 1}], got {tuple(block_table.shape)} and {tuple(cu_q.shape)}")
        if not block_table.device == seq_lens.device == cu_q.device:
            raise ValueError("rg_paged_seqs: tensors on different devices")
        if not _fits(63, max_q, max_len):
            raise RgError(4, "rg_paged_seqs")
        cols = block_table.shape[1]
        table_ld = block_table.stride(0) if n > 1 else cols
        if 0 < table_ld < cols:
            raise ValueError(f"rows of block_table overlap: {cols} entries, {table_ld} apart")
        self.device = seq_lens.get_device()
        self.block_table, self.seq_lens, self.cu_q = block_table, seq_lens, cu_q
        self.c = K.rg_paged_seqs_t(block_table.data_ptr(), table_ld, cols, n,
                                   seq_lens.data_ptr(), cu_q.data_ptr(), max_q, max_len)


def rg_kv_append(d, k, v, inv_freq, k_cache, v_cache, seqs: rg_paged_seqs, *, pos=None, q=None, q_out=None):
    """Put keys (rotated) and values of the new tokens into their pages; rotate q into q_out.  d None: nothing is rotated."""
    if (q is None) != (q_out is None):
        raise ValueError("rg_kv_append: q and q_out go together")
    device = _one_device("rg_kv_append", k, v, inv_freq, k_cache, v_cache, seqs, pos, q, q_out)
    _call("rg_kv_append", K.load().rg_kv_append, device, C.byref(d) if d is not None else None, _rows(k), _rows(v),
          _positions(pos) if pos is not None else None, None if inv_freq is None else inv_freq.data_ptr() if d is None else _frequencies(inv_freq, d),
          _cache(k_cache), _cache(v_cache), C.byref(seqs.c), _rows(q) if q is not None else None, _rows(q_out) if q_out is not None else None)


def rg_paged_attn_desc(*, scale: float, split: int = 0, window: int = 0, mask: int = 1) -> K.rg_paged_attn_desc_t:
    """Attention over a paged cache: `split` keys for each part (0: one part), a causal mask (mask=1) of the last `window` keys (0: all)."""
    if not _fits(32, split, window) or not _fits(8, mask):
        raise RgError(2, "rg_paged_attn_desc")
    return K.rg_paged_attn_desc_t(C.sizeof(K.rg_paged_attn_desc_t), split, window, scale, mask)


def rg_paged_attention_workspace_bytes(d: K.rg_paged_attn_desc_t, seqs: rg_paged_seqs, tokens: int, q_heads: int, dim: int, page_size: int = 0) -> int:
    """Bytes of workspace; `page_size` is needed where seqs has no max_len."""
    if page_size <= 0:
        if seqs.c.max_len <= 0 and d.split:
            raise ValueError("rg_paged_attention_workspace_bytes: give page_size, or seqs a max_len")
        page_size = 1 << 20                              # max_len is the bound
    return int(K.load().rg_paged_attention_workspace_bytes(C.byref(d), C.byref(seqs.c), page_size, tokens, q_heads, dim))


def _normalisers(q, lse):
    """Address and row stride of the normalisers (none: 0, 0)."""
    if lse is None:
        return None, 0
    import torch
    if lse.dtype != torch.float32 or lse.shape != q.shape[:2] or (lse.shape[1] > 1 and lse.stride(1) != 1):
        raise ValueError("lse is float32 [tokens, heads], contiguous along the heads")
    lse_ld = lse.stride(0) if lse.shape[0] > 1 else lse.shape[1]
    if lse_ld < lse.shape[1]:
        raise ValueError(f"rows of lse overlap: {lse.shape[1]} heads, {lse_ld} apart")
    return lse.data_ptr(), lse_ld


def rg_paged_attention(d: K.rg_paged_attn_desc_t, q, k_cache, v_cache, seqs: rg_paged_seqs, out, *, lse=None, ws=None):
    """out = attention of the rows q [tokens, heads, dim] over their sequences' pages; lse: float32 [tokens, heads] or None."""
    lse_ptr, lse_ld = _normalisers(q, lse)
    ws_ptr, ws_bytes = _workspace(ws)
    device = _one_device("rg_paged_attention", q, k_cache, v_cache, seqs, out, lse, ws)
    _call("rg_paged_attention", K.load().rg_paged_attention, device, C.byref(d), _rows(q), _cache(k_cache), _cache(v_cache), C.byref(seqs.c), _rows(out),
          lse_ptr, lse_ld, ws_ptr, ws_bytes)
    return out


# ---------------------------------------------------------------- four bits
class rg_weights_four:
    """Weights in four bits (see include/rg.h): codes uint8 [N, K / 2] (element 2 i in the low half of byte i), scales [N, ceil(K / group)] in
    bfloat16, float16 or float32, zeros uint8 of the scales' shape (None: all 8).  w_static=1: nothing in flight writes them."""
    __slots__ = ("codes", "scales", "zeros", "device", "c")

    def get_device(self) -> int:
        return self.device

    def __init__(self, codes, scales, *, zeros=None, group: int = 128, w_static: int = 0):
        import torch
        for name, t, types in (("codes", codes, (torch.uint8,)), ("scales", scales, (torch.bfloat16, torch.float16, torch.float32)), ("zeros", zeros, (torch.uint8,))):
            if t is not None and (t.dtype not in types or t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1)):
                raise ValueError(f"{name} is a {' or '.join(str(x) for x in types)} tensor of 2 dimensions, contiguous along the second")
        if not _fits(31, group, w_static):
            raise RgError(2, "rg_weights_four")
        N, half = codes.shape
        if group < 1 or scales.shape != (N, -(-2 * half // group)) or (zeros is not None and zeros.shape != scales.shape):
            raise ValueError(f"codes {tuple(codes.shape)} in groups of {group} do not go with scales {tuple(scales.shape)}" + (f" and zeros {tuple(zeros.shape)}" if zeros is not None else ""))
        device = codes.get_device()
        if scales.get_device() != device or (zeros is not None and zeros.get_device() != device):
            raise ValueError("rg_weights_four: tensors on different devices")
        # rows that overlap are the library's to refuse
        ld = lambda t: int(t.stride(0)) if t.shape[0] > 1 else int(t.shape[1])  # noqa: E731
        self.device, self.codes, self.scales, self.zeros = device, codes, scales, zeros
        code_ld = ld(codes) if N > 1 else -(-half // 16) * 16
        self.c = K.rg_weights_four_t(codes.data_ptr(), scales.data_ptr(), zeros.data_ptr() if zeros is not None else None, N, 2 * half, code_ld, ld(scales),
                           ld(zeros) if zeros is not None else 0, group, _code(scales), w_static)


def _matrix(t) -> bytes:
    if t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError("a matrix has 2 dimensions and contiguous rows")
    n, c = t.shape
    return _TENSOR.pack(t.data_ptr(), _code(t), n, c, t.stride(0) if n > 1 else c)       # one row: nothing lies a stride further


def rg_gemv_four(w: rg_weights_four, A, C_out, *, bias=None, act: int = 0, residual=None):
    """C_out[M, N] = epilogue(A[M, K] @ W[N, K]^T) for a few rows, W in four bits; the epilogue is rg_gemm's."""
    device = _one_device("rg_gemv_four", A, w, C_out, bias, residual)
    if bias is not None and (bias.dim() != 1 or bias.shape[0] != C_out.shape[1] or (bias.shape[0] > 1 and bias.stride(0) != 1)):
        raise ValueError(f"bias is a contiguous tensor of {C_out.shape[1]} elements")
    if residual is not None and (residual.shape != C_out.shape or (residual.shape[1] > 1 and residual.stride(1) != 1)):
        raise ValueError("residual has the result's shape and contiguous rows")
    e = _epilogue(bias, act, residual)
    if e is not None and residual is not None and residual.shape[0] <= 1:
        e.ldr = max(e.ldr, C_out.shape[1])
    _call("rg_gemv_four", K.load().rg_gemv_four, device, C.byref(w.c), _matrix(A), _matrix(C_out), C.byref(e) if e is not None else None)
    return C_out


def rg_cache_four_block_bytes(page_size: int, dim: int) -> int:
    """Bytes of one page of one head in a cache of four-bit codes."""
    return int(K.load().rg_cache_four_block_bytes(page_size, dim))


class rg_cache_four:
    """A paged cache of four-bit codes: a uint8 CUDA tensor [pages, heads, rg_cache_four_block_bytes(page_size, dim)], blocks contiguous."""
    __slots__ = ("tensor", "page_size", "dim", "device", "c")

    def get_device(self) -> int:
        return self.device

    def __init__(self, tensor, *, page_size: int, dim: int):
        import torch
        block = rg_cache_four_block_bytes(page_size, dim)
        if block == 0:
            raise RgError(3, "rg_cache_four")
        if tensor.dtype != torch.uint8 or tensor.dim() != 3 or tensor.stride(2) != 1 or tensor.shape[2] != block:
            raise ValueError(f"a cache of four-bit codes is a uint8 tensor [pages, heads, {block}], contiguous along the last dimension")
        n, h, _ = tensor.shape
        self.tensor, self.page_size, self.dim, self.device = tensor, page_size, dim, tensor.get_device()
        self.c = K.rg_cache_four_t(tensor.data_ptr(), n, page_size, h, dim, tensor.stride(0) if n > 1 else 0, tensor.stride(1) if h > 1 else 0)


def rg_kv_append_four(d, k, v, inv_freq, k_cache: rg_cache_four, v_cache: rg_cache_four, seqs: rg_paged_seqs, *, pos=None, q=None, q_out=None):
    """rg_kv_append into caches of four-bit codes."""
    if (q is None) != (q_out is None):
        raise ValueError("rg_kv_append_four: q and q_out go together")
    device = _one_device("rg_kv_append_four", k, v, inv_freq, k_cache, v_cache, seqs, pos, q, q_out)
    _call("rg_kv_append_four", K.load().rg_kv_append_four, device, C.byref(d) if d is not None else None, _rows(k), _rows(v),
          _positions(pos) if pos is not None else None, None if inv_freq is None else inv_freq.data_ptr() if d is None else _frequencies(inv_freq, d),
          C.byref(k_cache.c), C.byref(v_cache.c), C.byref(seqs.c), _rows(q) if q is not None else None, _rows(q_out) if q_out is not None else None)


def rg_kv_read_four(k_cache: rg_cache_four, v_cache: rg_cache_four, seqs: rg_paged_seqs, k_out, v_out):
    """k_out, v_out [tokens, heads, dim] = what the caches hold at the places of the batch's new tokens."""
    device = _one_device("rg_kv_read_four", k_out, v_out, k_cache, v_cache, seqs)
    _call("rg_kv_read_four", K.load().rg_kv_read_four, device, C.byref(k_cache.c), C.byref(v_cache.c), C.byref(seqs.c), _rows(k_out), _rows(v_out))
    return k_out, v_out


def rg_paged_attention_four(d: K.rg_paged_attn_desc_t, q, k_cache: rg_cache_four, v_cache: rg_cache_four, seqs: rg_paged_seqs, out, *, lse=None, ws=None):
    """rg_paged_attention over caches of four-bit codes."""
    lse_ptr, lse_ld = _normalisers(q, lse)
    ws_ptr, ws_bytes = _workspace(ws)
    device = _one_device("rg_paged_attention_four", q, k_cache, v_cache, seqs, out, lse, ws)
    _call("rg_paged_attention_four", K.load().rg_paged_attention_four, device, C.byref(d), _rows(q), C.byref(k_cache.c), C.byref(v_cache.c), C.byref(seqs.c), _rows(out),
          lse_ptr, lse_ld, ws_ptr, ws_bytes)
    return out
