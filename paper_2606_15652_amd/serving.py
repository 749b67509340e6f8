"""Binding of the operators around the MosaicQuant layers: RMS norm with 8-bit
output, the W8A8 product, the paged 4-bit cache and the attention over it.

As in the package's other calls only arguments are checked and marshalled here;
``include/mq.h`` documents each operator.  Values are fp16 or bf16.
"""
from __future__ import annotations

import ctypes as C
import math
from dataclasses import dataclass, field

from . import _check, _empty, _need, _need_out, _ptr, _scratch, _stream, _torch, load

LAYOUTS = {"rows": 0, "a8": 1}


def _types():
    global _types_of
    torch = _torch()
    _types_of = {torch.float16: 0, torch.bfloat16: 1, torch.float32: 2}
    return _types_of


_types_of = None
_INT_MAX = 2 ** 31 - 1                          # ctypes cuts what is beyond to its low 32 bits, without an error


def _dtype_code(dtype, name, fp32=False):
    code = (_types_of or _types()).get(dtype)
    if code is None or (code == 2 and not fp32):
        raise TypeError(f"{name} must be fp16{', bf16 or fp32' if fp32 else ' or bf16'}, got {dtype}")
    return code


def _need_rows(t, name, cols=None):
    """A matrix with contiguous rows (any row stride that a C int holds): its row stride; of a single row, which says
    nothing, its columns rounded up to 8."""
    if not isinstance(t, _torch().Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA (HIP) tensor")
    shape = t.shape
    if len(shape) != 2 or (cols is not None and shape[1] != cols):
        raise ValueError(f"{name} must be [rows, {'columns' if cols is None else cols}], got shape {tuple(shape)}")
    row, col = t.stride()
    if col != 1 and shape[1] > 1:
        raise ValueError(f"{name} must have contiguous rows")
    ld = row if shape[0] > 1 else -(-shape[1] // 8) * 8
    if ld > _INT_MAX or shape[0] > _INT_MAX or shape[1] > _INT_MAX:
        raise ValueError(f"{name}'s sizes and row stride must be below 2^31, got shape {tuple(shape)}, rows {ld} apart")
    return ld


def _need_max_q(max_q):
    if max_q > _INT_MAX:
        raise ValueError(f"max_q must be below 2^31, got {max_q}")


def _same_device(first, name, **others):
    at = first.get_device()
    for other, t in others.items():
        if t is not None and t.get_device() != at:
            raise ValueError(f"{other} is on {t.device}, {name} on {first.device}")


# ------------------------------------------------- 8-bit activations --
def _code_rows(M, K, device, stream):
    """int8 [M, K], rows padded to 16 bytes, and their stride."""
    ld = -(-K // 16) * 16
    rows = _empty((M, ld), _torch().int8, device, stream)
    return (rows if ld == K else rows[:, :K]), ld


def _need_codes(Xq8, K=None):
    """int8 rows as the kernels take them: (codes, row stride in bytes).  The bytes up to the next
    multiple of 16 after a row's last code have to be there too."""
    torch = _torch()
    ld = _need_rows(Xq8, "Xq8", K)
    if Xq8.dtype != torch.int8:
        raise TypeError(f"Xq8 must be torch.int8, got {Xq8.dtype}")
    M, K = Xq8.shape
    padded = -(-K // 16) * 16
    if M <= 1:
        ld = padded                             # one row: its stride says nothing
    if ld < padded or ld % 16:
        raise ValueError(f"Xq8's rows must start every multiple of 16 bytes, at least {padded}; got a row stride of {ld}")
    if padded != K and M and Xq8.storage_offset() + (M - 1) * ld + padded > Xq8.untyped_storage().nbytes():
        raise ValueError("Xq8's last row must be followed by its padding to 16 bytes")
    return ld


def rms_norm_quantize8(X, weight, eps: float = 1e-6, residual=None, layout: str = "rows", out=None, stream=None):
    """(Xq8, s_x) of the RMS norm of X [M, K], or with ``residual`` (Xq8, s_x, H) of that of
    H = X + residual.  ``layout``: "rows" (int8 [M, K] with padded rows, s_x fp32: for gemm_w8a8) or
    "a8" (uint8 [M, 3K/2], s_x fp16: for fused_gemm_a8).  ``out``: the same tensors, allocated by the
    caller; H may be X or residual itself."""
    torch = _torch()
    code = _dtype_code(getattr(X, "dtype", None), "X")
    ldx = _need_rows(X, "X")
    M, K = X.shape
    _need_out(weight, (K,), X.dtype, "weight")
    a8, H, ldq, ldr, ldh = LAYOUTS[layout] == 1, None, 0, 0, 0
    if residual is not None:
        if residual.dtype != X.dtype:
            raise TypeError(f"residual must be {X.dtype}, got {residual.dtype}")
        ldr = _need_rows(residual, "residual", K)
        if residual.shape[0] != M:
            raise ValueError(f"residual must have {M} rows, got {residual.shape[0]}")
    if out is None:
        dev = X.device
        if a8:
            Xq8 = _empty((M, 3 * K // 2), torch.uint8, dev, stream)
        else:
            Xq8, ldq = _code_rows(M, K, dev, stream)
        s_x = _empty((M,), torch.float16 if a8 else torch.float32, dev, stream)
        if residual is not None:
            H, ldh = _empty((M, K), X.dtype, dev, stream), K
        _same_device(X, "X", weight=weight, residual=residual)
    else:
        Xq8, s_x, H = (*out, None) if residual is None else out
        _need_out(s_x, (M,), torch.float16 if a8 else torch.float32, "out[1] (s_x)")
        if a8:
            _need_out(Xq8, (M, 3 * K // 2), torch.uint8, "out[0] (Xq8)")
        else:
            ldq = _need_codes(Xq8, K)
            if Xq8.shape[0] != M:
                raise ValueError(f"out[0] (Xq8) must have {M} rows, got {Xq8.shape[0]}")
        if residual is not None:
            ldh = _need_rows(H, "out[2] (H)", K)
            if H.dtype != X.dtype or H.shape[0] != M:
                raise ValueError(f"out[2] (H) must be {X.dtype} with {M} rows, got {H.dtype} with {H.shape[0]}")
        _same_device(X, "X", weight=weight, residual=residual, Xq8=Xq8, s_x=s_x, H=H)
    _check("mq_rms_norm_quantize8", load().mq_rms_norm_quantize8(
        M, K, code, X.data_ptr(), ldx, _ptr(residual), ldr, weight.data_ptr(), eps, _ptr(H), ldh, LAYOUTS[layout],
        Xq8.data_ptr(), ldq, s_x.data_ptr(), _stream(stream)))
    return (Xq8, s_x) if residual is None else (Xq8, s_x, H)


def quantize_rows8(X, out=None, stream=None):
    """Per-token INT8 quantisation of fp16 / bf16 X [M, K] into rows: (Xq8 int8 [M, K], s_x fp32 [M])."""
    torch = _torch()
    code = _dtype_code(getattr(X, "dtype", None), "X")
    ldx = _need_rows(X, "X")
    M, K = X.shape
    if out is None:
        Xq8, ldq = _code_rows(M, K, X.device, stream)
        s_x = _empty((M,), torch.float32, X.device, stream)
    else:
        Xq8, s_x = out
        ldq = _need_codes(Xq8, K)
        if Xq8.shape[0] != M:
            raise ValueError(f"out[0] (Xq8) must have {M} rows, got {Xq8.shape[0]}")
        _need_out(s_x, (M,), torch.float32, "out[1] (s_x)")
        _same_device(X, "X", Xq8=Xq8, s_x=s_x)
    _check("mq_quantize_rows8", load().mq_quantize_rows8(M, K, code, X.data_ptr(), ldx, Xq8.data_ptr(), ldq,
                                                         s_x.data_ptr(), _stream(stream)))
    return Xq8, s_x


def dequantize_act8(Xq8, s_x, layout: str = "rows", dtype=None, out=None, stream=None):
    """The values [M, K] that INT8 codes and their scales stand for, in fp16 (or ``dtype`` bf16)."""
    torch = _torch()
    if LAYOUTS[layout] == 1:
        _need(Xq8, torch.uint8, "Xq8", 2)
        M, K, ldq = Xq8.shape[0], Xq8.shape[1] * 2 // 3, 0
        if K * 3 != Xq8.shape[1] * 2:
            raise ValueError("Xq8 is not in the A8 layout")
    else:
        ldq = _need_codes(Xq8)
        M, K = Xq8.shape
    _need(s_x, torch.float16 if LAYOUTS[layout] == 1 else torch.float32, "s_x", 1)
    if s_x.shape[0] != M:
        raise ValueError(f"s_x must have {M} values, got {s_x.shape[0]}")
    dtype = torch.float16 if dtype is None else dtype
    Y = _empty((M, K), dtype, Xq8.device, stream) if out is None else out
    code, ldy = _dtype_code(Y.dtype, "out"), _need_rows(Y, "out", K)
    if Y.shape[0] != M:
        raise ValueError(f"out must have {M} rows, got {Y.shape[0]}")
    _same_device(Xq8, "Xq8", s_x=s_x, out=Y)
    _check("mq_dequantize_act8", load().mq_dequantize_act8(M, K, LAYOUTS[layout], Xq8.data_ptr(), ldq, s_x.data_ptr(), code,
                                                           Y.data_ptr(), ldy, _stream(stream)))
    return Y


# ------------------------------------------------------- W8A8 product --
@dataclass
class PackedWeight8:
    """INT8 weight of N channels of K codes in the library layout (include/mq.h), scales fp32 [N]."""
    N: int
    K: int
    Wq: "object"          # uint8 [mq_weight8_bytes(N, K)]
    s_w: "object"         # fp32 [N]
    _of: tuple = field(default=(), repr=False, init=False, compare=False)     # what _operands found to go together

    def _operands(self):
        """Addresses of the codes and scales, which have to be those of N and K: kernels read as much of them."""
        of, Wq, s_w = self._of, self.Wq, self.s_w
        if not (of and of[0] is Wq and of[1] is s_w and of[2] == (self.N, self.K, Wq.numel(), s_w.numel())):
            torch, need = _torch(), load().mq_weight8_bytes(self.N, self.K)
            if need == 0 or self.N > _INT_MAX or self.K > _INT_MAX:
                raise ValueError(f"no INT8 weight of {self.N} channels and {self.K} codes")
            _need_out(Wq, (need,), torch.uint8, "Wq")
            _need_out(s_w, (self.N,), torch.float32, "s_w")
            _same_device(Wq, "Wq", s_w=s_w)
            self._of = (Wq, s_w, (self.N, self.K, need, self.N))
        return Wq.data_ptr(), s_w.data_ptr()

    @property
    def nbytes(self) -> int:
        return self.Wq.numel() + 4 * self.N


def _weight8(N, K, device, stream):
    nbytes = load().mq_weight8_bytes(N, K)
    if nbytes == 0 or N > _INT_MAX or K > _INT_MAX:
        raise ValueError(f"no INT8 weight of {N} channels and {K} codes")
    return _empty((nbytes,), _torch().uint8, device, stream)


def quantize_weight8(W, stream=None) -> PackedWeight8:
    """fp32 W [N, K] -> INT8 codes with a scale for each channel."""
    torch = _torch()
    _need(W, torch.float32, "W", 2)
    N, K = W.shape
    Wq, s_w = _weight8(N, K, W.device, stream), _empty((N,), torch.float32, W.device, stream)
    _check("mq_quantize_weight8", load().mq_quantize_weight8(W.data_ptr(), N, K, K, Wq.data_ptr(), s_w.data_ptr(),
                                                             _stream(stream)))
    return PackedWeight8(N, K, Wq, s_w)


def repack_weight8(Wc, s_w, stream=None) -> PackedWeight8:
    """Canonical int8 codes [N, K] and their scales fp32 [N] -> the library layout."""
    torch = _torch()
    _need(Wc, torch.int8, "Wc", 2)
    N, K = Wc.shape
    _need_out(s_w, (N,), torch.float32, "s_w")
    _same_device(Wc, "Wc", s_w=s_w)
    Wq = _weight8(N, K, Wc.device, stream)
    _check("mq_repack_weight8", load().mq_repack_weight8(N, K, Wc.data_ptr(), K, Wq.data_ptr(), _stream(stream)))
    return PackedWeight8(N, K, Wq, s_w)


def unpack_weight8(pw: PackedWeight8, stream=None):
    """Library layout -> canonical int8 codes [N, K]."""
    torch = _torch()
    Wq, _ = pw._operands()
    Wc = _empty((pw.N, pw.K), torch.int8, pw.Wq.device, stream)
    _check("mq_unpack_weight8", load().mq_unpack_weight8(pw.N, pw.K, Wq, Wc.data_ptr(), pw.K, _stream(stream)))
    return Wc


def gemm_w8a8_workspace_bytes(M: int, N: int, K: int) -> int:
    return int(load().mq_gemm_w8a8_workspace_size(M, N, K))


def gemm_w8a8_tile(M: int, N: int, K: int):
    """(rows, columns) of the output tile one workgroup takes, and the splits of K (host logic only)."""
    r, c, s = C.c_int(0), C.c_int(0), C.c_int(0)
    _check("mq_gemm_w8a8_tile", load().mq_gemm_w8a8_tile(M, N, K, C.byref(r), C.byref(c), C.byref(s)))
    return r.value, c.value, s.value


def gemm_w8a8(Xq8, s_x, pw: PackedWeight8, bias=None, out=None, out_dtype=None, workspace=None, stream=None):
    """Y [M, N] = s_x s_w (Xq8 Wq^T) + bias, in fp16 (or ``out_dtype`` bf16, fp32); bias in Y's type."""
    torch = _torch()
    ldx = _need_codes(Xq8, pw.K)
    M = Xq8.shape[0]
    Wq, s_w = pw._operands()
    _need_out(s_x, (M,), torch.float32, "s_x")
    Y = out if out is not None else _empty((M, pw.N), out_dtype or torch.float16, Xq8.device, stream)
    code, ldy = _dtype_code(Y.dtype, "out", fp32=True), _need_rows(Y, "out", pw.N)
    if Y.shape[0] != M:
        raise ValueError(f"out must have {M} rows, got {Y.shape[0]}")
    if bias is not None:
        _need_out(bias, (pw.N,), Y.dtype, "bias")
    _same_device(Xq8, "Xq8", s_x=s_x, weight=pw.Wq, bias=bias, out=Y)
    lib = load()
    ws = lib.mq_gemm_w8a8_workspace_size(M, pw.N, pw.K)
    wbuf = _scratch(ws, Xq8.device, stream, workspace)
    _check("mq_gemm_w8a8", lib.mq_gemm_w8a8(
        M, pw.N, pw.K, Xq8.data_ptr(), ldx, s_x.data_ptr(), Wq, s_w, code, _ptr(bias),
        Y.data_ptr(), ldy, _ptr(wbuf), ws, _stream(stream)))
    return Y


# -------------------------------------------------------- 4-bit cache --
class _CacheStruct(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_params", C.c_void_p), ("v_params", C.c_void_p),
                ("pages", C.c_int), ("page_size", C.c_int), ("heads", C.c_int), ("head_dim", C.c_int)]


@dataclass
class KVCache4:
    """Paged keys and values in 4 bits (include/mq.h), on the device of its tensors."""
    pages: int
    page_size: int
    heads: int
    head_dim: int
    k: "object"           # uint8 [pages, heads, page_size * head_dim / 2]
    v: "object"
    k_params: "object"    # fp16 [pages, heads, page_size, 2]: scale, minimum
    v_params: "object"
    # what the library takes (mq_kv4_cache), and the fields and addresses that it was made of
    _struct: "object" = field(default=None, repr=False, init=False, compare=False)
    _of: tuple = field(default=(), repr=False, init=False, compare=False)

    def __post_init__(self):
        self._c

    @property
    def _c(self) -> int:
        """Address of the mq_kv4_cache of the fields as they are: made anew, and they checked again, once one has been
        replaced or a tensor has other memory."""
        k, v, kp, vp = self.k, self.v, self.k_params, self.v_params
        of = self._of
        if not (of and of[0] is k and of[1] is v and of[2] is kp and of[3] is vp and of[4] == (
                k.data_ptr(), v.data_ptr(), kp.data_ptr(), vp.data_ptr(), self.pages, self.page_size, self.heads, self.head_dim)):
            torch = _torch()
            codes = (self.pages, self.heads, self.page_size * self.head_dim // 2)
            params = (self.pages, self.heads, self.page_size, 2)
            _need_out(k, codes, torch.uint8, "k")
            _need_out(v, codes, torch.uint8, "v")
            _need_out(kp, params, torch.float16, "k_params")
            _need_out(vp, params, torch.float16, "v_params")
            _same_device(k, "k", v=v, k_params=kp, v_params=vp)
            now = (k.data_ptr(), v.data_ptr(), kp.data_ptr(), vp.data_ptr(), self.pages, self.page_size, self.heads, self.head_dim)
            self._struct, self._of = _CacheStruct(*now), (k, v, kp, vp, now)
        return C.addressof(self._struct)

    def __getstate__(self):                                 # addresses mean nothing in a copy
        return {name: value for name, value in self.__dict__.items() if name not in ("_struct", "_of")}

    @property
    def nbytes(self) -> int:
        return sum(t.numel() * t.element_size() for t in (self.k, self.v, self.k_params, self.v_params))


def kv4_cache(pages: int, page_size: int, heads: int, head_dim: int, device="cuda") -> KVCache4:
    """An empty cache of ``pages`` pages of ``page_size`` tokens."""
    torch = _torch()
    if pages < 1 or heads < 1 or page_size < 16 or page_size & (page_size - 1) or page_size > 65536 or head_dim not in (64, 128):
        raise ValueError(f"no cache of {pages} pages of {page_size} tokens, {heads} heads of {head_dim}")
    codes = (pages, heads, page_size * head_dim // 2)
    return KVCache4(pages, page_size, heads, head_dim,
                    torch.zeros(codes, dtype=torch.uint8, device=device), torch.zeros(codes, dtype=torch.uint8, device=device),
                    torch.zeros((pages, heads, page_size, 2), dtype=torch.float16, device=device),
                    torch.zeros((pages, heads, page_size, 2), dtype=torch.float16, device=device))


def _need_heads(t, name, heads, head_dim, tokens=None, dtype=None):
    """[tokens, heads, head_dim] with contiguous head rows: (token stride, head stride)."""
    torch = _torch()
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA (HIP) tensor")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    shape, strides = t.shape, t.stride()
    if len(shape) != 3 or shape[1] != heads or shape[2] != head_dim or (tokens is not None and shape[0] != tokens):
        raise ValueError(f"{name} must be [{'tokens' if tokens is None else tokens}, {heads}, {head_dim}], got {tuple(shape)}")
    if shape[0] > _INT_MAX:
        raise ValueError(f"{name} must have fewer than 2^31 tokens, got {shape[0]}")
    if strides[2] != 1:
        raise ValueError(f"{name} must have contiguous rows of {head_dim}")
    # a dimension of one is never stepped along
    return (strides[0] if shape[0] > 1 else 0), (strides[1] if heads > 1 else 0)


def kv4_append(cache: KVCache4, K, V, slots, stream=None) -> None:
    """Quantises the tokens K, V [T, heads, head_dim] (fp16 or bf16, any token and head strides that are
    multiples of 8) into ``slots`` (int64 [T], distinct; those outside the cache, -1 for one, are skipped)."""
    torch = _torch()
    code = _dtype_code(getattr(K, "dtype", None), "K")
    kt, kh = _need_heads(K, "K", cache.heads, cache.head_dim)
    vt, vh = _need_heads(V, "V", cache.heads, cache.head_dim, K.shape[0], K.dtype)
    _need_out(slots, (K.shape[0],), torch.int64, "slots")
    _same_device(cache.k, "the cache", K=K, V=V, slots=slots)
    _check("mq_kv4_append", load().mq_kv4_append(cache._c, K.shape[0], code, K.data_ptr(), kt, kh, V.data_ptr(), vt, vh,
                                                 slots.data_ptr(), _stream(stream)))


def kv4_read(cache: KVCache4, slots, dtype=None, out=None, stream=None):
    """(K, V) [T, heads, head_dim], the values of the cache at ``slots`` (int64 [T]; 0 outside the cache) in
    fp16 (or ``dtype`` bf16)."""
    torch = _torch()
    _need(slots, torch.int64, "slots", 1)
    T = slots.shape[0]
    if out is None:
        shape = (T, cache.heads, cache.head_dim)
        dtype = dtype or torch.float16
        K, V = _empty(shape, dtype, slots.device, stream), _empty(shape, dtype, slots.device, stream)
    else:
        K, V = out
    code = _dtype_code(K.dtype, "K")
    kt, kh = _need_heads(K, "K", cache.heads, cache.head_dim, T)
    vt, vh = _need_heads(V, "V", cache.heads, cache.head_dim, T, K.dtype)
    _same_device(cache.k, "the cache", slots=slots, K=K, V=V)
    _check("mq_kv4_read", load().mq_kv4_read(cache._c, T, code, slots.data_ptr(), K.data_ptr(), kt, kh, V.data_ptr(), vt, vh,
                                             _stream(stream)))
    return K, V


def attention_kv4_workspace_bytes(sequences: int, tokens: int, heads: int, group: int, head_dim: int, max_q: int,
                                  max_kv: int) -> int:
    return int(load().mq_attention_kv4_workspace_size(sequences, tokens, heads, group, head_dim, max_q, max_kv))


def attention_kv4(Q, cache: KVCache4, page_table, kv_lens, cu_q=None, max_q=None, max_kv=None, scale=None,
                  causal: bool = True, out=None, workspace=None, stream=None):
    """Attention of Q [tokens, query heads, head_dim] (fp16 or bf16) over the cache: O of Q's shape and type.

    Sequence b holds kv_lens[b] (int32) tokens in the pages page_table[b] (int32 [sequences, pages]); its
    queries are rows cu_q[b] .. cu_q[b + 1] (int32 [sequences + 1]) of Q and stand, if ``causal``, at its end.
    Without ``cu_q`` each sequence has one query.  ``max_q`` and ``max_kv`` bound the queries and tokens of a
    sequence (tighter bounds, faster launches; by default all rows of Q and all of the table).
    ``scale``: 1 / sqrt(head_dim) by default."""
    torch = _torch()
    D, heads = cache.head_dim, cache.heads
    code = _dtype_code(getattr(Q, "dtype", None), "Q")
    if Q.dim() != 3 or Q.shape[1] == 0 or Q.shape[1] % heads:
        raise ValueError(f"Q must be [tokens, a multiple of {heads} heads, {D}], got {tuple(Q.shape)}")
    T, Hq = Q.shape[0], Q.shape[1]
    qt, qh = _need_heads(Q, "Q", Hq, D)
    _need(page_table, torch.int32, "page_table", 2)
    B, table_pages = page_table.shape
    _need_out(kv_lens, (B,), torch.int32, "kv_lens")
    if cu_q is not None:
        _need_out(cu_q, (B + 1,), torch.int32, "cu_q")
        max_q = T if max_q is None else max_q
        _need_max_q(max_q)
    else:
        if T != B:
            raise ValueError(f"without cu_q, Q has one row for each of the {B} sequences; got {T}")
        max_q = 1
    most = table_pages * cache.page_size
    max_kv = most if max_kv is None else max_kv
    if max_kv > most:
        raise ValueError(f"max_kv {max_kv} is more than the page table's {most} tokens")
    O = _empty((T, Hq, D), Q.dtype, Q.device, stream) if out is None else out
    ot, oh = _need_heads(O, "out", Hq, D, T, Q.dtype)
    _same_device(cache.k, "the cache", Q=Q, page_table=page_table, kv_lens=kv_lens, cu_q=cu_q, out=O)
    lib, group = load(), Hq // heads
    ws = lib.mq_attention_kv4_workspace_size(B, T, heads, group, D, max_q, max_kv)
    wbuf = _scratch(ws, Q.device, stream, workspace)
    _check("mq_attention_kv4", lib.mq_attention_kv4(
        cache._c, B, T, group, max_q, max_kv, code, Q.data_ptr(), qt, qh, page_table.data_ptr(), table_pages,
        kv_lens.data_ptr(), _ptr(cu_q), 1.0 / math.sqrt(D) if scale is None else scale, causal, O.data_ptr(), ot, oh,
        _ptr(wbuf), ws, _stream(stream)))
    return O
