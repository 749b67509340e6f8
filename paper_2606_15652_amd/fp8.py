"""Binding of the operators in 8-bit floating point (OCP e4m3): the product with scales for blocks of 128, the paged
8-bit cache and the attention over it; and of sampling.

As in the package's other calls only arguments are checked and marshalled here; ``include/mq.h`` documents each
operator.  Values are fp16 or bf16.  A call runs on the device of its tensors, which need not be the current one,
on ``stream`` or that device's current stream.
"""
from __future__ import annotations

import ctypes as C
import math
from contextlib import nullcontext
from dataclasses import dataclass, field

from . import _check, _empty, _need, _need_out, _ptr, _scratch, _stream, _torch, load
from .serving import _INT_MAX, _dtype_code, _need_heads, _need_max_q, _need_rows, _same_device

_no_guard = nullcontext()


def _on(t, stream):
    """The context in which a launch goes to the device of ``t``; a stream has to be that device's."""
    torch = _torch()
    device = t.get_device()
    if stream is not None and stream.device_index != device:
        raise ValueError(f"the stream is of cuda:{stream.device_index}, the tensors are on cuda:{device}")
    return _no_guard if torch._C._cuda_getDevice() == device else torch.cuda.device(device)


# ----------------------------------------------------- block-scaled product --
def _groups(K):
    return -(-K // 128)


def _need_codes_fp8(Xq, K=None):
    """e4m3 rows as the kernels take them: their stride in bytes.  The bytes up to the next multiple of 16 after a row's
    last code have to be there too, and must not be NaN codes (0x7F, 0xFF): products read them."""
    torch = _torch()
    ld = _need_rows(Xq, "Xq", K)
    if Xq.dtype != torch.float8_e4m3fn:
        raise TypeError(f"Xq must be torch.float8_e4m3fn, got {Xq.dtype}")
    M, K = Xq.shape
    padded = -(-K // 16) * 16
    if M <= 1:
        ld = padded                             # one row: its stride says nothing
    if ld < padded or ld % 16:
        raise ValueError(f"Xq's rows must start every multiple of 16 bytes, at least {padded}; got a row stride of {ld}")
    if padded != K and M and Xq.storage_offset() + (M - 1) * ld + padded > Xq.untyped_storage().nbytes():
        raise ValueError("Xq's last row must be followed by its padding to 16 bytes")
    return ld


def _need_scales(s_x, M, K):
    """fp32 [M, groups] with the tokens next to each other: the stride of the groups."""
    torch = _torch()
    if not isinstance(s_x, torch.Tensor) or not s_x.is_cuda or s_x.dtype != torch.float32:
        raise TypeError("s_x must be an fp32 CUDA (HIP) tensor")
    if tuple(s_x.shape) != (M, _groups(K)):
        raise ValueError(f"s_x must be [{M}, {_groups(K)}], got {tuple(s_x.shape)}")
    token, group = s_x.stride()
    if (token != 1 and M > 1) or (group < M and s_x.shape[1] > 1):
        raise ValueError("s_x must have the tokens of a group next to each other (strides 1, at least the tokens)")
    if s_x.shape[1] == 1:
        return M
    if group > _INT_MAX:
        raise ValueError(f"s_x's groups must be less than 2^31 apart, got {group}")
    return group


def quantize_rows_fp8(X, out=None, stream=None):
    """Quantisation of fp16 / bf16 X [M, K] to e4m3 with a scale for each token and 128 channels: (Xq float8_e4m3fn [M, K]
    with padded rows, s_x fp32 [M, ceil(K / 128)], the tokens of a group next to each other)."""
    torch = _torch()
    code = _dtype_code(getattr(X, "dtype", None), "X")
    ldx = _need_rows(X, "X")
    M, K = X.shape
    if out is None:
        ldq = -(-K // 16) * 16
        rows = _empty((M, ldq), torch.float8_e4m3fn, X.device, stream)
        Xq, s_x = (rows if ldq == K else rows[:, :K]), _empty((_groups(K), M), torch.float32, X.device, stream).t()
        lds = M
    else:
        Xq, s_x = out
        ldq, lds = _need_codes_fp8(Xq, K), _need_scales(s_x, M, K)
        if Xq.shape[0] != M:
            raise ValueError(f"out[0] (Xq) must have {M} rows, got {Xq.shape[0]}")
        _same_device(X, "X", Xq=Xq, s_x=s_x)
    with _on(X, stream):
        _check("mq_quantize_rows_fp8", load().mq_quantize_rows_fp8(M, K, code, X.data_ptr(), ldx, Xq.data_ptr(), ldq, s_x.data_ptr(), lds,
                                                                   _stream(stream)))
    return Xq, s_x


@dataclass
class PackedWeightFP8:
    """e4m3 weight of N channels of K codes in the library layout (include/mq.h), a scale for each block of 128 x 128."""
    N: int
    K: int
    Wq: "object"          # uint8 [mq_weight_fp8_bytes(N, K)]
    s_w: "object"         # fp32 [ceil(N / 128), ceil(K / 128)]
    _of: tuple = field(default=(), repr=False, init=False, compare=False)     # what _operands found to go together

    def _operands(self):
        """Addresses of the codes and scales, which have to be those of N and K: kernels read as much of them."""
        of, Wq, s_w = self._of, self.Wq, self.s_w
        if not (of and of[0] is Wq and of[1] is s_w and of[2] == (self.N, self.K, Wq.numel(), s_w.numel())):
            torch, need = _torch(), load().mq_weight_fp8_bytes(self.N, self.K)
            if need == 0 or self.N > _INT_MAX or self.K > _INT_MAX:
                raise ValueError(f"no e4m3 weight of {self.N} channels and {self.K} codes")
            _need_out(Wq, (need,), torch.uint8, "Wq")
            _need_out(s_w, (_groups(self.N), _groups(self.K)), torch.float32, "s_w")
            _same_device(Wq, "Wq", s_w=s_w)
            self._of = (Wq, s_w, (self.N, self.K, need, s_w.numel()))
        return Wq.data_ptr(), s_w.data_ptr()

    @property
    def nbytes(self) -> int:
        return self.Wq.numel() + 4 * self.s_w.numel()


def _weight_fp8(N, K, device, stream):
    nbytes = load().mq_weight_fp8_bytes(N, K)
    if nbytes == 0 or N > _INT_MAX or K > _INT_MAX:
        raise ValueError(f"no e4m3 weight of {N} channels and {K} codes")
    return _empty((nbytes,), _torch().uint8, device, stream)


def quantize_weight_fp8(W, stream=None) -> PackedWeightFP8:
    """fp32 W [N, K] -> e4m3 codes with a scale for each block of 128 x 128."""
    torch = _torch()
    _need(W, torch.float32, "W", 2)
    N, K = W.shape
    Wq = _weight_fp8(N, K, W.device, stream)
    s_w = _empty((_groups(N), _groups(K)), torch.float32, W.device, stream)
    with _on(W, stream):
        _check("mq_quantize_weight_fp8", load().mq_quantize_weight_fp8(W.data_ptr(), N, K, K, Wq.data_ptr(), s_w.data_ptr(),
                                                                       _stream(stream)))
    return PackedWeightFP8(N, K, Wq, s_w)


def repack_weight_fp8(Wc, s_w, stream=None) -> PackedWeightFP8:
    """Canonical codes float8_e4m3fn [N, K] and their scales fp32 [ceil(N / 128), ceil(K / 128)] -> the library layout."""
    torch = _torch()
    _need(Wc, torch.float8_e4m3fn, "Wc", 2)
    N, K = Wc.shape
    _need_out(s_w, (_groups(N), _groups(K)), torch.float32, "s_w")
    _same_device(Wc, "Wc", s_w=s_w)
    Wq = _weight_fp8(N, K, Wc.device, stream)
    with _on(Wc, stream):
        _check("mq_repack_weight_fp8", load().mq_repack_weight_fp8(N, K, Wc.data_ptr(), K, Wq.data_ptr(), _stream(stream)))
    return PackedWeightFP8(N, K, Wq, s_w)


def unpack_weight_fp8(pw: PackedWeightFP8, stream=None):
    """Library layout -> canonical codes float8_e4m3fn [N, K]."""
    torch = _torch()
    Wq, _ = pw._operands()
    Wc = _empty((pw.N, pw.K), torch.float8_e4m3fn, pw.Wq.device, stream)
    with _on(Wc, stream):
        _check("mq_unpack_weight_fp8", load().mq_unpack_weight_fp8(pw.N, pw.K, Wq, Wc.data_ptr(), pw.K, _stream(stream)))
    return Wc


def gemm_fp8_workspace_bytes(M: int, N: int, K: int) -> int:
    return int(load().mq_gemm_fp8_workspace_size(M, N, K))


def gemm_fp8_tile(M: int, N: int, K: int):
    """(rows, columns) of the output tile one workgroup takes, and the splits of K (host logic only)."""
    r, c, s = C.c_int(0), C.c_int(0), C.c_int(0)
    _check("mq_gemm_fp8_tile", load().mq_gemm_fp8_tile(M, N, K, C.byref(r), C.byref(c), C.byref(s)))
    return r.value, c.value, s.value


def gemm_fp8(Xq, s_x, pw: PackedWeightFP8, bias=None, out=None, out_dtype=None, workspace=None, stream=None):
    """Y [M, N] = sum over groups of s_x s_w (Xq Wq^T) + bias, in fp16 (or ``out_dtype`` bf16, fp32); bias in Y's type.
    Rows whose K is no multiple of 16 are followed by their padding to 16 bytes, which must not hold NaN codes (as memory that was never
    written may): ``quantize_rows_fp8`` clears it, a program that makes codes itself does."""
    torch = _torch()
    ldx = _need_codes_fp8(Xq, pw.K)
    M = Xq.shape[0]
    Wq, s_w = pw._operands()
    lds = _need_scales(s_x, M, pw.K)
    Y = out if out is not None else _empty((M, pw.N), out_dtype or torch.float16, Xq.device, stream)
    code, ldy = _dtype_code(Y.dtype, "out", fp32=True), _need_rows(Y, "out", pw.N)
    if Y.shape[0] != M:
        raise ValueError(f"out must have {M} rows, got {Y.shape[0]}")
    if bias is not None:
        _need_out(bias, (pw.N,), Y.dtype, "bias")
    _same_device(Xq, "Xq", s_x=s_x, weight=pw.Wq, bias=bias, out=Y, workspace=workspace)
    lib = load()
    ws = lib.mq_gemm_fp8_workspace_size(M, pw.N, pw.K)
    with _on(Xq, stream):
        wbuf = _scratch(ws, Xq.device, stream, workspace)
        _check("mq_gemm_fp8", lib.mq_gemm_fp8(M, pw.N, pw.K, Xq.data_ptr(), ldx, s_x.data_ptr(), lds, Wq, s_w, code, _ptr(bias),
                                              Y.data_ptr(), ldy, _ptr(wbuf), ws, _stream(stream)))
    return Y


# -------------------------------------------------------- 8-bit cache --
class _CacheStruct8(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_scales", C.c_void_p), ("v_scales", C.c_void_p),
                ("pages", C.c_int), ("page_size", C.c_int), ("heads", C.c_int), ("head_dim", C.c_int)]


@dataclass
class KVCache8:
    """Paged keys and values in e4m3, a scale for each 32 tokens and head (include/mq.h), on the device of its tensors."""
    pages: int
    page_size: int
    heads: int
    head_dim: int
    k: "object"           # uint8 [pages, heads, page_size * head_dim]
    v: "object"
    k_scales: "object"    # uint8 [pages, heads, page_size / 32]: exponents + 127
    v_scales: "object"
    # what the library takes (mq_kv8_cache), and the fields and addresses that it was made of
    _struct: "object" = field(default=None, repr=False, init=False, compare=False)
    _of: tuple = field(default=(), repr=False, init=False, compare=False)

    def __post_init__(self):
        self._c

    @property
    def _c(self) -> int:
        """Address of the mq_kv8_cache of the fields as they are: made anew, and they checked again, once one has been
        replaced or a tensor has other memory."""
        k, v, ks, vs = self.k, self.v, self.k_scales, self.v_scales
        of = self._of
        if not (of and of[0] is k and of[1] is v and of[2] is ks and of[3] is vs and of[4] == (
                k.data_ptr(), v.data_ptr(), ks.data_ptr(), vs.data_ptr(), self.pages, self.page_size, self.heads, self.head_dim)):
            torch = _torch()
            codes = (self.pages, self.heads, self.page_size * self.head_dim)
            scales = (self.pages, self.heads, self.page_size // 32)
            _need_out(k, codes, torch.uint8, "k")
            _need_out(v, codes, torch.uint8, "v")
            _need_out(ks, scales, torch.uint8, "k_scales")
            _need_out(vs, scales, torch.uint8, "v_scales")
            _same_device(k, "k", v=v, k_scales=ks, v_scales=vs)
            now = (k.data_ptr(), v.data_ptr(), ks.data_ptr(), vs.data_ptr(), self.pages, self.page_size, self.heads, self.head_dim)
            self._struct, self._of = _CacheStruct8(*now), (k, v, ks, vs, now)
        return C.addressof(self._struct)

    def __getstate__(self):                                 # addresses mean nothing in a copy
        return {name: value for name, value in self.__dict__.items() if name not in ("_struct", "_of")}

    @property
    def nbytes(self) -> int:
        return sum(t.numel() for t in (self.k, self.v, self.k_scales, self.v_scales))


def kv8_cache(pages: int, page_size: int, heads: int, head_dim: int, device="cuda") -> KVCache8:
    """An empty cache of ``pages`` pages of ``page_size`` tokens."""
    torch = _torch()
    if pages < 1 or heads < 1 or page_size < 32 or page_size & (page_size - 1) or page_size > 65536 or head_dim not in (64, 128):
        raise ValueError(f"no cache of {pages} pages of {page_size} tokens, {heads} heads of {head_dim}")

    def zeros(*shape):
        return torch.zeros((pages, heads, *shape), dtype=torch.uint8, device=device)
    return KVCache8(pages, page_size, heads, head_dim, zeros(page_size * head_dim), zeros(page_size * head_dim),
                    zeros(page_size // 32), zeros(page_size // 32))


def kv8_append(cache: KVCache8, K, V, page_table, kv_lens, cu_new=None, stream=None) -> None:
    """Quantises the tokens K, V [T, heads, head_dim] (fp16 or bf16, any token and head strides that are multiples of 8)
    into the ends of sequences: sequence b has kv_lens[b] (int32) tokens with them, in the pages page_table[b] (int32
    [sequences, pages]), and rows cu_new[b] .. cu_new[b + 1] (int32 [sequences + 1]) are its last ones.  Without
    ``cu_new`` each sequence has one new token.  A block of 32 tokens whose scale changes is coded anew; sequences may
    have been shortened since they were written."""
    torch = _torch()
    code = _dtype_code(getattr(K, "dtype", None), "K")
    kt, kh = _need_heads(K, "K", cache.heads, cache.head_dim)
    T = K.shape[0]
    vt, vh = _need_heads(V, "V", cache.heads, cache.head_dim, T, K.dtype)
    _need(page_table, torch.int32, "page_table", 2)
    B, table_pages = page_table.shape
    _need_out(kv_lens, (B,), torch.int32, "kv_lens")
    if cu_new is not None:
        _need_out(cu_new, (B + 1,), torch.int32, "cu_new")
    elif T != B:
        raise ValueError(f"without cu_new, K has one row for each of the {B} sequences; got {T}")
    c = cache._c
    _same_device(cache.k, "the cache", K=K, V=V, page_table=page_table, kv_lens=kv_lens, cu_new=cu_new)
    with _on(K, stream):
        _check("mq_kv8_append", load().mq_kv8_append(c, B, T, code, K.data_ptr(), kt, kh, V.data_ptr(), vt, vh, page_table.data_ptr(),
                                                     table_pages, kv_lens.data_ptr(), _ptr(cu_new), _stream(stream)))


def kv8_read(cache: KVCache8, slots, dtype=None, out=None, stream=None):
    """(K, V) [T, heads, head_dim], the values of the cache at ``slots`` (int64 [T], page * page_size + place; 0 outside
    the cache) in fp16 (or ``dtype`` bf16)."""
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
    c = cache._c
    _same_device(cache.k, "the cache", slots=slots, K=K, V=V)
    with _on(slots, stream):
        _check("mq_kv8_read", load().mq_kv8_read(c, T, code, slots.data_ptr(), K.data_ptr(), kt, kh, V.data_ptr(), vt, vh,
                                                 _stream(stream)))
    return K, V


def attention_kv8_workspace_bytes(sequences: int, tokens: int, heads: int, group: int, head_dim: int, max_q: int,
                                  max_kv: int) -> int:
    return int(load().mq_attention_kv8_workspace_size(sequences, tokens, heads, group, head_dim, max_q, max_kv))


def attention_kv8(Q, cache: KVCache8, page_table, kv_lens, cu_q=None, max_q=None, max_kv=None, scale=None,
                  causal: bool = True, out=None, workspace=None, stream=None):
    """Attention of Q [tokens, query heads, head_dim] (fp16 or bf16) over the cache: O of Q's shape and type.
    Arguments as of ``attention_kv4``."""
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
    c = cache._c
    _same_device(cache.k, "the cache", Q=Q, page_table=page_table, kv_lens=kv_lens, cu_q=cu_q, out=O, workspace=workspace)
    lib, group = load(), Hq // heads
    ws = lib.mq_attention_kv8_workspace_size(B, T, heads, group, D, max_q, max_kv)
    with _on(Q, stream):
        wbuf = _scratch(ws, Q.device, stream, workspace)
        _check("mq_attention_kv8", lib.mq_attention_kv8(
            c, B, T, group, max_q, max_kv, code, Q.data_ptr(), qt, qh, page_table.data_ptr(), table_pages, kv_lens.data_ptr(),
            _ptr(cu_q), 1.0 / math.sqrt(D) if scale is None else scale, causal, O.data_ptr(), ot, oh, _ptr(wbuf), ws,
            _stream(stream)))
    return O


# ----------------------------------------------------------- sampling --
def _of_rows(value, rows, dtype, name, none, device):
    """A parameter for each row (a tensor) or for all: (tensor or None, number)."""
    if value is None:
        return None, none
    if isinstance(value, _torch().Tensor):
        _need_out(value, (rows,), dtype, name)
        if value.get_device() != device:
            raise ValueError(f"{name} is on {value.device}, logits on cuda:{device}")
        return value, none
    return None, value


def sample(logits, u, temperature=1.0, top_k=None, top_p=None, min_p=None, out=None, stream=None):
    """(tokens int64 [rows], probabilities fp32 [rows]): a token drawn from each row of logits [rows, vocab] (fp16, bf16 or
    fp32, contiguous rows) by the uniform numbers ``u`` (fp32 [rows], in [0, 1)).  ``temperature``, ``top_k``, ``top_p`` and
    ``min_p`` filter in this order (include/mq.h); each is a number for all rows or a tensor [rows] (fp32, top_k
    int32), None for none.  Temperature 0 takes the largest logit."""
    torch = _torch()
    code = _dtype_code(getattr(logits, "dtype", None), "logits", fp32=True)
    if not logits.is_cuda or logits.dim() != 2:
        raise ValueError("logits must be a CUDA (HIP) tensor [rows, vocab]")
    rows, vocab = logits.shape
    ldx, col = logits.stride()
    if col != 1 and vocab > 1:
        raise ValueError("logits must have contiguous rows")
    if rows > _INT_MAX or vocab > _INT_MAX:
        raise ValueError(f"logits must have fewer than 2^31 rows and columns, got {tuple(logits.shape)}")
    device = logits.get_device()
    _need_out(u, (rows,), torch.float32, "u")
    t, t1 = _of_rows(temperature, rows, torch.float32, "temperature", 1.0, device)
    k, k1 = _of_rows(top_k, rows, torch.int32, "top_k", 0, device)
    p, p1 = _of_rows(top_p, rows, torch.float32, "top_p", 1.0, device)
    m, m1 = _of_rows(min_p, rows, torch.float32, "min_p", 0.0, device)
    if not -(1 << 31) <= k1 < 1 << 31:
        raise ValueError(f"top_k {k1} is out of range")
    if out is None:
        tokens, probs = _empty((rows,), torch.int64, logits.device, stream), _empty((rows,), torch.float32, logits.device, stream)
    else:
        tokens, probs = out
        _need_out(tokens, (rows,), torch.int64, "out[0] (tokens)")
        _need_out(probs, (rows,), torch.float32, "out[1] (probs)")
    _same_device(logits, "logits", u=u, tokens=tokens, probs=probs)
    with _on(logits, stream):
        _check("mq_sample", load().mq_sample(rows, vocab, code, logits.data_ptr(), ldx if rows > 1 else vocab, u.data_ptr(), _ptr(t), t1,
                                             _ptr(k), k1, _ptr(p), p1, _ptr(m), m1, tokens.data_ptr(), probs.data_ptr(), _stream(stream)))
    return tokens, probs
