"""Binding of the operators in 8-bit floating point (OCP e4m3), the paged 8-bit cache and the attention over it, and of
sampling.

As in the package's other calls only arguments are checked and marshalled here; ``include/mq.h`` documents each
operator.  Values are fp16 or bf16.  A call runs on the device of its tensors, which need not be the current one,
on ``stream`` or that device's current stream.
"""
from __future__ import annotations

import ctypes as C
import math
from contextlib import nullcontext
from dataclasses import dataclass, field

from . import _check, _need, _need_out, _ptr, _scratch, _stream, _torch, load
from .serving import _dtype_code, _empty, _need_heads, _same_device

_no_guard = nullcontext()


def _on(t, stream):
    """The context in which a launch goes to the device of ``t``; a stream has to be that device's."""
    torch = _torch()
    device = t.get_device()
    if stream is not None and stream.device_index != device:
        raise ValueError(f"the stream is of cuda:{stream.device_index}, the tensors are on cuda:{device}")
    return _no_guard if torch._C._cuda_getDevice() == device else torch.cuda.device(device)


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
    ``cu_new`` each sequence has one new token.  A block of 32 tokens whose scale grows is coded anew."""
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


def sample(logits, u, temperature=1.0, top_k=None, top_p=None, min_p=None, out=None, workspace=None, stream=None):
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
    _same_device(logits, "logits", u=u, tokens=tokens, probs=probs, workspace=workspace)
    lib = load()
    ws = lib.mq_sample_workspace_size(rows, vocab)
    with _on(logits, stream):
        wbuf = _scratch(ws, logits.device, stream, workspace)
        _check("mq_sample", lib.mq_sample(rows, vocab, code, logits.data_ptr(), ldx if rows > 1 else vocab, u.data_ptr(), _ptr(t), t1,
                                          _ptr(k), k1, _ptr(p), p1, _ptr(m), m1, tokens.data_ptr(), probs.data_ptr(), _ptr(wbuf), ws,
                                          _stream(stream)))
    return tokens, probs
