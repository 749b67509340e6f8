"""Plain implementations, in 64 bits, of the operators around the layers (norm with 8-bit output,
8-bit product, 4-bit cache and the attention over it), and the inputs that their tests share.
CPU tensors in, CPU tensors out."""
import math

import torch

UNIT = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}   # half a step of the last place
TINY = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -133, torch.float32: 0.0}        # half the smallest number


def generator(*seed):
    g = torch.Generator()
    g.manual_seed(hash(seed) % (1 << 31))
    return g


def acts(M, K, dtype, seed, spread=1.0):
    """Rows with a few large channels."""
    g = generator(M, K, seed)
    x = torch.randn(M, K, generator=g) * spread
    x[:, torch.randint(0, K, (4,), generator=g)] *= 30.0
    return x.to(dtype)


# ------------------------------------------------------------------- norm --
def norm(x, gamma, eps, r=None):
    """(h in x's type, y in 64 bits)"""
    h = x if r is None else (x.float() + r.float()).to(x.dtype)
    d = h.double()
    return h, d * gamma.double() / torch.sqrt((d * d).mean(-1, keepdim=True) + eps)


# ------------------------------------------------------------------ cache --
def quantise4(x):
    """Codes (int64), scales and minima (fp32 tensors of fp16 values) of rows along the last dimension;
    the definition is in fp32."""
    x = x.float()
    finite = torch.isfinite(x).all(-1, keepdim=True)
    z = x.amin(-1, keepdim=True).half().float()
    s = ((x.amax(-1, keepdim=True) - z) / 15).half().float()
    ok = finite & torch.isfinite(z) & torch.isfinite(s)
    n = torch.where(ok & (s > 0), ((x - z) / s).round().clamp(0, 15), torch.zeros_like(x))
    nan = torch.full_like(z, math.nan)
    return n.long(), torch.where(ok, s, nan), torch.where(ok, z, nan)


def values4(x):
    n, s, z = quantise4(x)
    return z.double() + s.double() * n.double()


# -------------------------------------------------------------- attention --
def attention(q, k, v, scale, causal):
    """One sequence: q [nq, Hq, D], k and v [n, H, D] in 64 bits (NaN rows allowed) -> [nq, Hq, D]."""
    nq, hq, _ = q.shape
    n, h, _ = k.shape
    q, g = q.double(), hq // h
    out = torch.zeros_like(q)
    for i in range(nq):
        seen = max(0, min(n, n - nq + i + 1)) if causal else n
        if seen == 0:
            continue
        for j in range(hq):
            w = torch.softmax(scale * (k[:seen, j // g] @ q[i, j]), 0)
            out[i, j] = w @ v[:seen, j // g]
    return out


def attention_error(q, k, v, scale, dtype, o):
    """A bound of the kernel's error for one sequence, from its roundings:
    weights in fp16 (half a step of 2^-11, relative) times the code's part of the values, at most 15 s;
    weights below fp16's normal range (2^-25 of twice the largest scale, each of n, under a weight sum of
    at least one); scores in fp32 after D products, whose error turns into a relative one of the weights;
    the result's own rounding."""
    n, d = k.shape[0], k.shape[2]
    fin = torch.nan_to_num(v)
    spread = (fin.amax(-1) - fin.amin(-1)).max().item() if n else 0.0
    size = fin.abs().max().item() if n else 0.0
    mass = (q.double().abs().sum(-1).max() * torch.nan_to_num(k).abs().max()).item() * scale if n else 0.0
    score = (d + 8) * 2.0 ** -24 * mass * 2
    return (2.0 ** -11 + 2 * n * 2.0 ** -25) * spread * 1.01 + 2 * score * size + 2.0 ** -22 * size + UNIT[dtype] * o.abs() * 1.01 + TINY[dtype]


class Sequences:
    """Ragged sequences in a paged cache: per-sequence keys and values, a page table with the pages in
    random order, and the slots of every token."""

    def __init__(self, lens, heads, dim, page, dtype, seed, spread=1.0, most=None):
        g = generator(tuple(lens), heads, dim, page, seed)
        counts = [-(-n // page) for n in lens]
        self.pages, self.page, self.lens = sum(counts) + 2, page, lens
        order = torch.randperm(self.pages, generator=g)
        self.table = torch.full((len(lens), most or max(1, max(counts))), -1, dtype=torch.int32)
        self.k, self.v, self.slots, at = [], [], [], 0
        for b, (n, c) in enumerate(zip(lens, counts)):
            self.table[b, :c] = order[at:at + c].int()
            at += c
            t = torch.arange(n)
            self.slots.append(self.table[b, t // page].long() * page + t % page)
            k = torch.randn(n, heads, dim, generator=g) * spread
            k[..., ::16] += 3.0
            self.k.append(k.to(dtype))
            self.v.append((torch.randn(n, heads, dim, generator=g) * spread).to(dtype))
        self.kv_lens = torch.tensor(lens, dtype=torch.int32)
