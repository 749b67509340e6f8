"""Plain implementations, in 64 bits, of the operators in 8-bit floating point, and the inputs that their tests share.
CPU tensors in, CPU tensors out."""
import math

import torch

from serving_oracle import TINY, UNIT, generator

BLOCK = 32
MOST = 448.0


def round8(x):
    """The e4m3 value nearest to x (64 bits, |x| <= 448), of two the one with an even last digit."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return (x / step).round() * step


def byte8(x):
    """The byte of an e4m3 value (NaN: 0x7F), from the format: sign, four bits of exponent + 7, three of fraction."""
    a = torch.nan_to_num(x).abs()
    e = torch.floor(torch.log2(a.clamp(min=2.0 ** -6)))
    normal = a >= 2.0 ** -6
    frac = torch.where(normal, a / torch.exp2(e) - 1, a / 2.0 ** -6) * 8
    code = torch.where(normal, (e + 7) * 8, torch.zeros_like(a)) + frac
    code = torch.where(torch.isnan(x), torch.full_like(a, 127.0), code) + 128 * (torch.signbit(x) & ~torch.isnan(x))
    return code.to(torch.uint8)


def exponent(amax):
    """Least whole e >= -127 with amax <= 448 2^e (64 bits)."""
    e = torch.full_like(amax, -127.0)
    for i in range(-126, 122):
        e = torch.where(amax > MOST * 2.0 ** (i - 1), torch.full_like(e, float(i)), e)
    return e


class Rows8:
    """What one sequence's cache holds for keys and values: codes' values [n, H, D] and exponents [blocks, H]."""

    def __init__(self, heads, dim):
        self.n = [torch.zeros(0, heads, dim, dtype=torch.float64) for _ in range(2)]
        self.e = [torch.zeros(0, heads, dtype=torch.float64) for _ in range(2)]

    def append(self, k, v):
        k, v = k.double(), v.double()
        fine = torch.isfinite(k).all(-1) & torch.isfinite(v).all(-1)
        had = self.n[0].shape[0]
        for w, x in enumerate((k, v)):
            x = torch.where(fine[..., None], x, torch.zeros_like(x))
            rows, exps, at, done = [self.n[w][:had // BLOCK * BLOCK]], [self.e[w][:had // BLOCK]], had // BLOCK * BLOCK, 0
            while done < x.shape[0]:
                old = self.n[w][at:had] if at < had else x[:0]
                new = x[done:done + BLOCK - old.shape[0]]
                ok = fine[done:done + new.shape[0]]
                e = exponent(new.abs().amax((0, 2)))
                if old.shape[0]:
                    was = self.e[w][at // BLOCK]
                    e = torch.maximum(e, was)
                    # a NaN key stays one
                    old = torch.where(torch.isnan(old), old, round8(torch.nan_to_num(old) * torch.exp2(was - e)[:, None]))
                codes = round8(new * torch.exp2(-e)[:, None])
                codes = torch.where(ok[..., None], codes, torch.full_like(codes, math.nan if w == 0 else 0.0))
                rows += [old, codes]
                exps.append(e[None])
                done += new.shape[0]
                at += BLOCK
            if x.shape[0]:
                self.n[w], self.e[w] = torch.cat(rows), torch.cat(exps)
        return self

    def values(self):
        return [n * torch.exp2(e).repeat_interleave(BLOCK, 0)[:n.shape[0], :, None] for n, e in zip(self.n, self.e)]


def table_of(lens, page, seed, most=None, spare=2):
    """A page table with the pages in random order, unused entries -1, and how many pages there are."""
    counts = [-(-n // page) for n in lens]
    pages = sum(counts) + spare
    order = torch.randperm(pages, generator=generator(tuple(lens), page, seed))
    table = torch.full((len(lens), most or max(1, max(counts, default=1))), -1, dtype=torch.int32)
    at = 0
    for b, c in enumerate(counts):
        table[b, :c] = order[at:at + c].int()
        at += c
    return table, pages


def slots_of(table, b, first, last, page):
    t = torch.arange(first, last)
    return table[b, t // page].long() * page + t % page


def starts(counts):
    return torch.tensor([0, *counts]).cumsum(0).int()


def attention_error(q, k, v, n8, scale, dtype, o, ev):
    """A bound of the attention's error for one sequence (all queries see at least one token), from its roundings.
    n8: the values' codes, ev their exponents by token [n, H]:
    each weight in fp16, half a step of 2^-11 relative (fp16 calls: twice, 2^-22 and a little for the first rest's own), or
    2^-25 where it is below fp16's normal range, the largest product of weight and scale being at least 2^6 there;
    scores in fp32: D products, their scaling and the exponential, whose error is a relative one of the weight above
    and below; sums of n in fp32; the result's own rounding."""
    n, _, d = k.shape
    fin = torch.nan_to_num(v)
    size = fin.abs().max().item()
    mass = (q.double().abs().sum(-1).max() * torch.nan_to_num(k).abs().max()).item() * scale
    score = (d + 8) * 2.0 ** -24 * mass + 2.0 ** -22
    lost = n * torch.nan_to_num(n8).abs().max().item() * 2.0 ** -25 * 2.0 ** -6 * torch.exp2(ev).max().item()
    return ((2.0 ** -11 if dtype == torch.bfloat16 else 2.0 ** -21) * 1.01 + 2 * score + 2 * (n + 8) * 2.0 ** -24) * size + lost + UNIT[dtype] * o.abs() * 1.01 + TINY[dtype]
