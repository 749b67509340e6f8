"""The paged 8-bit cache after a sequence has been shortened: tokens that were taken back leave nothing, their scales included."""
import math

import pytest
import torch

import fp8_oracle as fo
from test_gpu_kv8 import HALF, Both, mq, rows

pytestmark = pytest.mark.gpu


class Shortened(fo.Rows8):
    """The definition, for sequences that get shorter between two appends."""

    def shorten(self, m):
        for w in range(2):
            self.n[w], self.e[w] = self.n[w][:m], self.e[w][:-(-m // fo.BLOCK)]

    def append(self, k, v):
        had = self.n[0].shape[0]
        at = had // fo.BLOCK * fo.BLOCK
        if k.shape[0] and at < had:
            for w in range(2):
                n, e = self.n[w][at:].clone(), self.e[w][at // fo.BLOCK].clone()
                for h in range(n.shape[1]):
                    big = torch.nan_to_num(n[:, h]).abs().max()
                    if big < 224:                                   # no token that is left needs the scale
                        least = -127.0 if big == 0 else max(-127.0, float(fo.exponent(big * 2.0 ** e[h])))
                        n[:, h] *= 2.0 ** (e[h] - least)
                        e[h] = least
                self.n[w] = torch.cat((self.n[w][:at], n))
                self.e[w] = torch.cat((self.e[w][:at // fo.BLOCK], e[None]))
        return super().append(k, v)


def both(most, page, heads, dim):
    t = Both(most, page, heads, dim)
    t.want = [Shortened(heads, dim) for _ in most]
    return t


def shorten(t, lens):
    t.lens = list(lens)
    for w, n in zip(t.want, lens):
        w.shorten(n)


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("big", [2.0, 60.0, 3e3])
def test_tokens_taken_back(dtype, dim, big):
    """Small tokens, larger ones that are taken back, small ones again: each has the scale of those that are there."""
    heads = 3
    t = both([120, 120, 120, 120], 64, heads, dim)
    t.append([rows(n, heads, dim, dtype, i) for i, n in enumerate([5, 17, 40, 64])])
    t.append([rows(n, heads, dim, dtype, 10 + i, big) for i, n in enumerate([9, 1, 30, 3])])
    t.check()
    shorten(t, [5, 17, 40, 64])
    t.append([rows(n, heads, dim, dtype, 20 + i, 0.1) for i, n in enumerate([4, 15, 1, 2])])
    t.check()
    shorten(t, [6, 20, 33, 65])
    t.append([rows(1, heads, dim, dtype, 30 + i, 0.1) for i in range(4)], single=True)
    t.check()
    for b in range(4):
        for got, want in zip(t.read(b, dtype), t.want[b].values()):
            assert torch.equal(got, want.to(dtype))


def test_small_values_survive():
    """One token of 30000 that is taken back: the next tokens, of 0.01, are as they would be without it."""
    for single in (True, False):
        a, b = (both([40], 32, 1, 64) for _ in range(2))
        first, rest = rows(3, 1, 64, torch.float16, 1, 0.01), [rows(1, 1, 64, torch.float16, 2 + i, 0.01) for i in range(4)]
        for t in (a, b):
            t.append([first])
        a.append([tuple(torch.full_like(x[:1], 30000.0) for x in first)])
        shorten(a, [3])
        for new in rest:
            a.append([new], single=single)
            b.append([new], single=single)
        a.check()
        # the tokens from before lost bits to the large one; those after it did not
        for got, want in zip(a.read(0, torch.float16), b.read(0, torch.float16)):
            assert torch.equal(got[3:], want[3:])


@pytest.mark.parametrize("dtype", HALF)
def test_zeros_not_finite_and_ranges(dtype):
    """What is left is zero, not finite, or as small as the format's smallest codes; stale codes behind it do not turn NaN."""
    t = both([64] * 4, 64, 2, 64)
    small = [rows(6, 2, 64, dtype, i, 1e-3) for i in range(4)]
    small[0][0].zero_()
    small[0][1].zero_()
    small[1][0][2, 0, 3] = math.inf
    small[2][1][4, 1, 0] = math.nan
    t.append(small)
    large = [rows(9, 2, 64, dtype, 9 + i, 1e3) for i in range(4)]
    large[3][0][1, 0, 0] = math.nan
    t.append(large)
    t.check()
    shorten(t, [6, 6, 6, 8])
    t.append([rows(2, 2, 64, dtype, 20 + i, 1e-4) for i in range(4)])
    t.check()
    # every value byte of the cache is still a number
    assert not ((t.cache.v & 0x7F) == 0x7F).any()
    # and the attention reads what the definition holds
    q = torch.ones(4, 2, 64).to(dtype).cuda()
    o = mq().attention_kv8(q, t.cache, t.table.cuda(), torch.tensor(t.lens, dtype=torch.int32).cuda())
    for b, w in enumerate(t.want):
        k, v = w.values()
        seen = torch.softmax(k.sum(-1) / 8, 0)
        want = (seen[..., None] * torch.nan_to_num(v)).sum(0)
        assert torch.equal(torch.isnan(o[b].cpu().double()), torch.isnan(want))
        # weights in fp16 (2^-11), scores in fp32, the result's rounding
        off = torch.nan_to_num(o[b].cpu().double() - want).abs()
        size = torch.nan_to_num(v).abs().max()
        assert (off <= (2.0 ** -11 + 2.0 ** -8) * size).all()


def test_again_and_again():
    """The same tokens put at the same place twice leave the same bytes."""
    t = both([100], 64, 2, 128)
    t.append([rows(37, 2, 128, torch.float16, 1)])
    new = rows(20, 2, 128, torch.float16, 2, 7.0)
    t.append([new])
    before = [x.clone() for x in (t.cache.k, t.cache.v, t.cache.k_scales, t.cache.v_scales)]
    shorten(t, [37])
    t.append([new])
    t.check()
    for x, y in zip((t.cache.k, t.cache.v, t.cache.k_scales, t.cache.v_scales), before):
        assert torch.equal(x, y)


def test_in_a_graph():
    """A captured step that writes the same place over and over, with values that grow and shrink."""
    t = both([40], 32, 2, 64)
    t.append([rows(4, 2, 64, torch.float16, 1, 0.05)])
    k, v = (torch.zeros(1, 2, 64).half().cuda() for _ in range(2))
    table, lens = t.table.cuda(), torch.tensor([5], dtype=torch.int32).cuda()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mq().kv8_append(t.cache, k, v, table, lens)
    for i, spread in enumerate((0.05, 100.0, 0.05, 1.0, 0.05)):
        a, b = rows(1, 2, 64, torch.float16, 10 + i, spread)
        k.copy_(a)
        v.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        shorten(t, [4])
        t.want[0].append(a, b)
        t.lens = [5]
        t.check()
