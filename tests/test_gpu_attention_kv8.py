"""Attention over the paged 8-bit cache, against softmax attention in 64 bits on the values that its codes stand for."""
import math

import pytest
import torch

import fp8_oracle as fo
import serving_oracle as so

pytestmark = pytest.mark.gpu
HALF = [torch.float16, torch.bfloat16]


def mq():
    import paper_2606_15652_amd as m
    return m


class Case:
    def __init__(self, lens, heads, dim, page, dtype, seed=0, spread=1.0, change=None, most=None):
        g = so.generator(tuple(lens), heads, dim, page, seed)
        self.lens, self.heads, self.dim, self.page, self.dtype = lens, heads, dim, page, dtype
        self.table, pages = fo.table_of(lens, page, seed, most)
        self.cache = mq().kv8_cache(pages, page, heads, dim)
        kv = []
        for n in lens:
            k = torch.randn(n, heads, dim, generator=g) * spread
            k[..., ::16] += 2.0
            kv.append([k.to(dtype), (torch.randn(n, heads, dim, generator=g) * spread).to(dtype)])
        if change:
            change(kv)
        k, v = (torch.cat([p[w] for p in kv]).cuda() for w in range(2))
        self.kv_lens = torch.tensor(lens, dtype=torch.int32)
        mq().kv8_append(self.cache, k, v, self.table.cuda(), self.kv_lens.cuda(), fo.starts(lens).cuda())
        self.held = [fo.Rows8(heads, dim).append(*p) for p in kv]

    def queries(self, counts, group, seed=0, spread=1.0):
        return (torch.randn(sum(counts), self.heads * group, self.dim, generator=so.generator(tuple(counts), group, seed)) * spread).to(self.dtype)

    def run(self, q, counts, scale=None, causal=True, single=None, **more):
        single = all(c == 1 for c in counts) if single is None else single
        if not single:
            more.setdefault("max_q", max(counts))
        return mq().attention_kv8(q.cuda(), self.cache, self.table.cuda(), self.kv_lens.cuda(),
                                  cu_q=None if single else fo.starts(counts).cuda(), scale=scale, causal=causal, **more)

    def check(self, q, counts, o, scale=None, causal=True, only=None):
        scale = 1 / math.sqrt(self.dim) if scale is None else scale
        at, worst = 0, 0.0
        for b, c in enumerate(counts):
            if only is None or b in only:
                k, v = self.held[b].values()
                qb, got = q[at:at + c], o[at:at + c].cpu().double()
                want = so.attention(qb, k, v, scale, causal)
                assert torch.equal(torch.isnan(got), torch.isnan(want)), b
                if c and k.shape[0]:
                    ev = self.held[b].e[1]
                    tol = fo.attention_error(torch.nan_to_num(qb.double(), 0, 0, 0), k, v, self.held[b].n[1], scale, self.dtype,
                                             torch.nan_to_num(want), ev)
                    off = torch.nan_to_num(got - want).abs()
                    worst = max(worst, (off / tol).max().item())
                    assert (off <= tol).all(), (b, worst)
                else:
                    assert not got.any()
            at += c
        return worst


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads,group", [(1, 1), (2, 4), (1, 8), (3, 5), (2, 16), (1, 17), (1, 40)])
def test_single_tokens(dtype, dim, heads, group):
    lens = [1, 2, 31, 32, 33, 130, 511, 700]
    t = Case(lens, heads, dim, 32 if group % 2 else 128, dtype)
    q = t.queries([1] * len(lens), group)
    t.check(q, [1] * len(lens), t.run(q, [1] * len(lens)))


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("heads,group,lens,counts", [
    (1, 1, [5, 64, 33], [5, 7, 33]), (2, 4, [100, 3, 40], [37, 3, 1]), (1, 8, [66, 130], [2, 4]), (2, 1, [300], [300]),
    (1, 5, [77, 1, 200], [60, 1, 129]), (1, 3, [40, 41, 42], [0, 41, 2])])
def test_prompts(dtype, dim, causal, heads, group, lens, counts):
    t = Case(lens, heads, dim, 64, dtype)
    q = t.queries(counts, group)
    t.check(q, counts, t.run(q, counts, causal=causal), causal=causal)


@pytest.mark.parametrize("dim,heads,group,count,n", [(128, 1, 1, 1, 20000), (64, 2, 4, 1, 9001), (128, 1, 8, 3, 5000), (64, 1, 4, 50, 3001),
                                                     (128, 1, 2, 300, 2000)])
def test_split_contexts(dim, heads, group, count, n):
    """Contexts that several workgroups share, beside short ones that one takes."""
    lens, counts = [n, 3, n // 2 + 1], [count, min(count, 3), count]
    t = Case(lens, heads, dim, 256, torch.float16)
    assert mq().attention_kv8_workspace_bytes(3, sum(counts), heads, group, dim, count, n) > 0
    q = t.queries(counts, group)
    t.check(q, counts, t.run(q, counts, max_kv=n))


def test_rows_that_see_nothing():
    """No tokens, fewer tokens than queries, and pages that are not there."""
    t = Case([0, 3, 40, 70], 2, 64, 32, torch.float16)
    counts = [4, 9, 5, 70]
    q = t.queries(counts, 4)
    o = t.run(q, counts)
    t.check(q, counts, o)
    assert not o[:4].any() and not o[4:10].any() and o[10].any()
    t.table[3, 0] = -1                                              # its first 32 tokens are seen by none
    t.table[2, :] = 1 << 20
    o = t.run(q, counts)
    assert not o[13:18].any() and not o[18:18 + 32].any()
    for w in range(2):
        t.held[3].n[w], t.held[3].e[w] = t.held[3].n[w][32:], t.held[3].e[w][1:]
    t.check(q[50:], [0, 0, 0, 38], o[50:])


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("group", [1, 4, 40])
def test_not_finite(dtype, group):
    """A token that is not finite reaches those who see it, a query that is not only itself."""
    def change(kv):
        kv[0][0][20, 0, 3], kv[0][1][45, 1, 7], kv[1][1][2, 0, 0] = math.inf, math.nan, -math.inf
    t = Case([50, 40], 2, 64, 32, dtype, change=change)
    counts = [50, 3]
    q = t.queries(counts, group)
    q[3, 0, 5], q[7, group, 9], q[51, 0, 0] = math.nan, math.inf, -math.inf
    o = t.run(q, counts)
    want_nan = torch.zeros(53, 2 * group, dtype=torch.bool)
    want_nan[20:50, :group] = True
    want_nan[45:50, group:] = True
    want_nan[50:, :group] = True
    want_nan[3, 0] = want_nan[7, group] = want_nan[51, 0] = True
    nan = torch.isnan(o.cpu()).all(-1)
    assert torch.equal(nan, want_nan) and torch.equal(torch.isnan(o.cpu()).any(-1), nan)
    q2 = q.clone()
    for r, h in ((3, 0), (7, group), (51, 0)):
        q2[r, h] = 0
    again = t.run(q2, counts)
    assert torch.equal(again.cpu()[~want_nan], o.cpu()[~want_nan])   # nothing else moved
    t.check(q2, counts, again)


@pytest.mark.parametrize("dtype", HALF)
def test_scales_far_apart(dtype):
    """Blocks of values thousands and millions of times larger that are given next to no weight, and of tiny values that have
    it all; zeros; a sink beside a long context."""
    def change(kv):
        k, v = kv[0]
        k.zero_()
        k[:64, 0, 0] = -60.0                                        # their weight is e^-60 of the others'
        v[:32] *= 200.0 if dtype == torch.float16 else 1e8
        v[64:] *= 1e-3
        k, v = kv[1]
        v[:96].zero_()
        v[96:] *= 1e-4
        k, v = kv[2]
        k.zero_()
        k[40, 0, 0], v[40] = 17.0, 1.0
        v[64:] *= 1e-2
    t = Case([150, 150, 2000], 1, 64, 32, dtype, change=change)
    q = torch.zeros(3, 1, 64).to(dtype)
    q[..., 0] = 1.0
    o = t.run(q, [1, 1, 1], scale=1.0)
    # by the weights that blocks have, not by the largest value: tokens 64 on of the first, 96 on of the second
    for b, first in ((0, 64), (1, 0), (2, 0)):
        k, v = t.held[b].values()
        want = so.attention(q[b:b + 1], k, v, 1.0, True)[0]
        p = torch.softmax(k[:, 0, 0].double(), 0)
        size = (p[:, None] * v[:, 0].abs()).sum(0)
        # a weight's half step, scores exact here, sums in fp32, products below the operands' range: 2^-25 of the largest
        # product of weight and scale times 2^-6, times the code
        lost = k.shape[0] * 448 * 2.0 ** -31 * (p * torch.exp2(t.held[b].e[1][:, 0]).repeat_interleave(32)[:k.shape[0]]).max()
        tol = (2.0 ** -11 + k.shape[0] * 2.0 ** -23) * size + 2 * lost + 2 * so.UNIT[dtype] * want.abs() + so.TINY[dtype]
        off = (o[b].cpu().double() - want).abs()
        assert (off <= tol).all(), (b, (off / tol).max())


@pytest.mark.parametrize("dtype", HALF)
def test_scores_of_any_size(dtype):
    """Keys and queries so large, or so far below zero, that weights are one or nothing; maxima that rise all along."""
    def change(kv):
        k, v = kv[0]
        k.zero_()
        k[:, 0, 0] = torch.arange(300).to(dtype)                    # rises from block to block
        kv[1][0].zero_()
        kv[1][0][:, 0, 1] = -448.0
        kv[2][0].zero_()
        kv[2][0][:, 0, 0] = 256.0
        kv[2][0][150, 0, 0] = 448.0
    t = Case([300, 300, 300], 1, 64, 32, dtype, change=change)
    big = 60000.0 if dtype == torch.float16 else 1e30
    q = torch.zeros(3, 1, 64).to(dtype)
    q[0, 0, 0], q[1, 0, 1], q[2, 0, 0] = 3.0, big, big
    o = t.run(q, [1, 1, 1], scale=1.0).cpu().double()
    held = [h.values() for h in t.held]
    same = held[0][0][:, 0, 0] == held[0][0][:, 0, 0].max()         # codes round the last keys to one value
    for b, want in ((0, held[0][1][same].mean(0)), (1, held[1][1].mean(0)), (2, held[2][1][150])):
        size = held[b][1].abs().max()
        assert (o[b] - want).abs().max() <= size * (2.0 ** -11 + 300 * 2.0 ** -23) + so.UNIT[dtype] * 1.01 * want.abs().max() + 1e-7, b


def test_smallest_queries_and_keys():
    """Scales whose product leaves fp32's range: scores of nothing, and hidden tokens stay hidden."""
    def change(kv):
        kv[0][0].zero_()
        kv[1][0].mul_(1e-36)
        kv[1][1].mul_(1e-30)
        kv[1][1][60:].mul_(1e-8)
    t = Case([90, 90], 1, 64, 32, torch.bfloat16, change=change)
    counts = [90, 40]
    q = t.queries(counts, 2)
    q[:60] *= 1e-38
    q[100:] = 2.0 ** -133
    t.check(q, counts, t.run(q, counts))


def test_strides_streams_workspace_and_graph():
    m = mq()
    t = Case([1500, 40, 700], 2, 128, 64, torch.bfloat16)
    counts, group = [1, 1, 1], 4
    q = t.queries(counts, group)
    o = t.run(q, counts)
    t.check(q, counts, o)
    wide = torch.full((3, 20, 256), 5.0, dtype=torch.bfloat16, device="cuda")
    wide[:, 2:10, 64:192] = q.cuda()
    out = torch.full((3, 9, 160), 3.0, dtype=torch.bfloat16, device="cuda")
    args = (t.cache, t.table.cuda(), t.kv_lens.cuda())
    ws = torch.empty(m.attention_kv8_workspace_bytes(3, 3, 2, group, 128, 1, t.table.shape[1] * 64), dtype=torch.uint8, device="cuda").fill_(255)
    m.attention_kv8(wide[:, 2:10, 64:192], *args, out=out[:, :8, 16:144], workspace=ws)
    assert torch.equal(out[:, :8, 16:144], o) and (out[:, 8] == 3).all() and (out[..., :16] == 3).all() and (out[..., 144:] == 3).all()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    other = m.attention_kv8(q.cuda(), *args, stream=stream)
    stream.synchronize()
    assert torch.equal(other, o)
    # captured: lengths, queries and the table are read when it runs
    qd, lens, table = q.cuda(), t.kv_lens.cuda(), t.table.cuda()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = m.attention_kv8(qd, t.cache, table, lens)
    for new in ([1500, 40, 700], [1, 33, 650], [0, 40, 64]):
        lens.copy_(torch.tensor(new, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, m.attention_kv8(qd, t.cache, table, lens)), new
        if new[0] == 0:
            assert not got[0].any()


def test_bounds_of_the_launch():
    """Queries past max_q are left out and lengths past max_kv cut; rows of Q behind the last sequence stay."""
    m = mq()
    t = Case([100, 90], 1, 64, 32, torch.float16)
    q = t.queries([4, 3, 5], 2)
    out = torch.full_like(q, 7.0).cuda()
    m.attention_kv8(q.cuda(), t.cache, t.table.cuda(), t.kv_lens.cuda(), cu_q=fo.starts([4, 3]).cuda(), max_q=4, out=out)
    t.check(q[:7], [4, 3], out[:7])
    assert (out[7:] == 7).all()
    out.fill_(7.0)
    m.attention_kv8(q.cuda(), t.cache, t.table.cuda(), t.kv_lens.cuda(), cu_q=fo.starts([4, 3]).cuda(), max_q=2, out=out)
    assert (out[2:4] == 7).all() and (out[6:] == 7).all()
    full = t.run(q[:7], [4, 3])
    assert torch.equal(out[:2], full[:2]) and torch.equal(out[4:6], full[4:6])
    assert not m.attention_kv8(q[:2].cuda(), t.cache, t.table.cuda(), t.kv_lens.cuda(), max_kv=0).any()
    assert m.attention_kv8(q[:0].cuda(), t.cache, t.table.cuda(), t.kv_lens.cuda(), cu_q=fo.starts([0, 0]).cuda()).shape == (0, 2, 64)


def test_stale_bytes_count_for_nothing():
    """What lies behind the lengths, in the same block and in pages of the table past them: the largest codes, scales and NaN keys."""
    m = mq()
    t = Case([37, 5], 1, 64, 32, torch.float16, most=4)
    q = t.queries([1, 1], 4)
    o = t.run(q, [1, 1])
    n = t.cache
    used = t.table[t.table >= 0].long()
    free = [p for p in range(n.pages) if p not in used.tolist()]
    n.k[free] = 0x7F
    n.v[free] = 0x7E
    n.v_scales[free] = 254
    t.table[t.table < 0] = free[0]
    k, v = torch.full((20, 1, 64), 3000.0).half(), torch.full((20, 1, 64), -3e4).half()
    k[3] = math.inf
    m.kv8_append(n, k.cuda(), v.cuda(), t.table[:1].cuda(), torch.tensor([57], dtype=torch.int32).cuda(), fo.starts([20]).cuda())
    got = t.run(q, [1, 1])
    assert torch.isfinite(got).all()
    # the growing scale coded 5 tokens anew; the others' results are the same
    t.held[0].append(k, v)
    for w in range(2):
        t.held[0].n[w] = t.held[0].n[w][:37]
    t.check(q, [1, 1], got)
    assert torch.equal(got[1], o[1])


def test_refusals():
    m = mq()
    t = Case([40, 40], 2, 64, 32, torch.float16)
    q = t.queries([1, 1], 2).cuda()
    table, lens, cu = t.table.cuda(), t.kv_lens.cuda(), fo.starts([1, 1]).cuda()
    for args, more in (((q.float(), t.cache, table, lens), {}), ((q[:, :3], t.cache, table, lens), {}), ((q[:1], t.cache, table, lens), {}),
                       ((q, t.cache, table.long(), lens), {}), ((q, t.cache, table, lens[:1]), {}), ((q, t.cache, table, lens, cu[:2]), {}),
                       ((q, t.cache, table, lens), {"max_kv": 65}), ((q, t.cache, table, lens), {"out": q.bfloat16()}),
                       ((q.cpu(), t.cache, table, lens), {}), ((q[..., :32], t.cache, table, lens), {})):
        with pytest.raises((TypeError, ValueError)):
            m.attention_kv8(*args, **more)
    for scale in (0.0, -1.0, math.nan, math.inf):
        with pytest.raises(m.MQError):
            m.attention_kv8(q, t.cache, table, lens, scale=scale)
