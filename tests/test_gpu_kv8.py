"""The paged 8-bit cache: codes, scales and bytes against the definition, bit by bit."""
import copy
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


def rows(n, heads, dim, dtype, seed, spread=1.0):
    g = so.generator(n, heads, dim, seed)
    k = torch.randn(n, heads, dim, generator=g) * spread
    k[..., ::16] += 3.0
    return k.to(dtype), (torch.randn(n, heads, dim, generator=g) * spread).to(dtype)


class Both:
    """A cache and the definition of what it holds, sequence by sequence."""

    def __init__(self, most, page, heads, dim, seed=0, pages=None):
        self.table, self.pages = fo.table_of(most, page, seed)
        self.page, self.lens = page, [0] * len(most)
        self.cache = mq().kv8_cache(self.pages, page, heads, dim)
        self.want = [fo.Rows8(heads, dim) for _ in most]

    def append(self, parts, single=False):
        """parts: (k, v) of each sequence."""
        self.lens = [n + p[0].shape[0] for n, p in zip(self.lens, parts)]
        k, v = (torch.cat([p[w] for p in parts]).cuda() for w in range(2))
        mq().kv8_append(self.cache, k, v, self.table.cuda(), torch.tensor(self.lens, dtype=torch.int32).cuda(),
                        cu_new=None if single else fo.starts([p[0].shape[0] for p in parts]).cuda())
        for w, p in zip(self.want, parts):
            w.append(*p)

    def check(self):
        """Every code and scale that counts, in its place."""
        c = self.cache
        h, d = c.heads, c.head_dim
        kb, vb, ke, ve = (t.cpu() for t in (c.k, c.v, c.k_scales, c.v_scales))
        kb = kb.view(self.pages, h, self.page // 32, 2, d // 64, 4, 16, 16)     # tile, c / 64, quarter, row, byte
        kb = kb.permute(0, 2, 3, 6, 1, 4, 5, 7).reshape(self.pages * self.page, h, d)
        vb = vb.view(self.pages, h, self.page // 32, d // 32, 4, 16, 2, 2, 4)   # pair, quarter, row, tile of channels, of tokens, token
        vb = vb.permute(0, 2, 7, 4, 8, 1, 3, 6, 5).reshape(self.pages * self.page, h, d)
        for b, (n, want) in enumerate(zip(self.lens, self.want)):
            s = fo.slots_of(self.table, b, 0, n, self.page)
            assert torch.equal(kb[s], fo.byte8(want.n[0])), b
            assert torch.equal(vb[s], fo.byte8(want.n[1])), b
            for held, e in ((ke, want.e[0]), (ve, want.e[1])):
                first = fo.slots_of(self.table, b, 0, n, self.page)[::32]
                got = held[first // self.page, :, first % self.page // 32]
                assert torch.equal(got.double() - 127, e), b

    def read(self, b, dtype):
        s = fo.slots_of(self.table, b, 0, self.lens[b], self.page).cuda()
        return [t.cpu() for t in mq().kv8_read(self.cache, s, dtype)]


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads,page,lens", [(1, 32, [1]), (2, 32, [31, 32, 33]), (3, 64, [64, 5, 100, 1]), (8, 128, [200, 129]), (5, 1024, [1100])])
def test_prompts(dtype, dim, heads, page, lens):
    t = Both(lens, page, heads, dim)
    t.append([rows(n, heads, dim, dtype, i) for i, n in enumerate(lens)])
    t.check()
    for b in range(len(lens)):
        for got, want in zip(t.read(b, dtype), t.want[b].values()):
            assert torch.equal(got, want.to(dtype))


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("dim", [64, 128])
def test_parts_and_tokens(dtype, dim):
    """Parts that begin and end inside blocks, and tokens one by one, with values that grow and shrink."""
    heads = 3
    t = Both([200, 200, 200], 64, heads, dim)
    t.append([rows(n, heads, dim, dtype, i, s) for i, (n, s) in enumerate([(5, 1.0), (0, 1.0), (40, 1e-3)])])
    t.check()
    t.append([rows(n, heads, dim, dtype, 9 + i, s) for i, (n, s) in enumerate([(27, 30.0), (32, 1.0), (23, 1e2)])])
    t.check()
    for i in range(40):
        t.append([rows(1, heads, dim, dtype, 100 * i + b, 2.0 ** ((7 * i + 3 * b) % 11 - 5)) for b in range(3)], single=i % 2 == 0)
    t.check()
    t.append([rows(n, heads, dim, dtype, 70 + i) for i, n in enumerate([0, 1, 64])])
    t.check()


def test_many_sequences():
    """The sequence of a block is looked for among 64 at a time: 70 and 4200 of them, most without new tokens."""
    for count, new in ((70, lambda b: (b * 7) % 5), (4200, lambda b: 1 if b % 97 == 0 else 0), (4200, lambda b: 33 if b in (0, 64, 4199) else 0)):
        t = Both([33] * count, 64, 1, 64, pages=None)
        t.append([rows(new(b), 1, 64, torch.float16, b) for b in range(count)])
        t.check()


@pytest.mark.parametrize("dtype", HALF)
def test_not_finite(dtype):
    t = Both([70, 40], 32, 2, 64)
    (k, v), (k2, v2) = rows(50, 2, 64, dtype, 1), rows(40, 2, 64, dtype, 2)
    k[3, 0, 5], v[7, 1, 60], k[33, 1, 0], v[33, 1, 0] = math.inf, math.nan, -math.inf, math.inf
    k2[:, 0] = math.nan                                             # a head that holds nothing else
    t.append([(k, v), (k2, v2)])
    t.check()
    got_k, got_v = t.read(0, dtype)
    assert torch.isnan(got_k[3, 0]).all() and (got_v[3, 0] == 0).all() and torch.isfinite(got_k[3, 1]).all()
    assert torch.isnan(got_k[7, 1]).all() and (got_v[7, 1] == 0).all()
    big, v = rows(20, 2, 64, dtype, 3, 1000.0)                      # the block's scale grows over a NaN key
    t.append([(big, v), (k2[:0], v2[:0])])
    t.check()
    assert torch.isnan(t.read(0, dtype)[0][33, 1]).all()


def test_ranges():
    """bf16 from its largest values to its subnormal ones; borders of the scale; zeros."""
    k, v = rows(33, 4, 64, torch.bfloat16, 5)
    v[:, 0] = 3.3895e38
    v[:, 1] = 2.0 ** -133
    v[:, 2] = 0.0
    v[:, 3] *= 1e-37
    k[:, 0], k[:, 1], k[:, 2] = 448.0, 450.0, 1.75 * 2.0 ** -60
    k[:, 3] *= 2.0 ** 100
    t = Both([66], 32, 4, 64)
    t.append([(k, v)])
    t.check()
    assert torch.equal(t.read(0, torch.bfloat16)[1][:, 1].float(), torch.full((33, 64), 2.0 ** -133))
    k2, v2 = rows(33, 4, 64, torch.bfloat16, 6, 1e30)               # codes of small values fall away
    t.append([(k2, v2)])
    t.check()


def test_every_code():
    """All 253 finite values of the format, with all ties between neighbours, keep or find their codes."""
    byte = torch.arange(256, dtype=torch.uint8)
    value = byte.view(torch.float8_e4m3fn).float()
    value = value[~torch.isnan(value)].sort().values.unique()
    both = torch.cat((value, (value[1:] + value[:-1]) / 2))
    both = both[(both * 2.0 ** 9 % 0.5 == 0)]                        # (all of them; fp16 holds them)
    x = torch.zeros(32, 1, 64)
    x.view(-1)[:both.numel()] = both
    assert torch.equal(x.half().float(), x) and x.max() == 448
    t = Both([32], 32, 1, 64)
    t.append([(x.half(), x.half())])
    t.check()
    got = t.read(0, torch.float16)[0].float().view(-1)
    assert torch.equal(got, x.view(-1).to(torch.float8_e4m3fn).float())


def test_what_is_skipped():
    """Tokens of pages outside the cache and past the table, slots outside, negative lengths, and blocks beside them."""
    m = mq()
    heads, dim, page = 2, 64, 32
    cache = m.kv8_cache(3, page, heads, dim)
    for t in (cache.k, cache.v, cache.k_scales, cache.v_scales):
        t.fill_(0x55)
    before = [t.clone() for t in (cache.k, cache.v, cache.k_scales, cache.v_scales)]
    k, v = (t.cuda() for t in rows(200, heads, dim, torch.float16, 1))
    lens = torch.tensor([40, 40, 100, 0], dtype=torch.int32).cuda()
    table = torch.tensor([[-1, 3], [99, -7], [-2, -2], [0, 1]], dtype=torch.int32).cuda()
    m.kv8_append(cache, k, v, table, lens, fo.starts([40, 40, 100, 0]).cuda())
    m.kv8_append(cache, k[:4], v[:4], table, torch.tensor([0, -3, 0, 0], dtype=torch.int32).cuda())
    for t, b in zip((cache.k, cache.v, cache.k_scales, cache.v_scales), before):
        assert torch.equal(t, b)
    table[0, 0] = 1                                                 # page 1 is written, its neighbours are not
    m.kv8_append(cache, k, v, table, lens, fo.starts([40, 40, 100, 0]).cuda())
    for t, b in zip((cache.k, cache.v, cache.k_scales, cache.v_scales), before):
        assert torch.equal(t[0], b[0]) and torch.equal(t[2], b[2]) and not torch.equal(t[1], b[1])
    # more new tokens than the length has: the last of them
    m.kv8_append(cache, k[:10], v[:10], torch.tensor([[2]], dtype=torch.int32).cuda(), torch.tensor([4], dtype=torch.int32).cuda(),
                 fo.starts([10]).cuda())
    got, _ = m.kv8_read(cache, torch.tensor([64, 65, 66, 67, -1, 96, 1 << 40]).cuda())
    want = fo.Rows8(heads, dim).append(k[6:10].cpu(), v[6:10].cpu()).values()[0].half()
    assert torch.equal(got[:4].cpu(), want) and not got[4:].any()


def test_strides_stream_graph_and_copies():
    m = mq()
    heads, dim = 4, 128
    g = so.generator(1)
    qkv = torch.randn(37, 3 * heads, dim, generator=g).half()
    t = Both([80], 64, heads, dim)
    t.want[0].append(qkv[:, heads:2 * heads], qkv[:, 2 * heads:])
    t.lens = [37]
    d = qkv.cuda()
    lens, table, cu = torch.tensor([37], dtype=torch.int32).cuda(), t.table.cuda(), fo.starts([37]).cuda()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    m.kv8_append(t.cache, d[:, heads:2 * heads], d[:, 2 * heads:], table, lens, cu, stream=stream)
    stream.synchronize()
    t.check()
    # a step of one token, captured once, its length read from the device
    k1, v1, step = torch.empty(1, heads, dim).half().cuda(), torch.empty(1, heads, dim).half().cuda(), torch.zeros(1, dtype=torch.int32).cuda()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        m.kv8_append(t.cache, k1, v1, table, step)
    for i in range(3):
        k, v = rows(1, heads, dim, torch.float16, i, 3.0 ** i)
        k1.copy_(k)
        v1.copy_(v)
        step.fill_(38 + i)
        graph.replay()
        torch.cuda.synchronize()
        t.want[0].append(k, v)
        t.lens = [38 + i]
        t.check()
    out = torch.full((40, heads + 1, 2 * dim), 7.0, dtype=torch.bfloat16, device="cuda")
    s = fo.slots_of(t.table, 0, 0, 40, 64).cuda()
    m.kv8_read(t.cache, s, out=(out[:, :heads, :dim], out[:, 1:, dim:]))
    for got, want in zip((out[:, :heads, :dim], out[:, 1:, dim:]), t.want[0].values()):
        assert torch.equal(got.cpu(), want.bfloat16())
    assert (out[:, heads, :dim] == 7).all() and (out[:, 0, dim:] == 7).all()
    other = copy.deepcopy(t.cache)
    t.cache.k.zero_()
    assert torch.equal(m.kv8_read(other, s)[0].cpu(), t.want[0].values()[0].half())


def test_long_offsets():
    """Pages whose bytes lie past 4 GB."""
    m = mq()
    heads, dim, page = 8, 128, 4096
    pages = 1100                                                    # 4.6 GB each of keys and values
    cache = m.kv8_cache(pages, page, heads, dim)
    k, v = rows(70, heads, dim, torch.float16, 3)
    table = torch.tensor([[pages - 1]], dtype=torch.int32).cuda()
    m.kv8_append(cache, k.cuda(), v.cuda(), table, torch.tensor([70], dtype=torch.int32).cuda(), fo.starts([70]).cuda())
    want = fo.Rows8(heads, dim).append(k, v).values()
    s = (torch.arange(70) + (pages - 1) * page).cuda()
    for got, w in zip(m.kv8_read(cache, s), want):
        assert torch.equal(got.cpu(), w.half())
    for counts in ([1], [70]):                                      # and the attention reads them there
        q = torch.randn(counts[0], heads, dim, generator=so.generator(9)).half()
        o = m.attention_kv8(q.cuda(), cache, table, torch.tensor([70], dtype=torch.int32).cuda(), cu_q=fo.starts(counts).cuda(), max_kv=70)
        exact = so.attention(q, *want, 1 / math.sqrt(dim), True)
        assert (o.cpu().double() - exact).abs().max() <= 2.0 ** -10 * exact.abs().max()


def test_refusals():
    m = mq()
    cache = m.kv8_cache(2, 32, 2, 64)
    k, v = (t.cuda() for t in rows(3, 2, 64, torch.float16, 1))
    table, lens = torch.zeros(3, 1, dtype=torch.int32).cuda(), torch.ones(3, dtype=torch.int32).cuda()
    for args in ((k, v.bfloat16(), table, lens), (k, v[:2], table, lens), (k[:2], v[:2], table, lens), (k, v, table.long(), lens),
                 (k, v, table, lens[:2]), (k, v, table, lens, lens), (k.float(), v.float(), table, lens), (k.cpu(), v, table, lens),
                 (k, v, table.cpu(), lens), (k[..., :32], v[..., :32], table, lens), (k.transpose(0, 1), v, table, lens)):
        with pytest.raises((TypeError, ValueError)):
            m.kv8_append(cache, *args)
    with pytest.raises(m.MQError):                                  # rows of 65
        m.kv8_append(cache, torch.zeros(3, 2, 65).half().cuda()[..., :64], v, table, lens)
    for bad in ((2, 16, 2, 64), (2, 48, 2, 64), (0, 32, 2, 64), (2, 32, 0, 64), (2, 32, 2, 96)):
        with pytest.raises(ValueError):
            m.kv8_cache(*bad)
    cache.k_scales = cache.k_scales[:1]
    with pytest.raises(ValueError):
        m.kv8_append(cache, k, v, table, lens)
