"""Attention over the paged 4-bit cache, against the definition in 64 bits on the values that the
cache holds; the tolerance is that of the kernel's roundings (serving_oracle.attention_error)."""
import math

import pytest
import torch

import serving_oracle as so

pytestmark = pytest.mark.gpu
DTYPES = [torch.float16, torch.bfloat16]


def mq():
    import paper_2606_15652_amd as m
    return m


def filled(seqs, heads, dim):
    m = mq()
    cache = m.kv4_cache(seqs.pages, seqs.page, heads, dim)
    if sum(seqs.lens):
        m.kv4_append(cache, torch.cat(seqs.k).cuda(), torch.cat(seqs.v).cuda(), torch.cat(seqs.slots).cuda())
    return cache


def check(lens, nqs, heads, group, dim, page, dtype, seed=0, scale=None, causal=True, spread=1.0, q_spread=1.0, prepare=None, **how):
    """lens, nqs: tokens and queries of each sequence (nqs None: one query each)."""
    m = mq()
    seqs = so.Sequences(lens, heads, dim, page, dtype, seed, spread)
    if prepare:
        prepare(seqs)
    cache = filled(seqs, heads, dim)
    counts = nqs or [1] * len(lens)
    q = (torch.randn(sum(counts), heads * group, dim, generator=so.generator(seed, 5)) * q_spread).to(dtype)
    cu = torch.tensor([0] + list(torch.tensor(counts).cumsum(0)), dtype=torch.int32)
    o = m.attention_kv4(q.cuda(), cache, seqs.table.cuda(), seqs.kv_lens.cuda(), cu_q=cu.cuda() if nqs else None, scale=scale,
                        causal=causal, **how).cpu()
    assert o.dtype == dtype and o.shape == q.shape
    scale = scale or 1 / math.sqrt(dim)
    for b, n in enumerate(lens):
        k, v = so.values4(seqs.k[b]), so.values4(seqs.v[b])
        part = slice(int(cu[b]), int(cu[b + 1]))
        if counts[b] == 0:
            continue
        want = so.attention(q[part], k, v, scale, causal)
        tol = so.attention_error(q[part], k, v, scale, dtype, want) if n else torch.zeros_like(want)
        off = (o[part].double() - want).abs()
        assert torch.equal(torch.isnan(o[part]), torch.isnan(want))
        assert (off <= tol).logical_or(torch.isnan(want)).all(), (b, n, (off / tol).nan_to_num().max())
    return q, cache, seqs, cu, o


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads,group", [(1, 1), (2, 4), (1, 8), (3, 5), (1, 16), (1, 17), (2, 1)])
def test_single_tokens(heads, group, dim, dtype):
    check([1, 2, 15, 16, 17, 31, 32, 33, 100, 257, 700], None, heads, group, dim, 16, dtype)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 1024])
def test_pages(page):
    check([1, page - 1, page, page + 1, 3 * page + 5], None, 2, 4, 128, page, torch.float16, seed=page)
    check([page + 1, 2 * page + 7], [9, 5], 2, 2, 64, page, torch.float16, seed=page)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads,group", [(1, 1), (2, 4), (1, 8), (1, 3)])
def test_prompts(heads, group, dim, dtype):
    check([40, 1, 130, 64, 300], [40, 1, 33, 64, 7], heads, group, dim, 16, dtype)


@pytest.mark.parametrize("nq", [2, 3, 4, 5, 16, 31, 33, 127, 129])
def test_few_queries_at_the_end_of_a_context(nq):
    check([nq, nq + 1, 200 + nq], [nq] * 3, 2, 4, 64, 32, torch.float16, seed=nq)


@pytest.mark.parametrize("heads,group", [(2, 4), (1, 1)])
def test_not_causal(heads, group):
    check([50, 33, 200], [20, 33, 64], heads, group, 128, 16, torch.float16, causal=False)
    check([50, 1], None, heads, group, 128, 16, torch.float16, causal=False)


def test_rows_that_see_nothing():
    # no tokens; more queries than tokens (the first ones stand before the first token); no queries
    _, _, _, cu, o = check([0, 3, 40, 0, 20], [2, 8, 40, 1, 0], 2, 2, 64, 16, torch.float16)
    assert not o[int(cu[0]):int(cu[1])].any() and not o[int(cu[1]):int(cu[1]) + 5].any()
    _, _, _, _, o = check([0, 7, 0], None, 2, 4, 128, 16, torch.float16)
    assert not o[0].any() and not o[2].any()


@pytest.mark.parametrize("lens", [[5000], [4096, 3], [2049, 4999, 130, 0]])
@pytest.mark.parametrize("dim", [64, 128])
def test_long_contexts_split_over_the_chip(lens, dim):
    check(lens, None, 1, 4, dim, 64, torch.float16)


def test_long_prompts():
    check([700], [600], 1, 2, 128, 64, torch.bfloat16)


@pytest.mark.parametrize("lens,nqs", [([1100, 513, 0, 64], [70, 65, 3, 64]), ([4100], [66]), ([2000, 700, 20], [1, 65, 20])])
def test_prompts_split_over_the_chip(lens, nqs):
    """Few workgroups of many columns, cut along the tokens; sequences that reach one part, several or none."""
    check(lens, nqs, 1, 2, 64, 32, torch.float16)
    check(lens, nqs, 2, 1, 128, 16, torch.bfloat16)


def test_bounds_given_by_the_host():
    q, cache, seqs, cu, o = check([30, 500, 77], [3, 7, 1], 2, 4, 128, 16, torch.float16, max_q=7, max_kv=500)
    m = mq()
    again = m.attention_kv4(q.cuda(), cache, seqs.table.cuda(), seqs.kv_lens.cuda(), cu_q=cu.cuda())
    assert (again.cpu().double() - o.double()).abs().max() <= 2e-3 * o.abs().max()


def test_one_token_shares_and_sharp_rows():
    # scores far apart: one token takes all the weight
    check([300, 33], None, 2, 4, 128, 16, torch.float16, scale=8.0, q_spread=4.0)
    # equal scores: q = 0
    check([300, 33], None, 2, 4, 128, 16, torch.float16, q_spread=0.0)


@pytest.mark.parametrize("spread", [1e-4, 300.0])
def test_sizes_of_values(spread):
    check([300, 33], None, 2, 4, 64, 16, torch.float16, spread=spread)
    check([100], [90], 2, 4, 64, 16, torch.bfloat16, spread=spread)


@pytest.mark.parametrize("dtype,q_spread", [(torch.float16, 2000.0), (torch.float16, 1e-6), (torch.bfloat16, 1e6), (torch.bfloat16, 1e-20)])
def test_sizes_of_queries(dtype, q_spread):
    check([200, 33], None, 2, 4, 64, 16, dtype, q_spread=q_spread, scale=1.0 / (8 * q_spread))


def test_values_whose_scales_differ_by_much():
    def prepare(seqs):
        for v in seqs.v:
            v *= torch.logspace(-3, 2, v.shape[0])[:, None, None].to(v.dtype)
    check([400, 64], None, 2, 2, 128, 16, torch.float16, prepare=prepare)

    def back(seqs):
        for v in seqs.v:
            v *= torch.logspace(2, -3, v.shape[0])[:, None, None].to(v.dtype)
    check([400, 64], [64, 64], 2, 2, 128, 16, torch.float16, prepare=back)


def test_rows_that_are_not_finite_reach_only_those_that_see_them():
    def prepare(seqs):
        seqs.k[0][20, 0, 3] = math.inf                      # key head 0, token 20
        seqs.v[1][5, 1, 0] = math.nan                       # key head 1, token 5
    _, _, _, cu, o = check([32, 16, 50], [32, 16, 50], 2, 2, 64, 16, torch.float16, prepare=prepare)
    assert torch.isfinite(o[:20]).all() and torch.isnan(o[20:32, :2]).all() and torch.isfinite(o[20:32, 2:]).all()
    assert torch.isfinite(o[32:37]).all() and torch.isnan(o[37:48, 2:]).all() and torch.isfinite(o[48:]).all()


def test_what_lies_past_the_end_is_never_seen():
    """Tokens of the last page past a sequence's length, and other pages, hold what is not finite."""
    m = mq()
    lens = [1, 13, 16, 35]
    seqs = so.Sequences(lens, 2, 64, 16, torch.float16, 3)
    cache = m.kv4_cache(seqs.pages, 16, 2, 64)
    for t in (cache.k, cache.v):
        t.fill_(0xFF)
    for t in (cache.k_params, cache.v_params):
        t.fill_(math.nan)
    m.kv4_append(cache, torch.cat(seqs.k).cuda(), torch.cat(seqs.v).cuda(), torch.cat(seqs.slots).cuda())
    for nqs in (None, [1, 13, 5, 35]):
        counts = nqs or [1] * 4
        q = torch.randn(sum(counts), 8, 64, generator=so.generator(4)).half()
        cu = torch.tensor([0] + list(torch.tensor(counts).cumsum(0)), dtype=torch.int32)
        o = m.attention_kv4(q.cuda(), cache, seqs.table.cuda(), seqs.kv_lens.cuda(), cu_q=cu.cuda() if nqs else None).cpu()
        for b in range(4):
            part = slice(int(cu[b]), int(cu[b + 1]))
            k, v = so.values4(seqs.k[b]), so.values4(seqs.v[b])
            want = so.attention(q[part], k, v, 0.125, True)
            assert ((o[part].double() - want).abs() <= so.attention_error(q[part], k, v, 0.125, torch.float16, want)).all()


def test_pages_outside_the_cache_hold_nothing():
    m = mq()
    seqs = so.Sequences([48, 40], 1, 64, 16, torch.float16, 6)
    cache = filled(seqs, 1, 64)
    table = seqs.table.clone()
    table[0, 1], table[1, 0] = -7, 1 << 30
    q = torch.randn(2, 4, 64, generator=so.generator(8)).half()
    o = m.attention_kv4(q.cuda(), cache, table.cuda(), seqs.kv_lens.cuda()).cpu()
    for b, left in ((0, list(range(16)) + list(range(32, 48))), (1, list(range(16, 40)))):
        k, v = so.values4(seqs.k[b])[left], so.values4(seqs.v[b])[left]
        want = so.attention(q[b:b + 1], k, v, 0.125, False)
        assert ((o[b:b + 1].double() - want).abs() <= so.attention_error(q[b:b + 1], k, v, 0.125, torch.float16, want)).all()


def test_strides_and_in_place_output():
    m = mq()
    seqs = so.Sequences([20, 70], 2, 128, 16, torch.float16, 9)
    cache = filled(seqs, 2, 128)
    qkv = torch.randn(2, 12, 128, generator=so.generator(10)).half().cuda()
    args = (cache, seqs.table.cuda(), seqs.kv_lens.cuda())
    want = m.attention_kv4(qkv[:, :8].contiguous(), *args)
    assert torch.equal(m.attention_kv4(qkv[:, :8], *args), want)
    out = torch.full((8, 2, 136), 3.0).half().cuda()
    m.attention_kv4(qkv[:, :8], *args, out=out.transpose(0, 1)[..., :128])
    assert torch.equal(out.transpose(0, 1)[..., :128], want) and (out[..., 128:] == 3).all()


def test_another_stream_a_workspace_and_the_same_again():
    m = mq()
    q, cache, seqs, _, o = check([3000, 100], None, 2, 4, 128, 16, torch.float16)
    qd, args = q.cuda(), (cache, seqs.table.cuda(), seqs.kv_lens.cuda())
    need = m.attention_kv4_workspace_bytes(2, 2, 2, 4, 128, 1, seqs.table.shape[1] * 16)
    assert need > 0
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    for _ in range(4):
        got = m.attention_kv4(qd, *args, workspace=ws, stream=stream)
        stream.synchronize()
        assert torch.equal(got.cpu(), o)


def test_in_a_graph():
    m = mq()
    q, cache, seqs, _, o = check([3000, 100], None, 2, 4, 128, 16, torch.float16)
    qd, table, lens = q.cuda(), seqs.table.cuda(), seqs.kv_lens.cuda()
    out = torch.empty_like(qd)
    ws = torch.empty(m.attention_kv4_workspace_bytes(2, 2, 2, 4, 128, 1, seqs.table.shape[1] * 16), dtype=torch.uint8, device="cuda")
    m.attention_kv4(qd, cache, table, lens, out=out, workspace=ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        m.attention_kv4(qd, cache, table, lens, out=out, workspace=ws)
    for i in range(4):
        lens[0] = 3000 - 700 * i                            # the lengths are read when it runs
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, m.attention_kv4(qd, cache, table, lens))
    lens[0] = 3000
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out.cpu(), o)


def test_a_cache_past_32_bits():
    """Pages near the end of more than 4 GB of codes."""
    m = mq()
    heads, dim, page = 64, 128, 256
    cache = m.kv4_cache(4200, page, heads, dim)
    g = so.generator(11)
    k, v = torch.randn(300, heads, dim, generator=g).half(), torch.randn(300, heads, dim, generator=g).half()
    t = torch.arange(300)
    table = torch.tensor([[4199, 4198]], dtype=torch.int32)
    m.kv4_append(cache, k.cuda(), v.cuda(), (table[0, t // page].long() * page + t % page).cuda())
    q = torch.randn(1, heads, dim, generator=g).half()
    o = m.attention_kv4(q.cuda(), cache, table.cuda(), torch.tensor([300], dtype=torch.int32).cuda()).cpu()
    kd, vd, scale = so.values4(k), so.values4(v), 1 / math.sqrt(dim)
    want = so.attention(q, kd, vd, scale, True)
    assert ((o.double() - want).abs() <= so.attention_error(q, kd, vd, scale, torch.float16, want)).all()


def test_refusals():
    m = mq()
    cache = m.kv4_cache(4, 16, 2, 64)
    q, table, lens = torch.zeros(2, 4, 64).half().cuda(), torch.zeros(2, 2, dtype=torch.int32).cuda(), torch.ones(2, dtype=torch.int32).cuda()
    cu = torch.tensor([0, 1, 2], dtype=torch.int32).cuda()
    for error, call in [
        (TypeError, lambda: m.attention_kv4(q.float(), cache, table, lens)),
        (ValueError, lambda: m.attention_kv4(q[:, :3], cache, table, lens)),
        (ValueError, lambda: m.attention_kv4(q[..., :32], cache, table, lens)),
        (ValueError, lambda: m.attention_kv4(q[:1], cache, table, lens)),
        (TypeError, lambda: m.attention_kv4(q, cache, table.long(), lens)),
        (TypeError, lambda: m.attention_kv4(q, cache, table, lens.long())),
        (ValueError, lambda: m.attention_kv4(q, cache, table, lens[:1])),
        (ValueError, lambda: m.attention_kv4(q, cache, table, lens, cu_q=cu[:2])),
        (ValueError, lambda: m.attention_kv4(q, cache, table, lens, max_kv=33)),
        (m.MQError, lambda: m.attention_kv4(q, cache, table, lens, scale=-1.0)),
        (m.MQError, lambda: m.attention_kv4(q, cache, table, lens, scale=math.nan)),
        (m.MQError, lambda: m.attention_kv4(q, cache, table, lens, cu_q=cu, max_q=-1)),
        (m.MQError, lambda: m.attention_kv4(torch.zeros(2, 4, 72).half().cuda()[..., 4:68], cache, table, lens)),
        (ValueError, lambda: m.attention_kv4(q, cache, table, lens, out=torch.zeros(2, 4, 32).half().cuda())),
        (TypeError, lambda: m.attention_kv4(q, cache, table, lens, out=torch.zeros(2, 4, 64).cuda())),
        (TypeError, lambda: m.attention_kv4(q.cpu(), cache, table, lens)),
    ]:
        with pytest.raises(error):
            call()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("nq", [1, 40])
@pytest.mark.parametrize("scale", [0.125, 1e-30])
def test_scales_of_every_size(nq, dtype, scale):
    """Values without spread, with a scale below fp16's normal range (an absolute 2^-25 of rounding, the tolerance
    2^-22), on a power of two, large and ordinary; keys without spread; one kind a sequence."""
    def prepare(seqs):
        g = so.generator(nq, 3)
        for b, size in enumerate([0.0, 2.0 ** -11, 15.0 / 8, 15 * 2.0 ** 10, 1.0]):
            ramp = torch.rand(77, 2, 64, generator=g)
            ramp[..., 0], ramp[..., 1] = 0.0, 1.0
            seqs.v[b] = ((ramp - 0.5) * size + (0.75 if b == 0 else 0.0)).to(dtype)
        seqs.k[4] = seqs.k[4][..., :1].repeat(1, 1, 64)
    check([77] * 5, [nq] * 5, 2, 4, 64, 16, dtype, seed=nq, scale=scale, prepare=prepare)


@pytest.mark.parametrize("nqs", [None, [40, 20]])
def test_rows_without_spread_below_a_step_of_fp16(nqs):
    """bf16 rows whose minimum rounds up past their maximum in fp16 (scale 0) are rows like others."""
    def prepare(seqs):
        for b in range(2):
            for t, size in ((0, 1e-6), (7, -1e-10), (18, 1e-7)):
                seqs.k[b][t], seqs.v[b][t] = size, -size
    _, _, _, _, o = check([70, 20], nqs, 2, 4, 64, 16, torch.bfloat16, prepare=prepare)
    assert torch.isfinite(o).all()


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("nqs", [None, [90, 40]])
def test_values_past_fp16s_range(nqs, dim):
    """bf16 value rows that the format holds (minimum and scale fit fp16), of values that do not: those who see them
    get them, those who do not get what they get without them."""
    large = {70: (6e4, 3e5), 75: (-6e4, 9e5), 80: (65000.0, 1e5), 85: (-65000.0, -20000.0), 88: (6.5e4, 6.5e4)}

    def prepare(seqs):
        g = so.generator(dim, 21)
        for b in range(2):
            for t, (lo, hi) in large.items():
                row = torch.rand(2, dim, generator=g)
                row[:, 0], row[:, 1] = 0.0, 1.0
                seqs.v[b][t] = (lo + (hi - lo) * row).bfloat16()
    q, _, seqs, cu, o = check([90, 90], nqs, 2, 4, dim, 16, torch.bfloat16, prepare=prepare)
    assert torch.isfinite(o).all()
    if nqs:                                                 # queries 0 .. 69 of the first sequence see none of them
        k, v = so.values4(seqs.k[0])[:70], so.values4(seqs.v[0])[:70]
        want = so.attention(q[:70], k, v, 1 / math.sqrt(dim), True)
        assert ((o[:70].double() - want).abs() <= so.attention_error(q[:70], k, v, 1 / math.sqrt(dim), torch.bfloat16, want)).all()


def test_prompts_with_the_bounds_left_to_their_defaults():
    """All rows of Q and the whole of a long table as bounds: launches of many workgroups that have nothing to do."""
    m = mq()
    lens, nqs = [600 + b for b in range(16)], [512 if b % 2 else 300 + b for b in range(16)]
    seqs = so.Sequences(lens, 8, 64, 64, torch.float16, 31, most=1024 * 2)
    cache = filled(seqs, 8, 64)
    q = torch.randn(sum(nqs), 32, 64, generator=so.generator(32)).half().cuda()
    cu = torch.tensor([0] + list(torch.tensor(nqs).cumsum(0)), dtype=torch.int32).cuda()
    o = m.attention_kv4(q, cache, seqs.table.cuda(), seqs.kv_lens.cuda(), cu_q=cu)
    again = m.attention_kv4(q, cache, seqs.table.cuda(), seqs.kv_lens.cuda(), cu_q=cu, max_q=512, max_kv=615)
    assert (o.double() - again.double()).abs().max() <= 2e-3 * again.abs().max()
    b, at = 3, int(cu[3])
    i = [0, 1, 255, 511]
    k, v = so.values4(seqs.k[b]), so.values4(seqs.v[b])
    for j in i:
        seen = lens[b] - nqs[b] + j + 1
        want = so.attention(q[at + j:at + j + 1].cpu(), k[:seen], v[:seen], 0.125, True)
        tol = so.attention_error(q[at + j:at + j + 1].cpu(), k[:seen], v[:seen], 0.125, torch.float16, want)
        assert ((o[at + j:at + j + 1].cpu().double() - want).abs() <= tol).all()


def sink(nq, nats, step):
    """One token `nats` above all others, which together have a share: their weights count in both sums alike.  Each is
    off by 2^-11 of itself, or by `step` of the largest."""
    m = mq()
    n, heads, dim = 4096, 256, 64                           # as many heads as CUs: contexts are not split
    g = so.generator(nq, 41)
    k, v = torch.zeros(n, 1, dim), torch.rand(n, 1, dim, generator=g)
    v[..., 0], v[..., 1] = 0.0, 1.0
    v = (v * 15).round() / 16                               # values and keys that the cache holds as they are
    k[0, :, 0], v[0] = 15.0, 0.0
    cache = m.kv4_cache(n // 64, 64, heads, dim)
    m.kv4_append(cache, k.half().cuda().expand(-1, heads, -1), v.half().cuda().expand(-1, heads, -1), torch.arange(n).cuda())
    table = torch.arange(n // 64, dtype=torch.int32)[None].cuda()
    q = torch.zeros(nq, heads, dim)
    q[..., 0] = nats / 15 * 8
    q = q.half()
    kd, vd = so.values4(k.half())[:, 0], so.values4(v.half())[:, 0]
    assert kd[0, 0] == 15 and torch.equal(vd, v[:, 0].double())
    o = m.attention_kv4(q.cuda(), cache, table, torch.tensor([n], dtype=torch.int32).cuda(),
                        cu_q=torch.tensor([0, nq], dtype=torch.int32).cuda()).cpu().double()
    w = torch.exp(0.125 * (kd @ q[0, 0].double() - 15 * q[0, 0, 0].double()))
    for i in range(nq):
        seen = n - nq + i + 1
        want = (w[:seen] @ vd[:seen]) / w[:seen].sum()
        tol = want * (2.0 ** -11 + 2.0 ** -18) + n * step * vd.max() + so.UNIT[torch.float16] * want + so.TINY[torch.float16]
        assert ((o[i] - want).abs() <= tol).all(), ((o[i] - want).abs() / tol).max()


@pytest.mark.parametrize("nats", [14.0, 17.0, 18.5, 20.0])
def test_a_sink_beside_a_long_context_many_queries(nats):
    sink(65, nats, 2.0 ** -33)                              # fp16's smallest step, halved, of weights held up to 2^8 at the maximum


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("nq", [1, 3, 40])
def test_small_values_beside_a_hidden_large_row(nq, dtype):
    """A token without weight whose values are ten million times the others': its scale does not cost theirs.  The
    weight of a code's part is held to fp16's smallest step at 2^-6 of the largest scale, 7.5 codes of it at most."""
    m = mq()
    n, dim, group = 64 + nq, 64, 4
    g = so.generator(nq, 43)
    k, v = torch.zeros(n, 1, dim), torch.rand(n, 1, dim, generator=g) * 2e-3
    k[..., 0], k[9, 0, 0], k[5, 0, 0] = 15.0, 30.0, 0.0     # scores: the first far above the second, that above the third
    v[5] = (torch.rand(dim, generator=g) - 0.5) * 50000
    k, v = k.to(dtype), v.to(dtype)
    cache = m.kv4_cache(-(-n // 16), 16, 1, dim)
    m.kv4_append(cache, k.cuda(), v.cuda(), torch.arange(n).cuda())
    table = torch.arange(-(-n // 16), dtype=torch.int32)[None].cuda()
    q = torch.zeros(nq, group, dim)
    q[..., 0] = 16.0
    q = q.to(dtype)
    kd, vd = so.values4(k), so.values4(v)
    o = m.attention_kv4(q.cuda(), cache, table, torch.tensor([n], dtype=torch.int32).cuda(),
                        cu_q=torch.tensor([0, nq], dtype=torch.int32).cuda()).cpu().double()
    want = so.attention(q, kd, vd, 0.125, True)
    large = so.quantise4(v)[1].max().item()
    rest = torch.cat((vd[:5], vd[6:]))
    tol = 2.0 ** -11 * (rest.max() - rest.min()) * 1.01 + 7.5 * 2.0 ** -25 * large * 2.0 ** -6 + math.exp(-60 * 0.99) * 3e4 \
        + 2.0 ** -22 * rest.max() + so.UNIT[dtype] * want.abs() * 1.01 + so.TINY[dtype]
    assert ((o - want).abs() <= tol).all(), ((o - want).abs() / tol).max()


@pytest.mark.parametrize("nats", [14.0, 17.0, 18.5, 20.0])
def test_a_sink_beside_a_long_context_one_query(nats):
    sink(1, nats, 2.0 ** -32)                               # half of fp16's smallest step at 2^-6 of the scale, 7.5 codes of it


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("q_spread", [1e6, 1e-6])
@pytest.mark.parametrize("nqs", [[1, 1], [3, 2], [40, 17]])
def test_queries_that_are_not_finite_change_no_others(nqs, q_spread, bad):
    m = mq()
    lens, heads, group, dim = [100, 60], 1, 4, 64
    seqs = so.Sequences(lens, heads, dim, 16, torch.bfloat16, 51)
    cache = filled(seqs, heads, dim)
    q = (torch.randn(sum(nqs), heads * group, dim, generator=so.generator(52)) * q_spread).bfloat16()
    hit = q.clone()
    hit[0, 1, 5] = bad
    cu = torch.tensor([0] + list(torch.tensor(nqs).cumsum(0)), dtype=torch.int32)
    scale = 1.0 / (2 * q_spread)
    o = m.attention_kv4(hit.cuda(), cache, seqs.table.cuda(), seqs.kv_lens.cuda(), cu_q=cu.cuda(), scale=scale).cpu()
    assert torch.isnan(o[0, 1]).any()
    for b in range(2):
        part = slice(int(cu[b]), int(cu[b + 1]))
        k, v = so.values4(seqs.k[b]), so.values4(seqs.v[b])
        want = so.attention(q[part], k, v, scale, True)
        off = (o[part].double() - want).abs()
        fine = off <= so.attention_error(q[part], k, v, scale, torch.bfloat16, want)
        if b == 0:
            fine[0, 1] = True
        assert fine.all()


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("group,nqs", [(1, None), (2, None), (3, None), (5, None), (8, None), (9, None), (16, None), (40, None),
                                       (1, [2, 1, 0, 2]), (1, [4, 3, 4, 1]), (4, [2, 2, 1, 2]), (3, [5, 1, 5, 4]), (8, [8, 8, 2, 8])])
def test_long_contexts_of_every_number_of_columns(group, nqs, dim):
    """Contexts cut into shares, by blocks of 4 (one, two or more queries in use), 8 and 16 columns, one block or several."""
    check([4999, 1100, 0, 70], nqs, 2, group, dim, 32, DTYPES[group % 2], seed=group)


@pytest.mark.parametrize("n,nq", [(300, 1), (5000, 1), (300, 3), (5000, 70)])
def test_scores_far_below_zero(n, nq):
    """Every score below -1e30: the highest takes all the weight all the same."""
    m = mq()
    g = so.generator(n, 61)
    k, v = torch.zeros(n, 1, 64), torch.randn(n, 1, 64, generator=g).bfloat16()
    k[:, 0, 0] = 2.0 + torch.randperm(n, generator=g) % 60 / 16
    k[n // 3, 0, 0] = 1.0                                   # seen by all
    k = k.bfloat16()
    cache = m.kv4_cache(-(-n // 16), 16, 1, 64)
    m.kv4_append(cache, k.cuda(), v.cuda(), torch.arange(n).cuda())
    q = torch.zeros(nq, 1, 64).bfloat16()
    q[..., 0] = -1e32
    o = m.attention_kv4(q.cuda(), cache, torch.arange(-(-n // 16), dtype=torch.int32)[None].cuda(), torch.tensor([n], dtype=torch.int32).cuda(),
                        cu_q=torch.tensor([0, nq], dtype=torch.int32).cuda(), scale=1.0).cpu().double()
    want = so.values4(v)[n // 3, 0]
    spread = (v.float().amax() - v.float().amin()).item()
    tol = (2.0 ** -11 + 2.0 ** -25) * spread * 1.01 + 2.0 ** -22 * want.abs().max() + so.UNIT[torch.bfloat16] * want.abs() * 1.01
    assert ((o[:, 0] - want).abs() <= tol).all()
