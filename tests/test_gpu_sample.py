"""Tokens drawn from logits: the same token as the definition in whole numbers gives, and its probability."""
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

import serving_oracle as so

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.float16, torch.bfloat16]
ONE = 1 << 43


def mq():
    import paper_2606_15652_amd as m
    return m


def draw(x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """One row's token and probability, from whole weights and exact sums.  x: fp32 numpy."""
    x = x.astype(np.longdouble)
    f32 = lambda v: Fraction(float(np.float32(v)))                  # noqa: E731
    if np.isnan(x).any():
        return -1, math.nan
    top = x.max()
    if top == -np.inf:
        return -1, 0.0
    order = np.lexsort((np.arange(len(x)), -x))
    if not temperature > 0:
        return int(order[0]), 1.0
    with np.errstate(invalid="ignore", over="ignore"):
        d = np.where(x == top, 0, (top - x) / np.longdouble(np.float32(temperature)))
    d = np.where(np.isnan(d), np.inf, d)
    w = np.rint(np.exp(-d) * np.longdouble(ONE)).astype(np.uint64)[order]
    n = len(w)
    if 0 < top_k < n:
        n = top_k
    sums = np.cumsum(w)
    if top_p < 1:
        need = max(1, math.ceil(f32(max(top_p, 0.0)) * int(sums[n - 1])))
        n = min(n, int(np.searchsorted(sums, need)) + 1)
    if min_p > 0:
        least = math.ceil(f32(min(min_p, 1.0)) * ONE)
        n = min(n, int((w >= least).sum()))
    s = int(sums[n - 1])
    target = s - 1 if not u < 1 else math.floor(f32(max(u, 0.0)) * s)
    i = int(np.searchsorted(sums, target, side="right"))
    return int(order[i]), int(w[i]) / s


def check(x, u, **more):
    """x [rows, V] on the GPU; parameters: numbers, or lists for each row."""
    rows = x.shape[0]
    types = {"top_k": torch.int32}
    given = {k: torch.tensor(v, dtype=types.get(k, torch.float32)).cuda() if isinstance(v, list) else v for k, v in more.items()}
    tokens, probs = mq().sample(x, torch.tensor(u, dtype=torch.float32).cuda(), **given)
    assert tokens.dtype == torch.int64 and probs.dtype == torch.float32
    tokens, probs, host = tokens.cpu().tolist(), probs.cpu(), x.float().cpu().numpy()
    for r in range(rows):
        row = {k: v[r] if isinstance(v, list) else v for k, v in more.items()}
        token, p = draw(host[r], float(np.float32(u[r])), **{k: v for k, v in row.items() if v is not None})
        assert tokens[r] == token, (r, tokens[r], token, row, u[r])
        # one rounding to fp32 of a quotient in fp64; weights off by a unit of 2^-43
        assert (math.isnan(p) and math.isnan(probs[r])) or abs(probs[r].item() - p) <= 2.0 ** -24 * 1.01 * p + 2.0 ** -40, (r, probs[r], p)
    return tokens


def logits(rows, vocab, dtype, seed, spread=3.0):
    return (torch.randn(rows, vocab, generator=so.generator(rows, vocab, seed)) * spread).to(dtype).cuda()


def params(rows, seed):
    rng = np.random.default_rng(seed)
    return {"temperature": rng.uniform(0.3, 2.0, rows).tolist(), "top_k": rng.integers(1, 300, rows).tolist(),
            "top_p": rng.uniform(0.05, 1.0, rows).tolist(), "min_p": (10.0 ** rng.uniform(-6, -0.2, rows)).tolist()}


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [1, 2, 3, 63, 64, 65, 1000, 2047, 4097, 32003, 131071])
def test_sizes_and_filters(dtype, vocab):
    rows = 6 if vocab > 10000 else 12
    x = logits(rows, vocab, dtype, 1)
    u = np.random.default_rng(vocab).random(rows).tolist()
    p = params(rows, vocab)
    check(x, u)
    check(x, u, **p)
    for name in p:
        check(x, u, **{name: p[name]})
    check(x, u, top_k=p["top_k"], top_p=p["top_p"])
    check(x, u, top_p=p["top_p"], min_p=p["min_p"], temperature=0.7)


@pytest.mark.parametrize("dtype", TYPES)
def test_every_token_has_its_share(dtype):
    """Evenly spread numbers give every token as often as its probability says, and ascend through the order."""
    vocab, rows = 37, 4096
    x = logits(1, vocab, dtype, 3, 1.5).expand(rows, vocab).contiguous()
    u = ((torch.arange(rows) + 0.5) / rows).cuda()
    tokens, probs = mq().sample(x, u, 0.8, top_p=0.97)
    order = torch.sort(x[0].float(), descending=True, stable=True).indices
    rank = torch.empty(vocab, dtype=torch.long, device="cuda")
    rank[order] = torch.arange(vocab, device="cuda")
    assert (rank[tokens].diff() >= 0).all()
    counts = torch.bincount(tokens, minlength=vocab)
    share = torch.zeros(vocab, device="cuda").scatter_(0, tokens, probs)
    assert (counts - share * rows).abs().max() <= 1.01 and abs(share.sum().item() - 1) < 1e-5


def test_borders():
    """Running sums that meet the target exactly: equal logits, whose weights are exact."""
    x = torch.zeros(9, 8).cuda()
    check(x, [0.0, 0.125, 0.25, 0.5, 0.875, 1 - 2.0 ** -24, 2.0 ** -140, 0.125 - 2.0 ** -27, 0.375])
    assert check(x, [0.125] * 9) == [1] * 9
    check(x, [0.99] * 9, top_p=[0.0, 0.125, 0.126, 0.25, 0.5, 0.875, 0.876, 1.0, 1.5])
    check(x, [0.99] * 9, top_k=[0, 1, 2, 7, 8, 9, -1, -(1 << 31), (1 << 31) - 1])
    check(x, [0.99] * 9, min_p=[0.0, 1.0, 2.0, 1e-30, 0.5, math.inf, 1e-40, 0.999, 0.1])
    y = torch.tensor([[0.0, -math.log(2), -math.log(4), -50.0]]).cuda().repeat(5, 1)
    check(y, [0.9999] * 5, min_p=[0.49, 0.51, 0.24, 0.26, 1e-20])
    check(y, [-0.5, 1.0, 7.0, math.inf, 0.0])
    tokens, _ = mq().sample(y, torch.tensor([math.nan] * 5).cuda(), top_p=torch.tensor([math.nan, 0.6, -1.0, 0.0, 1e-45]).cuda(),
                            min_p=torch.full((5,), math.nan).cuda())
    assert tokens.tolist() == [2, 1, 0, 0, 0]                       # (the last has a weight of 2^-72: none)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [3000, 5000, 300000, 1048576])
def test_many_equal(dtype, vocab):
    """More equal logits than are sorted at once: the index decides."""
    x = torch.full((4, vocab), -2.5, dtype=dtype)
    x[1, ::2] = -2.25
    x[2, 100:200] = 5.0
    x[3] = torch.randint(0, 3, (vocab,), generator=so.generator(vocab)).to(dtype) * 0.01
    x = x.cuda()
    check(x, [0.31, 0.7, 0.9, 0.5])
    check(x, [0.31, 0.7, 0.9, 0.5], top_k=[2500, vocab // 2 + 1, 150, vocab - 1], top_p=[0.9, 0.99, 0.5, 0.4])
    check(x, [0.999999, 0.0, 0.01, 0.999], top_p=[0.5, 0.5001, 0.9999, 0.00001])


def test_near_equal_fp32():
    """Logits that differ in their last bits only: one bin holds them all."""
    g = so.generator(5)
    x = (1.0 + torch.randint(0, 5000, (3, 20000), generator=g) * 2.0 ** -23).cuda()
    check(x, [0.2, 0.5, 0.8])
    check(x, [0.2, 0.5, 0.8], top_k=[7777, 3, 19999], top_p=[0.3, 0.99, 0.7])
    check(torch.cat((-x, x * 1e-3), 1), [0.2, 0.5, 0.8], top_k=[7777, 3, 19999])


@pytest.mark.parametrize("dtype", TYPES)
def test_masked_and_not_finite(dtype):
    inf, nan = math.inf, math.nan
    x = logits(10, 500, dtype, 7)
    x[0] = -inf
    x[1] = -inf
    x[1, 321] = -7.0
    x[2, 40:] = -inf
    x[3, 100], x[3, 7], x[3, 499] = inf, inf, inf
    x[4, 250] = nan
    x[5], x[5, 0] = -inf, nan
    x[6] = inf
    x[7, 3], x[7, 4] = inf, nan
    x[8] = -65504.0 if dtype != torch.bfloat16 else -3e38
    x[9] *= 0.0
    u = [0.5, 0.5, 0.9, 0.5, 0.5, 0.5, 0.2, 0.2, 0.7, 0.3]
    check(x, u)
    check(x, u, **params(10, 3))
    check(x, u, top_p=0.5, temperature=1e30)
    check(x, u, temperature=0.0)


def test_temperatures():
    x = logits(8, 3000, torch.float32, 9, 5.0)
    x[3, 50:53] = x[3].max() + 1
    u = [0.1, 0.5, 0.9, 0.5, 0.99, 0.3, 0.6, 0.8]
    assert check(x, u, temperature=[0.0, -1.0, math.nan, 0.0, -math.inf, 0.0, -0.0, 0.0]) == x.argmax(1).tolist()
    check(x, u, temperature=[1e-45, 1e-30, 1e-6, 1e-3, 100.0, 1e10, 3e38, math.inf], top_p=0.9)
    big = x.clone()
    big *= 1e37
    check(big, u, temperature=[1e37, 1e38, 3e38, 1e36, 1e30, 1.0, 2e37, 3e37])
    assert mq().sample(x, torch.tensor(u).cuda(), 0.0)[1].tolist() == [1.0] * 8


@pytest.mark.parametrize("dtype", TYPES)
def test_strides_and_alignment(dtype):
    base = logits(5, 1103, dtype, 11)
    u = [0.1, 0.3, 0.5, 0.7, 0.9]
    for first, last in ((0, 1103), (1, 1000), (3, 1102), (7, 8), (5, 1021)):
        check(base[:, first:last], u, top_p=0.9)
    check(base[2:3, 1:900], u[:1])
    check(base[::2], u[:3], top_k=40)


def test_stream_graph_and_out():
    m = mq()
    x, u = logits(3, 9000, torch.float32, 1), torch.tensor([0.2, 0.6, 0.95]).cuda()
    want = m.sample(x, u, 0.9, top_k=100, top_p=0.9, min_p=0.01)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    got = m.sample(x, u, 0.9, top_k=100, top_p=0.9, min_p=0.01, stream=stream)
    stream.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    k, out = torch.tensor([100] * 3, dtype=torch.int32).cuda(), (torch.zeros(3, dtype=torch.int64).cuda(), torch.zeros(3).cuda())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        m.sample(x, u, 0.9, top_k=k, top_p=0.9, min_p=0.01, out=out)
    for i in range(3):
        x.copy_(logits(3, 9000, torch.float32, 20 + i))
        k.fill_(5 * i + 1)
        graph.replay()
        torch.cuda.synchronize()
        want = m.sample(x, u, 0.9, top_k=5 * i + 1, top_p=0.9, min_p=0.01)
        assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])
    assert m.sample(x[:0], u[:0])[0].shape == (0,)


def test_refusals():
    m = mq()
    x, u = logits(3, 100, torch.float32, 1), torch.rand(3).cuda()
    for args, more in (((x.double(), u), {}), ((x[0], u), {}), ((x, u[:2]), {}), ((x, u.double()), {}), ((x.t().contiguous().t(), u), {}),
                       ((x, u.cpu()), {}), ((x.cpu(), u), {}), ((x, u), {"top_k": torch.ones(3).cuda()}), ((x, u), {"top_p": torch.ones(2).cuda()}),
                       ((x, u), {"temperature": torch.ones(3)}), ((x, u), {"top_k": 1 << 40}), ((x, u), {"out": (u, u)})):
        with pytest.raises((TypeError, ValueError)):
            m.sample(*args, **more)
    for more in ({"temperature": -1.0}, {"temperature": math.nan}, {"top_p": -0.1}, {"min_p": -1.0}, {"min_p": math.nan}):
        with pytest.raises(m.MQError):
            m.sample(x, u, **more)
    with pytest.raises(m.MQError):
        m.sample(torch.empty(1, (1 << 20) + 1, dtype=torch.float16, device="cuda"), u[:1])
    with pytest.raises(m.MQError):
        m.sample(x[:, :0], u)
