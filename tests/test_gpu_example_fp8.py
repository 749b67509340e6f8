"""The decoder layer of the examples in 8-bit floating point, and its tokens: single tokens give what the same tokens give inside
a prompt, and the layer what its steps give in plain arithmetic on the same weights."""
import importlib.util
import math
import os
import sys

import pytest
import torch

import fp8_oracle as fo
import serving_oracle as so
from test_gpu_sample import draw

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ex():
    spec = importlib.util.spec_from_file_location("decoder_layer", os.path.join(ROOT, "examples", "decoder_layer.py"))
    m = importlib.util.module_from_spec(spec)
    sys.modules[spec.name] = m                             # (its dataclasses look for their module)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("dim", [64, 128])
def test_prompts_and_single_tokens_agree(ex, dim):
    layer = ex.random_layer(hidden=512, heads=8, kv_heads=2, head_dim=dim, ffn=512, vocab=1003, seed=dim, fp8=True)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    counts = [40, 17]
    whole = torch.randn((sum(counts) + 2 * 3, 512), generator=g, device="cuda").half()
    a, b = whole[:43], whole[43:]                          # 40 + 3 and 17 + 3 tokens
    full = ex.forward(layer, ex.Batch(layer, 2, 128, page=32, fp8=True), torch.cat((a, b)), [43, 20])
    two = ex.Batch(layer, 2, 128, page=64, fp8=True)
    part = ex.forward(layer, two, torch.cat((a[:40], b[:17])), counts)
    # every step is per token, and attention over nearly the same cache (a block's scale may have grown with its later tokens):
    # what differs is the order of sums, and roundings
    scale = full.abs().max()
    assert (part[:40] - full[:40]).abs().max() <= 0.05 * scale
    for i in range(3):
        step = ex.forward(layer, two, torch.stack((a[40 + i], b[17 + i])), [1, 1])
        assert (step[0] - full[40 + i]).abs().max() <= 0.05 * scale and (step[1] - full[43 + 17 + i]).abs().max() <= 0.05 * scale
    assert two.lens == [43, 20]


def test_cache_attention_projection_and_draw_against_plain_arithmetic():
    """The operators of one step together: append, attention, projection, draw, each on what the one before gave."""
    import paper_2606_15652_amd as mq
    g = so.generator(4)
    heads, group, dim, vocab, lens, counts = 2, 4, 64, 777, [70, 33], [5, 1]
    table, pages = fo.table_of(lens, 32, 1)
    cache = mq.kv8_cache(pages, 32, heads, dim)
    kv = [[torch.randn(n, heads, dim, generator=g).half() for _ in range(2)] for n in lens]
    held = [fo.Rows8(heads, dim) for _ in lens]
    for first, last in (([0, 0], [65, 32]), ([65, 32], lens)):
        new = [[t[f:n] for t in p] for p, f, n in zip(kv, first, last)]
        mq.kv8_append(cache, torch.cat([p[0] for p in new]).cuda(), torch.cat([p[1] for p in new]).cuda(), table.cuda(),
                      torch.tensor(last, dtype=torch.int32).cuda(), fo.starts([p[0].shape[0] for p in new]).cuda())
        for h, p in zip(held, new):
            h.append(*p)
    q = torch.randn(sum(counts), heads * group, dim, generator=g).half()
    o = mq.attention_kv8(q.cuda(), cache, table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), cu_q=fo.starts(counts).cuda(), max_q=5)
    at = 0
    for h, c in zip(held, counts):
        want = so.attention(q[at:at + c], *h.values(), 1 / math.sqrt(dim), True)
        assert (o[at:at + c].cpu().double() - want).abs().max() <= 2.0 ** -11 * want.abs().max() + 1e-4
        at += c
    w = mq.quantize_weight_fp8((torch.randn(vocab, heads * group * dim, generator=g) / 22.6).cuda())
    codes, scales = mq.quantize_rows_fp8(o.view(sum(counts), -1))
    logits = mq.gemm_fp8(codes, scales, w, out_dtype=torch.float32)
    a = codes.cpu().double() * scales.cpu().double().repeat_interleave(128, 1)
    b = mq.unpack_weight_fp8(w).cpu().double() * w.s_w.cpu().double().repeat_interleave(128, 0)[:vocab].repeat_interleave(128, 1)
    want = a @ b.t()
    # 128 products to a group and as many fmas as groups, and windows of eight cut at 2^-13 of their largest product
    assert ((logits.cpu().double() - want).abs() <= (200 * 2.0 ** -24 + 7 * 2.0 ** -13) * (a.abs() @ b.abs().t())).all()
    u = torch.rand(sum(counts), generator=g)
    tokens, probs = mq.sample(logits, u.cuda(), 0.7, top_k=50, top_p=0.9, min_p=0.01)
    for r in range(sum(counts)):
        token, p = draw(logits[r].cpu().numpy(), float(u[r]), 0.7, 50, 0.9, 0.01)
        assert tokens[r] == token and abs(probs[r].item() - p) <= 1e-6


def test_step_in_a_graph():
    """A step of single tokens, captured whole and replayed as contexts grow: as the same calls without a graph."""
    import paper_2606_15652_amd as mq
    heads, group, dim, vocab, b = 2, 4, 128, 1001, 3
    g = torch.Generator(device="cuda")
    g.manual_seed(5)

    def rand(*shape):
        return torch.randn(shape, generator=g, device="cuda").half()
    table = torch.randperm(6, device="cuda").int().reshape(b, 2)
    caches = [mq.kv8_cache(6, 64, heads, dim) for _ in range(2)]
    w = mq.quantize_weight_fp8(rand(vocab, heads * group * dim).float() / 32)
    k, v, q, u = rand(b, heads, dim), rand(b, heads, dim), rand(b, heads * group, dim), torch.rand(b, device="cuda")
    lens = torch.ones(b, dtype=torch.int32, device="cuda")

    def step(cache):
        mq.kv8_append(cache, k, v, table, lens)
        o = mq.attention_kv8(q, cache, table, lens)
        logits = mq.gemm_fp8(*mq.quantize_rows_fp8(o.view(b, -1)), w, out_dtype=torch.float32)
        return o, logits, *mq.sample(logits, u, 0.9, top_k=40, top_p=0.9)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(caches[0])
    for n in range(1, 41):
        k.copy_(rand(b, heads, dim) * (1 + n % 5))
        v.copy_(rand(b, heads, dim))
        q.copy_(rand(b, heads * group, dim))
        u.copy_(torch.rand(b, generator=g, device="cuda"))
        lens.copy_(torch.tensor([n, n + 20 if n > 1 else 1, 1], dtype=torch.int32))
        graph.replay()
        want = step(caches[1])
        torch.cuda.synchronize()
        for x, y in zip(got, want):
            assert torch.equal(x, y), n
