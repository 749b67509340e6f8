"""The decoder layer of the examples: single tokens give what the same tokens give inside a prompt, and the
layer as a whole what its steps give in plain arithmetic on the same weights."""
import importlib.util
import math
import os
import sys

import pytest
import torch

import serving_oracle as so

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
    layer = ex.random_layer(hidden=512, heads=8, kv_heads=2, head_dim=dim, ffn=512, vocab=1003, seed=dim)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    counts = [40, 17]
    whole = torch.randn((sum(counts) + 2 * 3, 512), generator=g, device="cuda").half()
    a, b = whole[:43], whole[43:]                          # 40 + 3 and 17 + 3 tokens
    one = ex.Batch(layer, 2, 128, page=16)
    full = ex.forward(layer, one, torch.cat((a, b)), [43, 20])
    two = ex.Batch(layer, 2, 128, page=32)
    part = ex.forward(layer, two, torch.cat((a[:40], b[:17])), counts)
    # every step is per token, and attention over the same cache: what differs is the order of sums and roundings
    scale = full.abs().max()
    assert (part[:40] - full[:40]).abs().max() <= 0.05 * scale
    for i in range(3):
        step = ex.forward(layer, two, torch.stack((a[40 + i], b[17 + i])), [1, 1])
        assert (step[0] - full[40 + i]).abs().max() <= 0.05 * scale and (step[1] - full[43 + 17 + i]).abs().max() <= 0.05 * scale
    assert two.lens == [43, 20]


def test_against_plain_arithmetic(ex):
    """With the codes that the library makes taken as they are, each step is checked by its own tests; here the
    layer's result against the same chain in fp64 from the dequantised weights: 8- and 4-bit activations are
    roundings of a few per cent of a row, so the directions have to agree, not the digits."""
    import paper_2606_15652_amd as mq
    layer = ex.random_layer(hidden=512, heads=4, kv_heads=2, head_dim=128, ffn=512, vocab=500, seed=3)
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    x = torch.randn((30, 512), generator=g, device="cuda").half()
    got = ex.forward(layer, ex.Batch(layer, 1, 64), x, [30]).double().cpu()

    def dense(pw):
        wc, sw, rc = (t.cpu() for t in mq.unpack_weights(pw))

        def nibbles(t):
            v = torch.stack((t & 15, t >> 4), -1).flatten(-2).long()
            return torch.where(v > 7, v - 16, v).double()
        w = nibbles(wc).view(pw.N, -1, 128) * sw.double()[..., None]
        rowptr, kb = pw.rowptr.cpu().tolist(), pw.kb.cpu().tolist()
        for nb in range(pw.N // 128):
            for p in range(rowptr[nb], rowptr[nb + 1]):
                w[nb * 128:(nb + 1) * 128, kb[p]] += nibbles(rc[p]) * pw.s_r[p].cpu().double()[:, None]
        return w.reshape(pw.N, pw.K)

    def norm(v, gamma):
        return v / torch.sqrt((v * v).mean(-1, keepdim=True) + ex.EPS) * gamma.double().cpu()
    h = x.double().cpu()
    qkv = (norm(h, layer.norm1) @ dense(layer.qkv).t()).view(30, 8, 128)
    k, v = so.values4(qkv[:, 4:6].half()), so.values4(qkv[:, 6:].half())
    h = h + so.attention(qkv[:, :4], k, v, 1 / math.sqrt(128), True).reshape(30, -1) @ dense(layer.o).t()
    gate, up = (norm(h, layer.norm2) @ dense(layer.gate_up).t()).chunk(2, dim=1)
    h = h + (torch.nn.functional.silu(gate) * up) @ dense(layer.down).t()
    out = mq.unpack_weight8(layer.out).double().cpu() * layer.out.s_w.double().cpu()[:, None]
    want = norm(h, layer.norm3) @ out.t()
    cos = torch.nn.functional.cosine_similarity(got, want, dim=1)
    assert cos.min() > 0.98, cos.min()
