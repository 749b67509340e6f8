"""Attention over the 8-bit cache for batches that mix prompts with single tokens, whose contexts several workgroups share."""
import pytest
import torch

import fp8_oracle as fo
from test_gpu_attention_kv8 import HALF, Case, mq

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("dim,heads,group,lens,counts", [
    (128, 1, 8, [900, 1500, 3, 700, 2100, 40, 1, 1999], [300, 1, 1, 0, 1, 5, 1, 130]),
    (64, 2, 4, [2500, 5, 1200, 0, 33], [1, 5, 700, 0, 1]),
    (64, 1, 3, [1500, 1400], [43, 44])])
def test_prompts_among_single_tokens(dtype, dim, heads, group, lens, counts):
    m = mq()
    t = Case(lens, heads, dim, 64, dtype)
    q = t.queries(counts, group)
    most = max(lens)
    need = m.attention_kv8_workspace_bytes(len(lens), sum(counts), heads, group, dim, max(counts), most)
    assert need > 100000                                            # (contexts are shared)
    ws = torch.full((need + 4096,), 255, dtype=torch.uint8, device="cuda")
    o = t.run(q, counts, max_kv=most, workspace=ws[:need])
    assert (ws[need:] == 255).all()
    t.check(q, counts, o)
    # rows without a query of the batch stay, and looser bounds give the same up to the order of sums
    out = torch.full((q.shape[0] + 3, *q.shape[1:]), 7.0, dtype=dtype, device="cuda")
    more = torch.cat((q, q[:3]))
    m.attention_kv8(more.cuda(), t.cache, t.table.cuda(), t.kv_lens.cuda(), cu_q=fo.starts(counts).cuda(), out=out)
    assert (out[q.shape[0]:] == 7).all()
    t.check(q, counts, out[:q.shape[0]])


def test_bounds_far_above():
    """max_q and max_kv of a serving program's largest batch: taken, with the same results."""
    m = mq()
    lens, counts = [300, 40, 1000, 7] * 5, [100, 1, 60, 7] * 5
    t = Case(lens, 1, 128, 64, torch.float16, most=1 << 14)
    q = t.queries(counts, 8)
    t.check(q, counts, t.run(q, counts, max_q=1 << 20))
    assert m.attention_kv8_workspace_bytes(20, sum(counts), 1, 8, 128, 1 << 20, 1 << 20) < 100 << 20


def test_two_graphs_of_one_workspace_size():
    """Two captured batches replayed in turn, lengths changed between: each as its own eager call."""
    m = mq()
    lens, counts = [900, 1500, 3, 700], [300, 1, 1, 130]
    cases = [Case(lens, 1, 64, 64, torch.bfloat16, seed=s) for s in (1, 2)]
    qs = [t.queries(counts, 4, seed=s).cuda() for s, t in enumerate(cases)]
    lens_d = [t.kv_lens.cuda() for t in cases]
    tables, cu = [t.table.cuda() for t in cases], fo.starts(counts).cuda()
    graphs, got = [], []
    for t, q, n, table in zip(cases, qs, lens_d, tables):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got.append(m.attention_kv8(q, t.cache, table, n, cu_q=cu, max_q=300))
        graphs.append(g)
    for new in ([900, 1500, 3, 700], [300, 1, 1, 130], [0, 700, 2, 500]):
        for n in lens_d:
            n.copy_(torch.tensor(new, dtype=torch.int32))
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for t, q, n, table, o in zip(cases, qs, lens_d, tables, got):
            assert torch.equal(o, m.attention_kv8(q, t.cache, table, n, cu_q=cu, max_q=300)), new
