"""Memory of calls on a stream of their own: what the launch writes is not memory that the current stream's pending work may be
using, which is where the current stream's pool would take it from."""
import pytest
import torch

import fp8_oracle as fo

pytestmark = pytest.mark.gpu


def pool_of(t):
    """The stream whose pool the tensor's memory is of."""
    at = t.untyped_storage().data_ptr()
    for s in torch.cuda.memory_snapshot():
        if s["address"] <= at < s["address"] + s["total_size"]:
            return s["stream"]
    raise AssertionError("memory of no pool")


def tensors(x):
    return [x] if isinstance(x, torch.Tensor) else [t for y in x for t in tensors(y)] if isinstance(x, (tuple, list)) else []


def weight_parts(pw):
    return [v for v in vars(pw).values() if isinstance(v, torch.Tensor)]


@pytest.fixture
def scratches(monkeypatch):
    import paper_2606_15652_amd as m
    from paper_2606_15652_amd import fp8, serving
    seen, real = [], m._scratch

    def scratch(*args, **more):
        t = real(*args, **more)
        if t is not None:
            seen.append(t)
        return t
    for module in (m, fp8, serving):
        monkeypatch.setattr(module, "_scratch", scratch)
    return seen


def test_results_and_workspaces(scratches):
    import paper_2606_15652_amd as m
    side, here = torch.cuda.Stream(), torch.cuda.current_stream()
    x = torch.randn(70, 14336).half().cuda()
    w = torch.randn(512, 14336).cuda() * 0.01
    lens, table, cu = [700, 900], fo.table_of([700, 900], 64, 1)[0].cuda(), fo.starts([100, 1]).cuda()
    cache8, cache4 = m.kv8_cache(30, 64, 2, 64), m.kv4_cache(30, 64, 2, 64)
    kv_lens = torch.tensor(lens, dtype=torch.int32).cuda()
    q = torch.randn(101, 8, 64).half().cuda()
    logits, u, slots = torch.randn(3, 1000).cuda(), torch.rand(3).cuda(), torch.arange(40).cuda()
    pw8, pwf, pw4 = m.quantize_weight8(w), m.quantize_weight_fp8(w), m.prepare_weight(w, 8)
    code8, codef, code4 = m.quantize_rows8(x), m.quantize_rows_fp8(x), m.quantize_act(x)
    torch.cuda.synchronize()
    calls = [lambda s: m.quantize_rows_fp8(x, stream=s), lambda s: m.gemm_fp8(*codef, pwf, stream=s),
             lambda s: m.unpack_weight_fp8(pwf, stream=s), lambda s: weight_parts(m.quantize_weight_fp8(w, stream=s)),
             lambda s: m.kv8_read(cache8, slots, stream=s), lambda s: m.attention_kv8(q, cache8, table, kv_lens, cu_q=cu, stream=s),
             lambda s: m.sample(logits, u, stream=s), lambda s: m.quantize_rows8(x, stream=s), lambda s: m.gemm_w8a8(*code8, pw8, stream=s),
             lambda s: m.attention_kv4(q, cache4, table, kv_lens, cu_q=cu, stream=s), lambda s: m.kv4_read(cache4, slots, stream=s),
             lambda s: m.quantize_act(x, stream=s), lambda s: m.fused_gemm(*code4, pw4, stream=s), lambda s: m.linear(x, pw4, stream=s),
             lambda s: weight_parts(m.prepare_weight(w, 8, stream=s))]
    for i, call in enumerate(calls):
        for stream in (side, here, None):
            scratches.clear()
            got = tensors(call(stream))
            torch.cuda.synchronize()
            assert got and {pool_of(t) for t in [*got, *scratches]} == {(stream or here).cuda_stream}, i


def test_same_results():
    """On the stream's own memory the calls give what they give on the current stream."""
    import paper_2606_15652_amd as m
    side = torch.cuda.Stream()
    x, w = torch.randn(70, 14336).half().cuda(), torch.randn(512, 14336).cuda() * 0.01
    pw = m.quantize_weight_fp8(w)
    want = m.gemm_fp8(*m.quantize_rows_fp8(x), pw)
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        got = m.gemm_fp8(*m.quantize_rows_fp8(x, stream=side), pw, stream=side)
        side.synchronize()
        assert torch.equal(got, want)
        del got
