"""A weight of one channel: its row's stride says nothing (torch calls it contiguous whatever that is)."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_one_channel_with_a_stride_of_its_own():
    import paper_2606_15652_amd as m
    w = torch.randn(256, 1).cuda().t()
    assert w.shape == (1, 256) and w.stride(0) < 256 and w.is_contiguous()
    plain = w.clone(memory_format=torch.contiguous_format).reshape(256).reshape(1, 256)
    a, b = m.quantize_weight_fp8(w), m.quantize_weight_fp8(plain)
    assert torch.equal(a.Wq, b.Wq) and torch.equal(a.s_w, b.s_w)
    codes = m.unpack_weight_fp8(b)
    odd = codes.view(torch.uint8).as_strided((1, 256), (1, 1)).view(torch.float8_e4m3fn)
    assert torch.equal(m.repack_weight_fp8(odd, b.s_w).Wq, b.Wq)
    a, b = m.quantize_weight8(w), m.quantize_weight8(plain)
    assert torch.equal(a.Wq, b.Wq) and torch.equal(a.s_w, b.s_w)
    assert torch.equal(m.repack_weight8(m.unpack_weight8(b).as_strided((1, 256), (1, 1)), b.s_w).Wq, b.Wq)
