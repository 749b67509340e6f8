"""Strides and sizes that a C int does not hold are refused: cut to their low 32 bits they would name other rows.

Every such view is of memory that is there, and its low 32 bits are a stride that the calls take."""
import pytest
import torch

pytestmark = pytest.mark.gpu
FAR = 2 ** 32 + 256


def mq():
    import paper_2606_15652_amd as m
    return m


def far(rows, cols, dtype):
    """Two rows and more, FAR elements apart."""
    base = torch.empty((rows - 1) * FAR + cols, dtype=dtype, device="cuda")
    x = base.as_strided((rows, cols), (FAR, 1))
    x.view(torch.uint8).zero_() if dtype == torch.float8_e4m3fn else x.zero_()
    return x


def test_rows_of_activations():
    m = mq()
    x = far(2, 256, torch.float16)
    for call in (lambda: m.quantize_rows_fp8(x), lambda: m.quantize_rows8(x), lambda: m.rms_norm_quantize8(x, torch.ones(256).half().cuda())):
        with pytest.raises(ValueError, match="2.31"):
            call()


def test_rows_of_codes_scales_and_results():
    m = mq()
    q, s = m.quantize_rows_fp8(torch.ones(2, 256).half().cuda())
    pw = m.quantize_weight_fp8(torch.ones(64, 256).cuda())
    with pytest.raises(ValueError, match="2.31"):
        m.gemm_fp8(far(2, 256, torch.float8_e4m3fn), s, pw)
    with pytest.raises(ValueError, match="2.31"):
        m.gemm_fp8(q, s, pw, out=far(2, 64, torch.float16))
    wide = far(2, 2, torch.float32).t()
    with pytest.raises(ValueError, match="2.31"):
        m.gemm_fp8(q, wide, pw)
    with pytest.raises(ValueError, match="2.31"):
        m.quantize_rows_fp8(torch.ones(2, 256).half().cuda(), out=(q, wide))
    q8, s8 = m.quantize_rows8(torch.ones(2, 256).half().cuda())
    pw8 = m.quantize_weight8(torch.ones(64, 256).cuda())
    with pytest.raises(ValueError, match="2.31"):
        m.gemm_w8a8(far(2, 256, torch.int8), s8, pw8)
    with pytest.raises(ValueError, match="2.31"):
        m.gemm_w8a8(q8, s8, pw8, out=far(2, 64, torch.float16))


def test_columns():
    """One row of 2^32 + 256 values is not one of 256."""
    m = mq()
    x = torch.empty(1, FAR, dtype=torch.float16, device="cuda")
    with pytest.raises(ValueError, match="2.31"):
        m.quantize_rows_fp8(x)
    with pytest.raises(ValueError, match="2.31"):
        m.sample(x, torch.zeros(1).cuda())


def test_weights():
    m = mq()
    w = torch.empty(1, FAR, dtype=torch.float32, device="cuda")
    for call in (m.quantize_weight_fp8, m.quantize_weight8):
        with pytest.raises(ValueError):
            call(w)


@pytest.mark.parametrize("bits", [4, 8])
def test_queries(bits):
    m = mq()
    cache = (m.kv4_cache if bits == 4 else m.kv8_cache)(1, 32, 1, 64)
    q, table = torch.zeros(3, 1, 64).half().cuda(), torch.zeros(1, 1, dtype=torch.int32).cuda()
    lens, cu = torch.tensor([3], dtype=torch.int32).cuda(), torch.tensor([0, 3], dtype=torch.int32).cuda()
    with pytest.raises(ValueError, match="2.31"):
        (m.attention_kv4 if bits == 4 else m.attention_kv8)(q, cache, table, lens, cu_q=cu, max_q=2 ** 32 + 1)
    many = torch.zeros(1, 1, 64).half().cuda().expand(2 ** 32 + 1, 1, 64)
    slots = torch.zeros(1, dtype=torch.int64).cuda().expand(2 ** 32 + 1)
    with pytest.raises(ValueError):
        if bits == 4:
            m.kv4_append(cache, many, many, slots)
        else:
            m.kv8_append(cache, many, many, table, lens, cu_new=cu)
