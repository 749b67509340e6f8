"""RMS norm with the residual's addition and 8-bit output, against the definition in 64 bits."""
import numpy as np
import pytest
import torch

import serving_oracle as so

pytestmark = pytest.mark.gpu
EPS = 1e-5
DTYPES = [torch.float16, torch.bfloat16]


def mq():
    import paper_2606_15652_amd as m
    return m


def check(x, gamma, r, layout, eps=EPS):
    """Runs the operator and checks h exactly, scales and codes against their definition."""
    m = mq()
    M, K = x.shape
    got = m.rms_norm_quantize8(x.cuda(), gamma.cuda(), eps, residual=None if r is None else r.cuda(), layout=layout)
    codes = m.unpack_act8(got[0]).cpu() if layout == "a8" else got[0].cpu()
    s = got[1].cpu()
    h, y = so.norm(x, gamma, eps, r)
    if r is not None:
        assert torch.equal(got[2].cpu(), h)
    assert s.dtype == (torch.float16 if layout == "a8" else torch.float32)
    s64 = y.abs().amax(-1) / 127
    # fp32: the sum of K squares by lanes of at most 64 and their tree, the root and three products
    rel = (64 + 10 + 8) * 2.0 ** -24
    if layout == "a8":
        assert ((s.double() - s64).abs() <= (2.0 ** -11 + rel) * s64 + 2.0 ** -25).all()
    else:
        assert ((s.double() - s64).abs() <= rel * s64).all()
    # a code is the nearest integer of y over the scale that is held (rows: over the exact one, which the kernel does
    # not depend on): half a step and the quotient's error of a few fp32 units of 127
    held = s.double() if layout == "a8" else s64
    ratio = torch.where(held[:, None] > 0, y / torch.where(held > 0, held, 1.0)[:, None], torch.zeros_like(y))
    off = (codes.double() - ratio.clamp(-127, 127)).abs()
    assert off.max() <= 0.5 + 127 * (rel + 4 * 2.0 ** -24), off.max()
    return got


@pytest.mark.parametrize("layout", ["rows", "a8"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,K", [(1, 128), (3, 512), (64, 1024), (5, 4096), (2, 14336), (1, 16512), (2, 32768), (1, 65536), (777, 640)])
def test_norm(M, K, dtype, layout):
    g = so.generator(M, K)
    gamma = (1 + 0.2 * torch.randn(K, generator=g)).to(dtype)
    check(so.acts(M, K, dtype, 1), gamma, so.acts(M, K, dtype, 2, 0.5), layout)
    check(so.acts(M, K, dtype, 3), gamma, None, layout)


@pytest.mark.parametrize("K", [8, 24, 40, 1000, 5128, 16392, 40008])
def test_odd_widths_in_rows(K):
    x, r = so.acts(9, K, torch.float16, 1), so.acts(9, K, torch.float16, 2)
    codes, s, h = check(x, torch.ones(K).half(), r, "rows")
    assert codes.shape == (9, K) and codes.stride(0) == -(-K // 16) * 16
    # what lies between a row's end and the next is zero
    assert not codes.as_strided((9, codes.stride(0)), (codes.stride(0), 1))[:, K:].any()


def test_strided_and_in_place():
    m = mq()
    x, r, w = so.acts(33, 520, torch.float16, 1), so.acts(33, 520, torch.float16, 2), torch.ones(512).half()
    want = check(x[:, :512], w, r[:, 8:], "rows")
    xd, rd = x.cuda(), r.cuda()
    for target in (xd[:, :512], rd[:, 8:]):                # H over X, then over the residual
        got = m.rms_norm_quantize8(xd[:, :512] if target.data_ptr() == xd.data_ptr() else x.cuda()[:, :512], w.cuda(), EPS,
                                   residual=rd[:, 8:], out=(torch.empty_like(want[0]), torch.empty_like(want[1]), target))
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.equal(target, want[2])


@pytest.mark.parametrize("layout", ["rows", "a8"])
def test_zero_and_non_finite_rows(layout):
    m = mq()
    x = so.acts(8, 512, torch.bfloat16, 1)
    x[0] = 0
    x[2, 17] = float("inf")
    x[4, 511] = float("nan")
    x[6, 3] = 3e38                                          # its square passes fp32's range
    codes, s = m.rms_norm_quantize8(x.cuda(), torch.ones(512).bfloat16().cuda(), EPS, layout=layout)
    codes = m.unpack_act8(codes) if layout == "a8" else codes
    assert s[0] == 0 and not codes[0].any()
    for row in (2, 4, 6):
        assert torch.isnan(s[row]) and not codes[row].any()
    for row in (1, 3, 5, 7):
        assert torch.isfinite(s[row]) and codes[row].abs().max() == 127


def test_empty():
    codes, s, h = mq().rms_norm_quantize8(torch.empty(0, 256).half().cuda(), torch.ones(256).half().cuda(), EPS,
                                          residual=torch.empty(0, 256).half().cuda())
    assert codes.shape == (0, 256) and s.shape == (0,) and h.shape == (0, 256)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,K", [(1, 8), (7, 1000), (130, 4096), (2, 28672)])
def test_quantize_rows8(M, K, dtype):
    x = so.acts(M, K, dtype, 5)
    x[0] = 0
    codes, s = mq().quantize_rows8(x.cuda())
    s32 = x.float().abs().amax(-1) / 127
    assert torch.equal(s.cpu(), s32)
    ratio = torch.where(s32[:, None] > 0, x.double() / torch.where(s32 > 0, s32, 1.0).double()[:, None], torch.zeros(M, K).double())
    assert (codes.cpu().double() - ratio).abs().max() <= 0.5 + 127 * 4 * 2.0 ** -24


@pytest.mark.parametrize("dtype", DTYPES)
def test_dequantize(dtype):
    m = mq()
    x = so.acts(21, 1024, torch.float16, 7)
    codes, s = m.quantize_rows8(x.cuda()[:, :1000])
    want = (codes.double() * s.double()[:, None]).to(dtype)
    assert torch.equal(m.dequantize_act8(codes, s, "rows", dtype), want)
    a8, sa = m.quantize_act8(x.cuda())
    want = (m.unpack_act8(a8).double() * sa.double()[:, None]).to(dtype)
    assert torch.equal(m.dequantize_act8(a8, sa, "a8", dtype), want)


def test_feeds_the_w4a8_layer():
    """The A8 operand written by the norm gives what quantising the same codes again gives."""
    import oracle
    m = mq()
    x, w = so.acts(19, 512, torch.float16, 1), torch.ones(512).half()
    codes, s = m.rms_norm_quantize8(x.cuda(), w.cuda(), EPS, layout="a8")
    again = m.repack_act8(m.unpack_act8(codes))
    assert torch.equal(codes, again)
    W = np.random.default_rng(3).standard_normal((256, 512)).astype(np.float32)
    pw = m.prepare_weight(torch.from_numpy(W).cuda(), 3)
    y = m.fused_gemm_a8(codes, s, pw).cpu().double()
    _, _, y64 = oracle.linear_a8(m.unpack_act8(codes).cpu().numpy(), s.cpu().view(torch.int16).numpy().view(np.uint16),
                                 oracle.prepare_weight(W, 3))
    assert np.abs(y.numpy() - y64).max() <= 2e-3 * np.abs(y64).max()


def test_another_stream():
    m = mq()
    x, w, r = so.acts(64, 4096, torch.float16, 1).cuda(), torch.ones(4096).half().cuda(), so.acts(64, 4096, torch.float16, 2).cuda()
    want = m.rms_norm_quantize8(x, w, EPS, residual=r)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    got = m.rms_norm_quantize8(x, w, EPS, residual=r, stream=stream)
    stream.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_refusals():
    m = mq()
    x, w = torch.zeros(4, 512).half().cuda(), torch.ones(512).half().cuda()
    for error, call in [
        (TypeError, lambda: m.rms_norm_quantize8(x.float(), w.float(), EPS)),
        (TypeError, lambda: m.rms_norm_quantize8(x, w.bfloat16(), EPS)),
        (TypeError, lambda: m.rms_norm_quantize8(x.cpu(), w, EPS)),
        (ValueError, lambda: m.rms_norm_quantize8(x, w[:256].contiguous(), EPS)),
        (ValueError, lambda: m.rms_norm_quantize8(x, w, EPS, residual=x[:3])),
        (TypeError, lambda: m.rms_norm_quantize8(x, w, EPS, residual=x.bfloat16())),
        (ValueError, lambda: m.rms_norm_quantize8(x.t(), torch.ones(4).half().cuda(), EPS)),
        (KeyError, lambda: m.rms_norm_quantize8(x, w, EPS, layout="columns")),
        (m.MQError, lambda: m.rms_norm_quantize8(x, w, -1.0)),
        (m.MQError, lambda: m.rms_norm_quantize8(x[:, :508], w[:508].contiguous(), EPS)),          # not a multiple of 8
        (m.MQError, lambda: m.rms_norm_quantize8(x[:, 4:500], w[4:500].contiguous(), EPS)),        # rows not aligned
        (m.MQError, lambda: m.rms_norm_quantize8(x[:, :320], w[:320].contiguous(), EPS, layout="a8")),
    ]:
        with pytest.raises(error):
            call()


def test_scales_are_rounded_to_single_first():
    """As the other quantisers' scales are.  Of 65536 rows about eight lie where one rounding alone gives the other
    neighbour; the definition's own error, below 2^-50, moves a row over a tie of fp32 once in some thousand runs."""
    m = mq()
    x = so.acts(65536, 128, torch.float16, 5)
    gamma = (1 + 0.2 * torch.randn(128, generator=so.generator(128, 6))).half()
    s = m.rms_norm_quantize8(x.cuda(), gamma.cuda(), EPS, layout="a8")[1].cpu()
    s64 = so.norm(x, gamma, EPS, None)[1].abs().amax(-1) / 127
    twice = s64.numpy().astype(np.float32).astype(np.float16)
    assert (twice != s64.numpy().astype(np.float16)).any()  # the rows tell
    assert np.array_equal(s.numpy(), twice)


@pytest.mark.parametrize("size", [1e-36, 1e-37, 2e-38, 1e-38, 1e-39, 1e-40])
def test_tiny_rows(size):
    """bf16 rows down to fp32's subnormal numbers, where 127 over the largest value passes fp32's range: the codes are
    those of the scale that is held."""
    m = mq()
    x = so.acts(6, 520, torch.float32, 11) * 0.01
    x = (x / x.abs().amax(-1, keepdim=True) * size).bfloat16()
    codes, s = m.quantize_rows8(x.cuda())
    held = x.double().abs().amax(-1) / 127
    assert ((s.cpu().double() - held).abs() <= 2.0 ** -23 * held + 2.0 ** -149).all() and (s > 0).all()
    held = s.cpu().double()
    off = (codes.cpu().double() - (x.double() / held[:, None]).clamp(-127, 127)).abs()
    assert off.max() <= 0.5 + 127 * 4 * 2.0 ** -23, off.max()


@pytest.mark.parametrize("layout", ["rows", "a8"])
@pytest.mark.parametrize("eps,x_size,g_size", [(1e-5, 1e-30, 1e-8), (1e-5, 1e-20, 1e-17), (0.0, 1e-37, 1.0), (0.0, 1e-20, 1e-17)])
def test_tiny_products(eps, x_size, g_size, layout):
    """Norms whose h gamma is below 3.7e-37, with and without an eps that hides the row."""
    m = mq()
    x = (so.acts(5, 512, torch.float32, 12) * x_size).bfloat16()
    gamma = ((1 + 0.2 * torch.randn(512, generator=so.generator(512, 13))) * g_size).bfloat16()
    codes, s = m.rms_norm_quantize8(x.cuda(), gamma.cuda(), eps, layout=layout)
    codes = (m.unpack_act8(codes) if layout == "a8" else codes).cpu().double()
    eps = float(np.float32(eps))
    _, y = so.norm(x, gamma, eps)
    top = (x.double() * gamma.double()).abs().amax(-1)
    # h gamma has an absolute 2^-150 of fp32's subnormal numbers; beside it the roundings of the other norms' test
    rel = (64 + 10 + 8) * 2.0 ** -24 + 2.0 ** -150 / top
    s64 = y.abs().amax(-1) / 127
    assert ((s.cpu().double() - s64).abs() <= ((2.0 ** -11 if layout == "a8" else 0.0) + rel) * s64
            + (2.0 ** -25 if layout == "a8" else 2.0 ** -149)).all()
    held = s.cpu().double()
    ratio = torch.where(held[:, None] > 0, y / torch.where(held > 0, held, 1.0)[:, None], torch.zeros_like(y)).clamp(-127, 127)
    off = (codes - ratio).abs()
    assert (off <= 0.5 + 127 * (rel + 4 * 2.0 ** -23)[:, None] + (127 * 2.0 ** -149 / held)[:, None].nan_to_num(0, 0, 0)).all(), off.max()


@pytest.mark.parametrize("layout", ["rows", "a8"])
def test_zeros_without_eps(layout):
    """0 / 0: such a row is not finite, and its codes are 0."""
    m = mq()
    x = so.acts(3, 256, torch.float16, 14)
    x[1] = 0
    codes, s = m.rms_norm_quantize8(x.cuda(), torch.ones(256).half().cuda(), 0.0, layout=layout)
    codes = m.unpack_act8(codes) if layout == "a8" else codes
    assert torch.isnan(s[1]) and not codes[1].any() and torch.isfinite(s[[0, 2]]).all() and codes[[0, 2]].abs().amax() == 127


def test_the_stride_of_a_single_row():
    """One row (or none) is never stepped along: whatever stride the view has."""
    m = mq()
    x, w = so.acts(1, 516, torch.float16, 21).cuda(), torch.ones(512).half().cuda()
    one = torch.zeros(3, 516).half().cuda()
    one[0, :512] = x[0, :512]
    view = one[:1, :512]                                    # its rows 516 apart, if there were more
    want = m.rms_norm_quantize8(x[:, :512].contiguous(), w, EPS, residual=x[:, :512].contiguous())
    got = m.rms_norm_quantize8(view, w, EPS, residual=view)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert torch.equal(m.quantize_rows8(view)[0], m.quantize_rows8(x[:, :512].contiguous())[0])
    out = torch.zeros(2, 516).half().cuda()
    m.dequantize_act8(want[0], want[1], out=out[:1, :512])
    assert torch.equal(out[:1, :512], m.dequantize_act8(want[0], want[1])) and not out[1].any() and not out[0, 512:].any()
    none = torch.zeros(0, 516).half().cuda()[:, :512]
    assert m.rms_norm_quantize8(none, w, EPS)[0].shape == (0, 512)
