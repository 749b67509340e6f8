"""W8A8 product with scales for each token and channel, against exact integer sums."""
import pytest
import torch

import serving_oracle as so
from test_abi_serving import W8A8_TILES

pytestmark = pytest.mark.gpu


def mq():
    import paper_2606_15652_amd as m
    return m


def operands(M, N, K, seed=0):
    g = so.generator(M, N, K, seed)
    pad = -(-K // 16) * 16
    x = torch.randint(-128, 128, (M, pad), generator=g, dtype=torch.int8)    # what lies past K counts for nothing
    w = torch.randint(-128, 128, (N, K), generator=g, dtype=torch.int8)
    return x[:, :K], 0.01 + torch.rand(M, generator=g), w, 1e-4 + 1e-3 * torch.rand(N, generator=g)


def check(M, N, K, dtype=torch.float16, bias=False, seed=0, rows=None):
    m = mq()
    x, sx, w, sw = operands(M, N, K, seed)
    b = torch.randn(N, generator=so.generator(N, 1)).to(dtype) if bias else None
    base = torch.empty(M, x.stride(0) if M > 1 else -(-K // 16) * 16, dtype=torch.int8)
    base[:, :K] = x
    base[:, K:] = 77
    xd = base.cuda()[:, :K]
    pw = m.repack_weight8(w.cuda(), sw.cuda())
    y = m.gemm_w8a8(xd, sx.cuda(), pw, bias=None if b is None else b.cuda(), out_dtype=dtype)
    assert y.dtype == dtype and y.shape == (M, N)
    i = torch.arange(M) if rows is None else torch.tensor(sorted(rows))
    # integer sums are exact in double: |sum| <= 128^2 131056 < 2^53
    total = (xd[i.cuda()].double() @ w.cuda().double().t()).cpu()
    prod = total * (sx[i].double()[:, None] * sw.double())
    want = prod if b is None else prod + b.double()
    # the sum in fp32, the product of the scales and with it, the bias: four fp32 roundings, and the type's own
    tol = 4 * 2.0 ** -24 * (prod.abs() + (want - prod).abs()) + so.UNIT[dtype] * want.abs() * 1.001 + so.TINY[dtype]
    off = (y.cpu()[i].double() - want).abs()
    assert (off <= tol).all(), (off / tol).max()
    return xd, sx.cuda(), pw, y


@pytest.mark.parametrize("K", [1, 15, 16, 17, 64, 65, 127, 512, 1000, 4096, 14336])
@pytest.mark.parametrize("M,N", [(1, 1), (1, 1000), (3, 130), (16, 16), (17, 255), (33, 512), (130, 129)])
def test_sizes(M, N, K):
    check(M, N, K, [torch.float16, torch.bfloat16, torch.float32][(M + N + K) % 3], bias=(M + K) % 2 == 0)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,N,K", [(64, 4096, 4096), (77, 25599, 640), (200, 1024, 5120), (256, 1024, 1024), (300, 513, 2000),
                                   (512, 2048, 192), (1157, 1536, 4096), (2048, 4096, 1024), (2050, 4099, 513)])
def test_larger(M, N, K, dtype):
    check(M, N, K, dtype, bias=True)


def test_longest_sums():
    m = mq()
    K = 131056
    x, w = torch.full((2, K), -128, dtype=torch.int8), torch.full((3, K), -128, dtype=torch.int8)
    w[1], w[2] = 127, 0
    y = m.gemm_w8a8(x.cuda(), torch.ones(2).cuda(), m.repack_weight8(w.cuda(), torch.ones(3).cuda()), out_dtype=torch.float32)
    assert torch.equal(y.cpu().double(), torch.tensor([[128.0 * 128 * K, -128.0 * 127 * K, 0.0]] * 2).double())


@pytest.mark.parametrize("M,N,K", [(1, 14336, 4096), (1, 4096, 14336), (4, 8192, 8192), (8, 28672, 8192), (32, 4096, 28672)])
def test_decode_shapes(M, N, K):
    check(M, N, K, torch.bfloat16)


def test_large_prefill():
    check(4097, 8200, 4096, torch.float16, bias=True, rows=[0, 1, 127, 128, 255, 256, 2047, 2048, 4095, 4096])


@pytest.mark.parametrize("N,K", [(1, 1), (16, 64), (100, 1000), (513, 130), (4096, 512)])
def test_weight_layout(N, K):
    m = mq()
    _, _, w, sw = operands(1, N, K, 9)
    pw = m.repack_weight8(w.cuda(), sw.cuda())
    assert torch.equal(m.unpack_weight8(pw).cpu(), w)
    pn, pk = -(-N // 64), -(-K // 128) * 2
    want = torch.zeros(pn * 64, pk * 64, dtype=torch.int8)
    want[:N, :K] = w
    # block, row / 4, piece, row % 4; piece of 64 codes, quarter, code -> block, codes, piece, quarter, row, code
    want = want.reshape(pn, 4, 4, 4, pk, 4, 16).permute(0, 4, 2, 5, 1, 3, 6)
    assert torch.equal(pw.Wq.cpu().view(torch.int8), want.reshape(-1))


@pytest.mark.parametrize("N,K", [(1, 1), (37, 100), (512, 4096)])
def test_quantize_weight(N, K):
    m = mq()
    w = torch.randn(N, K, generator=so.generator(N, K)) * 0.02
    if N > 2:
        w[1] = 0
        w[2, 5] = float("inf")
    pw = m.quantize_weight8(w.cuda())
    codes, s = m.unpack_weight8(pw).cpu(), pw.s_w.cpu()
    s32 = w.abs().amax(-1) / 127
    assert torch.equal(s, s32)
    ok = torch.isfinite(s32) & (s32 > 0)
    assert not codes[~ok].any()
    assert torch.equal(codes[ok], (w[ok] / s32[ok, None]).round().clamp(-127, 127).to(torch.int8))


def test_strided_output_and_stream():
    m = mq()
    xd, sx, pw, y = check(70, 300, 512)
    out = torch.full((70, 304), 5.0, dtype=torch.float16, device="cuda")
    m.gemm_w8a8(xd, sx, pw, out=out[:, :300])
    assert torch.equal(out[:, :300], y) and (out[:, 300:] == 5).all()
    out = torch.full((70, 301), 5.0, dtype=torch.float16, device="cuda")                # rows at odd addresses
    m.gemm_w8a8(xd, sx, pw, out=out[:, 1:])
    assert torch.equal(out[:, 1:], y) and (out[:, 0] == 5).all()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    again = m.gemm_w8a8(xd, sx, pw, stream=stream)
    stream.synchronize()
    assert torch.equal(again, y)


def test_the_same_again():
    xd, sx, pw, y = check(40, 4096, 8192)
    for _ in range(5):
        assert torch.equal(mq().gemm_w8a8(xd, sx, pw), y)


def test_a_scale_that_is_not_finite_stays_in_its_row():
    m = mq()
    xd, sx, pw, y = check(20, 64, 128)
    sx[3] = float("nan")
    z = m.gemm_w8a8(xd, sx, pw)
    assert torch.isnan(z[3]).all() and torch.equal(torch.cat((z[:3], z[4:])), torch.cat((y[:3], y[4:])))


def test_empty():
    m = mq()
    _, _, w, sw = operands(1, 32, 64)
    assert m.gemm_w8a8(torch.empty(0, 64, dtype=torch.int8).cuda(), torch.empty(0).cuda(),
                       m.repack_weight8(w.cuda(), sw.cuda())).shape == (0, 32)


def test_refusals():
    m = mq()
    x, sx, w, sw = operands(4, 32, 64)
    x, sx, pw = x.contiguous().cuda(), sx.cuda(), m.repack_weight8(w.cuda(), sw.cuda())
    odd = torch.zeros(4, 72, dtype=torch.int8).cuda()
    for error, call in [
        (TypeError, lambda: m.gemm_w8a8(x.float(), sx, pw)),
        (TypeError, lambda: m.gemm_w8a8(x, sx.half(), pw)),
        (TypeError, lambda: m.gemm_w8a8(x.cpu(), sx, pw)),
        (ValueError, lambda: m.gemm_w8a8(x, sx[:3], pw)),
        (ValueError, lambda: m.gemm_w8a8(x[:, :48].contiguous(), sx, pw)),
        (ValueError, lambda: m.gemm_w8a8(odd[:, :64], sx, pw)),                         # a row stride of 72
        (ValueError, lambda: m.gemm_w8a8(torch.zeros(64, 4, dtype=torch.int8).cuda().t(), sx, pw)),
        (m.MQError, lambda: m.gemm_w8a8(torch.zeros(4 * 64 + 8, dtype=torch.int8).cuda()[8:].view(4, 64), sx, pw)),
        (TypeError, lambda: m.gemm_w8a8(x, sx, pw, bias=torch.zeros(32).cuda())),
        (ValueError, lambda: m.gemm_w8a8(x, sx, pw, bias=torch.zeros(31).half().cuda())),
        (ValueError, lambda: m.gemm_w8a8(x, sx, pw, out=torch.zeros(4, 31).half().cuda())),
        (TypeError, lambda: m.gemm_w8a8(x, sx, pw, out_dtype=torch.float64)),
        (ValueError, lambda: m.repack_weight8(torch.zeros(2, 131057, dtype=torch.int8).cuda(), sw[:2].cuda())),
        (TypeError, lambda: m.repack_weight8(w.cuda().float(), sw.cuda())),
    ]:
        with pytest.raises(error):
            call()


@pytest.mark.parametrize("M,N,K,ld", [(2, 64, 128, (1 << 31) - 128), (17, 130, 256, 1 << 26), (129, 4096, 144, 69000000),
                                      (300, 5000, 1000, 33947648), (256, 25600, 4096, 33947648), (260, 65536, 128, 16900096)])
def test_rows_far_apart(M, N, K, ld):
    """Activations as a view of a larger tensor, each tile's rows more than 4 GB in all: every kernel and tile."""
    m = mq()
    x, sx, w, sw = operands(M, N, K, 3)
    x, sx, pw = x.contiguous().cuda(), sx.cuda(), m.repack_weight8(w.cuda(), sw.cuda())
    pad = -(-K // 16) * 16
    near = torch.zeros((M, pad), dtype=torch.int8, device="cuda")[:, :K]
    near.copy_(x)
    far = torch.empty((M - 1) * ld + pad, dtype=torch.int8, device="cuda").as_strided((M, K), (ld, 1))
    far.copy_(x)
    assert torch.equal(m.gemm_w8a8(far, sx, pw), m.gemm_w8a8(near, sx, pw))


def test_no_rows_of_an_odd_width():
    m = mq()
    _, _, w, sw = operands(1, 32, 100)
    pw = m.repack_weight8(w.cuda(), sw.cuda())
    assert m.gemm_w8a8(torch.empty(0, 100, dtype=torch.int8).cuda(), torch.empty(0).cuda(), pw).shape == (0, 32)


def test_weights_that_do_not_go_together():
    """Codes and scales of another size than N and K say are refused before a kernel reads past them."""
    m = mq()
    x, sx, w, sw = operands(4, 64, 128)
    x, sx = x.contiguous().cuda(), sx.cuda()
    good = m.repack_weight8(w.cuda(), sw.cuda())
    y = m.gemm_w8a8(x, sx, good)
    short, cpu = good.Wq[:4096], good.Wq.cpu()
    for error, pw in [
        (ValueError, m.PackedWeight8(64, 128, short, good.s_w)),
        (ValueError, m.PackedWeight8(65, 128, good.Wq, good.s_w)),
        (ValueError, m.PackedWeight8(64, 128, good.Wq, good.s_w[:63])),
        (TypeError, m.PackedWeight8(64, 128, good.Wq, good.s_w.half())),
        (TypeError, m.PackedWeight8(64, 128, good.Wq.view(torch.int8), good.s_w)),
        (TypeError, m.PackedWeight8(64, 128, cpu, good.s_w)),
        (ValueError, m.PackedWeight8(0, 128, good.Wq, good.s_w)),
    ]:
        with pytest.raises(error):
            m.gemm_w8a8(x, sx, pw)
        with pytest.raises(error):
            m.unpack_weight8(pw)
    good.Wq = short                                         # replaced after it was used
    with pytest.raises(ValueError):
        m.gemm_w8a8(x, sx, good)
    assert torch.equal(m.gemm_w8a8(x, sx, m.repack_weight8(w.cuda(), sw.cuda())), y)


@pytest.mark.parametrize("shape,expect", W8A8_TILES, ids=[f"M{m}_N{n}_K{k}" for (m, n, k), _ in W8A8_TILES])
def test_every_kernel(shape, expect):
    assert mq().gemm_w8a8_tile(*shape) == expect
    for dtype in (torch.float16, torch.bfloat16, torch.float32):
        check(*shape, dtype, bias=dtype != torch.float32, seed=4)


def test_a_weight_past_32_bits():
    """More than 2^32 codes: laid out, read back, and multiplied."""
    m = mq()
    N, K = 1 << 20, 4112
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    w = torch.randint(-128, 128, (N, K), generator=g, device="cuda", dtype=torch.int8)
    pw = m.repack_weight8(w, torch.ones(N, device="cuda"))
    assert pw.Wq.numel() > 1 << 32 and torch.equal(m.unpack_weight8(pw), w)
    x = torch.randint(-128, 128, (40, K), generator=g, device="cuda", dtype=torch.int8)
    for rows in (3, 40):
        y = m.gemm_w8a8(x[:rows], torch.ones(rows, device="cuda"), pw, out_dtype=torch.float32)
        for n in (0, N // 2 + 77, N - 1):
            assert torch.equal(y[:, n].double(), (x[:rows].double() * w[n].double()).sum(1).float().double())
