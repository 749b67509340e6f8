"""fp32 results of the block-scaled e4m3 product: its sums are fp32's, by every kernel that makes them."""
import math

import pytest
import torch

import serving_oracle as so
from test_gpu_gemm_fp8 import E4M3, by_token, groups, mq, operands, padded

pytestmark = pytest.mark.gpu


def reference(x, sx, w, sw, rows):
    """The products in 64 bits, and 2^24 times the bound of their error in fp32: 128 products of a group (exact; their additions in
    some order, each towards zero perhaps, a step of 2^-23), the product of the scales, a fma for each group, and the sums of up to eight waves or splits."""
    K, N = x.shape[1], w.shape[0]
    a = (x[rows].double() * sx[rows].double().repeat_interleave(128, 1)[:, :K]).cuda()
    b = (w.double() * sw.double().repeat_interleave(128, 0)[:N].repeat_interleave(128, 1)[:, :K]).cuda()
    return (a @ b.t()).cpu(), ((2 * 128 + groups(K) + 10) * (a.abs() @ b.abs().t())).cpu()


def check(M, N, K, x, sx, w, sw, bias=None, rows=None, norm=True):
    m = mq()
    pw = m.repack_weight_fp8(w.cuda(), sw.cuda())
    y = m.gemm_fp8(padded(x), by_token(sx), pw, bias=None if bias is None else bias.cuda(), out_dtype=torch.float32)
    assert y.dtype == torch.float32 and y.shape == (M, N)
    i = torch.arange(M) if rows is None else torch.tensor(rows)
    want, size = reference(x, sx, w, sw, i)
    if bias is not None:
        want = want + bias.double()
    off = (y.cpu()[i].double() - want).abs()
    tol = 2.0 ** -24 * size + 2.0 ** -24 * want.abs()
    assert (off <= tol).all(), (off / tol).max()
    if norm:
        # of one size each and in no order: some tens of roundings of 2^-24 of a sum, far from 1e-5
        assert off.norm() <= 1e-6 * want.norm(), (off.norm() / want.norm()).item()


# Every kernel: streaming by one, two and four pieces, at 16 and 32 rows; 64 x 64, 128 x 64 and 128 x 128, whole and in
# splits; 128 x 128 by two and four slots, and in place of 256 x 256.
PLANS = [(1, 512, 512, (16, 16, 1)), (16, 4096, 4096, (16, 32, 1)), (9, 14336, 1024, (16, 64, 1)), (30, 512, 512, (32, 16, 1)),
         (32, 4096, 4096, (32, 32, 1)), (64, 4096, 1000, (64, 64, 1)), (64, 512, 14336, (64, 64, 4)), (131, 8191, 5000, (128, 64, 1)),
         (300, 8192, 2100, (128, 128, 1)), (1024, 8192, 1000, (128, 128, 1)), (131, 4096, 14336, (128, 128, 4)), (70, 2050, 4000, (128, 64, 4)),
         (33, 8191, 14336, (64, 64, 2)), (70, 8191, 14336, (128, 64, 2)), (257, 4098, 14336, (128, 128, 2)), (1201, 32003, 1000, (256, 256, 1))]


@pytest.mark.parametrize("M,N,K,plan", PLANS)
def test_every_kernel(M, N, K, plan):
    assert mq().gemm_fp8_tile(M, N, K) == plan
    x, sx, w, sw = operands(M, N, K)
    bias = torch.randn(N, generator=so.generator(N)) if M % 2 else None
    check(M, N, K, x, sx, w, sw, bias, rows=None if M * N < 1 << 21 else list(range(0, M, max(1, M // 50))) + [M - 1])


@pytest.mark.parametrize("M", [1, 20, 70, 300])
@pytest.mark.parametrize("K", [8, 128, 1000])
def test_small_products_beside_large_ones(M, K):
    """Eight neighbours whose largest product is 2^16 times the others, and cancels: what is left are the others."""
    N = 130
    g = so.generator(M, K)
    x, w = torch.rand(M, K, generator=g) + 0.5, torch.rand(N, K, generator=g) + 0.5
    x[:, ::8], w[:, ::8] = 256.0, 256.0
    w[:, ::16] = -256.0
    if K == 8:
        w[:, 0] = 0.0
        x[:, 0] = 448.0
    x, w = x.to(E4M3), w.to(E4M3)
    sx, sw = torch.ones(M, groups(K)), torch.ones(groups(N), groups(K))
    check(M, N, K, x, sx, w, sw, norm=False)
    m = mq()
    y = m.gemm_fp8(padded(x), by_token(sx), m.repack_weight_fp8(w.cuda(), sw.cuda()), out_dtype=torch.float32).cpu().double()
    want = x.double() @ w.double().t()
    # all are multiples of 2^-8; sums up to 2^16 (times the neighbours of a group of 128: eight) are then exact in fp32 but for 2^20 2^-24 a step
    assert (y - want).abs().max() <= 0.0625 * K / 8, (y - want).abs().max()


def test_every_code_by_every_code():
    """One product an output: all 254 by 254 finite ones, exactly, and NaN where a code is."""
    m = mq()
    byte = torch.arange(256, dtype=torch.uint8)
    for M in (256, 16):
        x = torch.zeros(256, 16, dtype=torch.uint8)
        x[:, 3] = byte
        w = x.clone()
        pw = m.repack_weight_fp8(w.cuda().view(E4M3), torch.ones(2, 1).cuda())
        y = m.gemm_fp8(padded(x[:M].view(E4M3)), by_token(torch.ones(M, 1)), pw, out_dtype=torch.float32).cpu()
        v = byte.view(E4M3).float()
        want = v[:M, None] * v
        assert torch.equal(torch.isnan(y), torch.isnan(want)) and torch.equal(torch.nan_to_num(y), torch.nan_to_num(want))


@pytest.mark.parametrize("M", [7, 90])
def test_strides_and_graph(M):
    m = mq()
    N, K = 515, 3000
    x, sx, w, sw = operands(M, N, K)
    pw = m.repack_weight_fp8(w.cuda(), sw.cuda())
    xd, sd = padded(x, more=32), by_token(sx)
    y = m.gemm_fp8(xd, sd, pw, out_dtype=torch.float32)
    for first, ld in ((0, 516), (1, 517), (0, 520)):
        out = torch.full((M, ld), math.pi, device="cuda")
        m.gemm_fp8(xd, sd, pw, out=out[:, first:first + N])
        assert torch.equal(out[:, first:first + N], y) and (out[:, first + N:] == math.pi).all() and (out[:, :first] == math.pi).all()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = m.gemm_fp8(xd, sd, pw, out_dtype=torch.float32)
    for seed in range(3):
        x = operands(M, N, K, seed)[0]
        xd.view(torch.uint8).copy_(x.view(torch.uint8))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, m.gemm_fp8(xd, sd, pw, out_dtype=torch.float32))
