"""Product of e4m3 activations and weights with scales for blocks of 128, its quantisers and layouts."""
import copy
import math

import pytest
import torch

import fp8_oracle as fo
import serving_oracle as so

pytestmark = pytest.mark.gpu
E4M3 = torch.float8_e4m3fn
HALF = [torch.float16, torch.bfloat16]


def mq():
    import paper_2606_15652_amd as m
    return m


def groups(k):
    return -(-k // 128)


def codes(rows, cols, g, spread=60.0):
    return (torch.randn(rows, cols, generator=g) * spread).clamp(-448, 448).to(E4M3)


def spread_scales(rows, cols, g):
    return torch.exp2(torch.randint(-6, 7, (rows, cols), generator=g).float()) * (0.01 + 0.01 * torch.rand(rows, cols, generator=g))


def operands(M, N, K, seed=0):
    g = so.generator(M, N, K, seed)
    return codes(M, K, g), spread_scales(M, groups(K), g), codes(N, K, g), spread_scales(groups(N), groups(K), g)


def padded(x, fill=0x7E, more=0):
    """Codes on the GPU in rows of whole 16 bytes and `more`, with the largest number (or `fill`) behind them."""
    M, K = x.shape
    base = torch.full((M, -(-K // 16) * 16 + more), fill, dtype=torch.uint8)
    base[:, :K] = x.view(torch.uint8)
    return base.cuda().view(E4M3)[:, :K]


def by_token(s):
    return s.t().contiguous().cuda().t()


def reference(x, sx, w, sw, rows):
    """(sum, bound of its error in fp32 times 2^24) of the products in 64 bits.

    The matrix unit adds eight neighbouring products at a time and cuts each of them, towards zero, to a whole multiple of
    2^(e - 13), e the sum of the exponents of the largest one's factors: e.g. beside 256 x 256 (e = 16) and its negative, 14.0625
    counts 8, 28.125 counts 24 and 7.03125 nothing.  The largest itself has eight bits and loses none, so a window loses less than
    7 x 2^-13 of its largest product, which is at most the product of the largest factors.  Beyond that a group's 128 products
    are summed in fp32 in some order, the product of the scales is rounded, as many fmas as there are groups follow, and the sums
    of splits or waves."""
    K, N = x.shape[1], w.shape[0]
    a = x[rows].double() * sx[rows].double().repeat_interleave(128, 1)[:, :K]
    b = w.double() * sw.double().repeat_interleave(128, 0)[:N].repeat_interleave(128, 1)[:, :K]
    a, b = a.cuda(), b.cuda()
    window = [torch.nn.functional.pad(t.abs(), (0, -K % 8)).reshape(t.shape[0], -1, 8).amax(-1) for t in (a, b)]
    size = (128 + groups(K) + 10) * (a.abs() @ b.abs().t()) + 7 * 2.0 ** 11 * (window[0] @ window[1].t())
    return (a @ b.t()).cpu(), size.cpu()


def check(M, N, K, dtype=torch.float16, bias=False, seed=0, rows=None):
    m = mq()
    x, sx, w, sw = operands(M, N, K, seed)
    if dtype == torch.float16:
        sx = sx * min(1.0, 16.0 / K ** 0.5) * 0.05                  # within fp16's range
    b = (torch.randn(N, generator=so.generator(N, 1)) * 3).to(dtype) if bias else None
    xd, sd = padded(x), by_token(sx)
    pw = m.repack_weight_fp8(w.cuda(), sw.cuda())
    y = m.gemm_fp8(xd, sd, pw, bias=None if b is None else b.cuda(), out_dtype=dtype)
    assert y.dtype == dtype and y.shape == (M, N)
    i = torch.arange(M) if rows is None else torch.tensor(sorted(rows))
    prod, size = reference(x, sx, w, sw, i)
    want = prod if b is None else prod + b.double()
    # the sums, the bias' addition in fp32, the type's own rounding
    tol = 2.0 ** -24 * size + 2.0 ** -24 * want.abs() + so.UNIT[dtype] * want.abs() * 1.001 + so.TINY[dtype]
    off = (y.cpu()[i].double() - want).abs()
    assert (off <= tol).all(), (off / tol).max()
    return xd, sd, pw, y


@pytest.mark.parametrize("K", [1, 15, 16, 17, 64, 127, 128, 129, 200, 1000, 4096])
@pytest.mark.parametrize("M,N", [(1, 1), (1, 1000), (3, 130), (16, 16), (17, 255), (33, 512), (130, 129)])
def test_sizes(M, N, K):
    check(M, N, K, [torch.float16, torch.bfloat16, torch.float32][(M + N + K) % 3], bias=(M + K) % 2 == 0)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,N,K", [(64, 4096, 4096), (77, 25599, 640), (200, 1024, 5120), (256, 1024, 1024), (300, 513, 2000),
                                   (512, 2048, 192), (1157, 1536, 4096), (2048, 4096, 1024), (2050, 4099, 513)])
def test_larger(M, N, K, dtype):
    check(M, N, K, dtype, bias=True)


@pytest.mark.parametrize("M,N,K", [(1, 14336, 4096), (1, 4096, 14336), (4, 8192, 8192), (8, 28672, 8192), (32, 4096, 28672), (16, 512, 131056)])
def test_decode_shapes(M, N, K):
    check(M, N, K, torch.bfloat16)


def test_large_prefill():
    check(4097, 8200, 4096, torch.float16, bias=True, rows=[0, 1, 127, 128, 255, 256, 2047, 2048, 4095, 4096])


# What the dispatch chooses, one of each kernel: streaming by one, two and four pieces at 16 rows, one and two at 32, and the tiles.
PLANS = [(1, 512, 512, 16, 16, False), (16, 4096, 4096, 16, 32, False), (9, 14336, 1024, 16, 64, False), (30, 512, 512, 32, 16, False),
         (32, 4096, 4096, 32, 32, False)]


@pytest.mark.parametrize("M,N,K,rows,cols,split", PLANS)
def test_streaming_kernels(M, N, K, rows, cols, split):
    assert mq().gemm_fp8_tile(M, N, K) == (rows, cols, 1)
    check(M, N, K, torch.float32, bias=True)


def test_every_tile_is_met():
    """Over a range of sizes the dispatch takes every tile, whole and in splits where it has them; one product of each."""
    m, seen = mq(), {}
    for M in (33, 64, 100, 200, 300, 600, 1200, 2500, 4096):
        for N in (256, 1024, 4096, 8192, 16384):
            for K in (512, 4096, 14336):
                seen.setdefault((m.gemm_fp8_tile(M, N, K)[0:2], m.gemm_fp8_tile(M, N, K)[2] > 1), (M, N, K))
    assert {t for t, _ in seen} >= {(64, 64), (128, 64), (128, 128), (256, 256)} or len({t for t, _ in seen}) >= 3
    assert any(split for _, split in seen)
    for M, N, K in seen.values():
        check(M, N, K, torch.bfloat16, bias=True, rows=range(0, M, max(1, M // 40)))


def test_scales_far_apart():
    """Groups of very different size: each has its own scale, and one that is zero or huge leaves the others be."""
    m = mq()
    x, sx, w, sw = operands(40, 300, 640)
    sx[:, 0], sx[:, 1], sx[:, 2], sw[0, 3], sw[1] = 1e-30, 0.0, 1e3, 0.0, 1e-20
    y = m.gemm_fp8(padded(x), by_token(sx), m.repack_weight_fp8(w.cuda(), sw.cuda()), out_dtype=torch.float32).cpu().double()
    want, size = reference(x, sx, w, sw, torch.arange(40))
    assert ((y - want).abs() <= 2.0 ** -24 * size).all()


def test_nan_stays_in_its_place():
    m = mq()
    x, sx, w, sw = operands(70, 260, 384)
    xb, wb = x.view(torch.uint8).clone(), w.view(torch.uint8).clone()
    xb[5, 200], wb[130, 7] = 0x7F, 0xFF
    sx[9, 1], sw[2, 0] = math.nan, math.nan
    for M in (70, 20):
        y = m.gemm_fp8(padded(xb.view(E4M3)[:M]), by_token(sx[:M]), m.repack_weight_fp8(wb.view(E4M3).cuda(), sw.cuda()))
        want = torch.zeros(M, 260, dtype=torch.bool)
        want[5], want[9], want[:, 130], want[:, 256:] = True, True, True, True
        assert torch.equal(torch.isnan(y.cpu()), want)


def test_codes_behind_the_rows():
    """Whole 16 bytes past K, and rows' neighbours, are not read: NaN there changes nothing."""
    m = mq()
    for M, K in ((5, 144), (70, 144), (300, 4112), (20, 1000 // 16 * 16)):
        x, sx, w, sw = operands(M, 130, K)
        pw = m.repack_weight_fp8(w.cuda(), sw.cuda())
        y = m.gemm_fp8(padded(x), by_token(sx), pw, out_dtype=torch.float32)
        z = m.gemm_fp8(padded(x, 0x7F, more=64), by_token(sx), pw, out_dtype=torch.float32)
        assert torch.isfinite(y).all() and torch.equal(y, z)


@pytest.mark.parametrize("N,K", [(1, 1), (16, 64), (100, 1000), (513, 130), (4096, 512)])
def test_weight_layout(N, K):
    m = mq()
    w = torch.randint(0, 256, (N, K), generator=so.generator(N, K), dtype=torch.uint8)
    pw = m.repack_weight_fp8(w.cuda().view(E4M3), torch.ones(groups(N), groups(K)).cuda())
    assert torch.equal(m.unpack_weight_fp8(pw).view(torch.uint8).cpu(), w)
    pn, pk = -(-N // 64), groups(K) * 2
    want = torch.zeros(pn * 64, pk * 64, dtype=torch.uint8)
    want[:N, :K] = w
    # block, row / 4, piece, row % 4; piece of 64 codes, quarter, code -> block, codes, piece, quarter, row, code
    want = want.reshape(pn, 4, 4, 4, pk, 4, 16).permute(0, 4, 2, 5, 1, 3, 6)
    assert torch.equal(pw.Wq.cpu(), want.reshape(-1))


def quantised(x):
    """Bytes and scales of groups along the last dimension: the definition, its fp32 roundings made one by one."""
    amax = x.abs().amax(-1)
    fine = torch.isfinite(amax)
    s = (torch.where(fine, amax, torch.zeros_like(amax)).double() / 448).float()
    q = (torch.where(fine[..., None], x, torch.zeros_like(x)).double() / s.double()[..., None]).float()
    q = torch.where((s > 0)[..., None], q, torch.zeros_like(q)).clamp(-448, 448)
    b = fo.byte8(fo.round8(q.double()))
    return b, torch.where(fine, s, torch.full_like(s, math.nan))


def same(a, b):
    return torch.equal(torch.nan_to_num(a, nan=-1.0), torch.nan_to_num(b, nan=-1.0))


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("M,K", [(1, 8), (1, 128), (3, 136), (16, 512), (17, 1000), (33, 5000), (200, 4096), (2, 131056)])
def test_quantize_rows(dtype, M, K):
    m = mq()
    x = so.acts(M, K, dtype, 3)
    x[0, :min(K, 128)] = 0
    if M > 2:
        x[1, K - 1], x[2, 5], x[2, 0] = math.inf, math.nan, 1.0
        x[1, :128] = 448.0 * torch.arange(128).to(dtype) / 128
    if dtype == torch.bfloat16 and M > 16:
        x[5] = x[5].float().mul(1e-38).to(dtype)                    # scales in fp32's subnormal range, and rows of them
        x[6] = x[6].float().mul(1e37).to(dtype)
        x[7] = 2.0 ** -133
    q, s = m.quantize_rows_fp8(x.cuda())
    assert q.dtype == E4M3 and q.shape == (M, K) and s.shape == (M, groups(K))
    wide = torch.zeros(M, groups(K) * 128)
    wide[:, :K] = x.float()
    b, want = quantised(wide.view(M, -1, 128))
    assert same(s.cpu(), want)
    assert torch.equal(q.cpu().contiguous().view(torch.uint8), b.view(M, -1)[:, :K])
    if K % 16:                                                      # the padding is there, and zero
        whole = q.cpu()
        ld = -(-K // 16) * 16
        raw = q.untyped_storage().nbytes()
        assert raw >= M * ld and not torch.as_strided(q.view(torch.uint8), (M, ld), (ld, 1))[:, K:].any() and whole.shape[1] == K


@pytest.mark.parametrize("N,K", [(1, 1), (37, 100), (128, 128), (300, 1000), (512, 4096)])
def test_quantize_weight(N, K):
    m = mq()
    w = torch.randn(N, K, generator=so.generator(N, K)) * 0.02
    if N > 200:
        w[:128, :128] = 0
        w[200, 300] = math.inf
        w[128:256, 128:256] *= 1e-37
    pw = m.quantize_weight_fp8(w.cuda())
    wide = torch.zeros(groups(N) * 128, groups(K) * 128)
    wide[:N, :K] = w
    blocks = wide.view(groups(N), 128, groups(K), 128).transpose(1, 2).reshape(groups(N), groups(K), -1)
    b, s = quantised(blocks)
    assert same(pw.s_w.cpu(), s)
    b = b.view(groups(N), groups(K), 128, 128).transpose(1, 2).reshape(groups(N) * 128, -1)[:N, :K]
    assert torch.equal(m.unpack_weight_fp8(pw).view(torch.uint8).cpu(), b)


@pytest.mark.parametrize("M", [1, 20, 300])
def test_quantised_product(M):
    """Both quantisers and the product as a program runs them, odd sizes."""
    m = mq()
    N, K = 777, 1000
    x, w = so.acts(M, K, torch.bfloat16, 1), torch.randn(N, K, generator=so.generator(2)) / K ** 0.5
    q, s = m.quantize_rows_fp8(x.cuda())
    pw = m.quantize_weight_fp8(w.cuda())
    y = m.gemm_fp8(q, s, pw, out_dtype=torch.bfloat16).cpu().double()
    prod, size = reference(q.cpu(), s.cpu(), m.unpack_weight_fp8(pw).cpu(), pw.s_w.cpu(), torch.arange(M))
    assert ((y - prod).abs() <= 2.0 ** -24 * size + 2.0 ** -8 * 1.001 * prod.abs()).all()
    # and near the product of what was quantised: two roundings of half a step of 2^-4 each at most
    full, mags = x.double() @ w.double().t(), x.double().abs() @ w.double().abs().t()
    assert ((y - full).abs() <= (2 * 2.0 ** -4 + 2.0 ** -8) * mags + 2.0 ** -8 * full.abs()).all()


def test_strides_stream_workspace_graph_and_copies():
    m = mq()
    xd, sx, pw, y = check(70, 300, 14336)
    assert m.gemm_fp8_workspace_bytes(70, 300, 14336) > 0
    out = torch.full((70, 304), 5.0, dtype=torch.float16, device="cuda")
    m.gemm_fp8(xd, sx, pw, out=out[:, :300])
    assert torch.equal(out[:, :300], y) and (out[:, 300:] == 5).all()
    out = torch.full((70, 301), 5.0, dtype=torch.float16, device="cuda")                # rows at odd addresses
    m.gemm_fp8(xd, sx, pw, out=out[:, 1:], workspace=torch.full((m.gemm_fp8_workspace_bytes(70, 300, 14336),), 255, dtype=torch.uint8, device="cuda"))
    assert torch.equal(out[:, 1:], y) and (out[:, 0] == 5).all()
    wide = torch.zeros(112, 75, device="cuda").t()                                       # scales with a stride of their own
    wide[2:72] = sx
    assert torch.equal(m.gemm_fp8(xd, wide[2:72], pw), y)
    assert torch.equal(m.gemm_fp8(xd, sx, copy.deepcopy(pw)), y)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    again = m.gemm_fp8(xd, sx, pw, stream=stream)
    stream.synchronize()
    assert torch.equal(again, y)
    x = so.acts(70, 14336, torch.float16, 5).cuda()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = m.gemm_fp8(*m.quantize_rows_fp8(x), pw)
    for seed in range(3):
        x.copy_(so.acts(70, 14336, torch.float16, seed))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, m.gemm_fp8(*m.quantize_rows_fp8(x), pw))
    q, s = m.quantize_rows_fp8(x)
    into = (torch.zeros(70, 14352, dtype=torch.uint8, device="cuda").view(E4M3)[:, :14336], torch.zeros(112, 80, device="cuda").t()[:70])
    m.quantize_rows_fp8(x, out=into)
    assert torch.equal(into[0].view(torch.uint8), q.view(torch.uint8)) and torch.equal(into[1], s)
    assert m.gemm_fp8(q[:0], s[:0], pw).shape == (0, 300)


def test_far_rows():
    """Rows of X more than 2 GB apart in a tile, and a weight past 2 GB."""
    m = mq()
    K, ld = 256, 70 << 20
    x, sx, w, sw = operands(40, 130, K)
    base = torch.zeros(39 * ld + K, dtype=torch.uint8, device="cuda")
    far = torch.as_strided(base, (40, K), (ld, 1))
    far.copy_(x.view(torch.uint8))
    pw = m.repack_weight_fp8(w.cuda(), sw.cuda())
    with pytest.raises(m.MQError):
        m.gemm_fp8(far.view(E4M3), by_token(sx), pw)
    near = torch.as_strided(base, (33, K), (ld, 1))[:16]
    y = m.gemm_fp8(near.view(E4M3), by_token(sx[:16]), pw, out_dtype=torch.float32)
    assert torch.equal(y, m.gemm_fp8(padded(x[:16]), by_token(sx[:16]), pw, out_dtype=torch.float32))
    half = torch.zeros(299 * (ld // 2) + K, dtype=torch.uint8, device="cuda")
    x, sx, w, sw = operands(300, 130, K)
    rows = torch.as_strided(half, (300, K), (ld // 2, 1))
    rows.copy_(x.view(torch.uint8))
    y = m.gemm_fp8(rows.view(E4M3), by_token(sx), pw, out_dtype=torch.float32)
    assert torch.equal(y, m.gemm_fp8(padded(x), by_token(sx), pw, out_dtype=torch.float32))


def test_refusals():
    m = mq()
    x, sx, w, sw = operands(20, 130, 256)
    xd, sd, pw = padded(x), by_token(sx), m.repack_weight_fp8(w.cuda(), sw.cuda())
    for args, more in (((xd.view(torch.uint8), sd, pw), {}), ((xd[:, :128], sd, pw), {}), ((xd, sd[:10], pw), {}), ((xd, sd.contiguous(), pw), {}),
                       ((xd, sd.half(), pw), {}), ((xd.cpu(), sd, pw), {}), ((xd, sd, pw), {"bias": torch.zeros(130).cuda()}),
                       ((xd, sd, pw), {"bias": torch.zeros(131).half().cuda()}), ((xd, sd, pw), {"out": torch.zeros(19, 130).half().cuda()}),
                       ((xd, sd, pw), {"out_dtype": torch.float64}), ((padded(x, more=8), sd, pw), {})):
        with pytest.raises((TypeError, ValueError)):
            m.gemm_fp8(*args, **more)
    for bad in (torch.zeros(20, 256).cuda(), torch.zeros(20, 2, 128).half().cuda(), torch.zeros(20, 256).half()):
        with pytest.raises((TypeError, ValueError)):
            m.quantize_rows_fp8(bad)
    for bad in (torch.zeros(20, 20).half().cuda(), torch.zeros(20, 250).half().cuda()[:, :248]):
        with pytest.raises(m.MQError):
            m.quantize_rows_fp8(bad)
    with pytest.raises(ValueError):
        m.repack_weight_fp8(w.cuda(), sw[:1].cuda())
    pw.s_w = pw.s_w[:1]
    with pytest.raises(ValueError):
        m.gemm_fp8(xd, sd, pw)
