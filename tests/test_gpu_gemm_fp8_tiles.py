"""Block-scaled e4m3 product, 16-bit results: every tile whole, in splits and by each number of slots, at sizes that end inside tiles,
pieces and groups; aligned and unaligned rows of the result; weights past 2 and 4 GB."""
import pytest
import torch

import serving_oracle as so
from test_gpu_gemm_fp8 import E4M3, HALF, by_token, check, groups, mq, padded, spread_scales

pytestmark = pytest.mark.gpu

# (rows, columns) of the tile and splits; 128 x 128 has four slots up to 256 workgroups (the first of its two), and two beyond.
PLANS = [(64, 1000, 1000, (64, 64, 1)), (33, 8191, 14333, (64, 64, 2)), (61, 515, 14333, (64, 64, 4)),
         (131, 8191, 5000, (128, 64, 1)), (70, 8191, 14327, (128, 64, 2)), (70, 2050, 4004, (128, 64, 4)),
         (300, 8190, 2111, (128, 128, 1)), (1021, 8191, 1007, (128, 128, 1)), (257, 4098, 14321, (128, 128, 2)), (131, 4095, 14330, (128, 128, 4)),
         (1201, 32003, 1000, (256, 256, 1)), (769, 32003, 5003, (256, 256, 1)), (4095, 8190, 4007, (256, 256, 1)), (4095, 8191, 129, (256, 256, 1)),
         (4096, 8192, 127, (256, 256, 1))]


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("M,N,K,plan", PLANS)
def test_sizes_that_end_inside(M, N, K, plan, dtype):
    m = mq()
    assert m.gemm_fp8_tile(M, N, K) == plan
    rows = None if M * N < 1 << 20 else sorted({0, 1, 15, 16, 17, 63, 64, 127, 128, M // 2, *range(0, M, max(1, M // 12)), M - 2, M - 1} & set(range(M)))
    xd, sd, pw, y = check(M, N, K, dtype, bias=M % 2 == 1, rows=rows)
    bias = (torch.randn(N, generator=so.generator(N, 1)) * 3).to(dtype).cuda() if M % 2 == 1 else None
    # rows 16 bytes apart, at odd addresses, and neither
    for first, ld in ((0, -(-N // 8) * 8), (8, -(-N // 8) * 8 + 16), (1, N + 1), (0, N | 1), (3, (N + 10) | 1)):
        out = torch.full((M, ld), 5.0, dtype=dtype, device="cuda")
        m.gemm_fp8(xd, sd, pw, bias=bias, out=out[:, first:first + N])
        assert torch.equal(out[:, first:first + N], y), (first, ld)
        assert (out[:, :first] == 5).all() and (out[:, first + N:] == 5).all(), (first, ld)


def test_every_tile_is_chosen():
    """All four tiles, the first three in two and four splits too."""
    m, seen = mq(), set()
    for M in (33, 64, 70, 131, 257, 1201, 4096):
        for N in (257, 515, 2050, 4098, 8191, 32003):
            for K in (129, 1000, 4004, 5000, 14336):
                seen.add(m.gemm_fp8_tile(M, N, K))
    assert seen == {plan for *_, plan in PLANS}


@pytest.mark.parametrize("N,K", [(150001, 14336), (33001, 131056)])
def test_weights_past_2_and_4_gb(N, K):
    m = mq()
    g = torch.Generator(device="cuda")
    g.manual_seed(N)
    w = torch.empty(N, K, dtype=torch.uint8, device="cuda")
    for at in range(0, N, 8192):                                    # finite codes of ordinary size, both signs
        w[at:at + 8192] = torch.randint(0, 96, w[at:at + 8192].shape, generator=g, device="cuda", dtype=torch.uint8)
    w[:, ::2] |= 0x80
    assert w.numel() > 1 << (31 if K == 14336 else 32)
    sw = spread_scales(groups(N), groups(K), so.generator(1)).cuda()
    pw = m.repack_weight_fp8(w.view(E4M3), sw)
    rows = torch.cat((torch.arange(0, N, N // 200), torch.arange(N - 70, N))).cuda()
    part, part_s = w[rows].view(E4M3).cpu(), sw.cpu()
    for M in (1, 20, 40, 300):
        x = (torch.randn(M, K, generator=so.generator(M)) * 60).clamp(-448, 448).to(E4M3)
        sx = spread_scales(M, groups(K), so.generator(M, 2)) * 1e-3
        y = m.gemm_fp8(padded(x), by_token(sx), pw, out_dtype=torch.bfloat16)[:, rows].cpu().double()
        # the oracle takes one scale a block of 128 channels: each of the chosen channels as a block of its own
        for i in range(0, len(rows), 90):
            of = rows[i:i + 90].cpu()
            scales = part_s[of // 128]                              # [channels, groups]
            wide = part[i:i + 90].double() * scales.double().repeat_interleave(128, 1)[:, :K]
            a = (x.double() * sx.double().repeat_interleave(128, 1)[:, :K]).cuda()
            b = wide.cuda()
            want = (a @ b.t()).cpu()
            window = [torch.nn.functional.pad(t.abs(), (0, -K % 8)).reshape(t.shape[0], -1, 8).amax(-1) for t in (a, b)]
            size = ((128 + groups(K) + 10) * (a.abs() @ b.abs().t()) + 7 * 2.0 ** 11 * (window[0] @ window[1].t())).cpu()
            off = (y[:, i:i + 90] - want).abs()
            assert (off <= 2.0 ** -24 * size + so.UNIT[torch.bfloat16] * 1.001 * want.abs()).all(), (M, i)
    assert torch.equal(m.unpack_weight_fp8(pw).view(torch.uint8), w)
