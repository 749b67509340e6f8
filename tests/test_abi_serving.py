"""Argument checks of the C calls around the layers, without a GPU: every call below fails its checks
or is empty, so the fake addresses are never used."""
import ctypes as C

import pytest

from test_abi import A, INVALID, MISALIGNED, OK, SHAPE, WORKSPACE, lib  # noqa: F401


def test_rms_norm_quantize8(lib):
    def f(M=4, K=512, type=0, X=A, ldx=512, R=A, ldr=512, gamma=A, eps=1e-5, H=A, ldh=512, layout=0, Xq=A, ldq=512, s=A):
        return lib.mq_rms_norm_quantize8(M, K, type, X, ldx, R, ldr, gamma, eps, H, ldh, layout, Xq, ldq, s, None)
    assert f(M=0) == OK
    for bad in (dict(M=-1), dict(type=2), dict(type=-1), dict(layout=2), dict(eps=-1.0), dict(eps=float("nan")), dict(X=None),
                dict(gamma=None), dict(Xq=None), dict(s=None), dict(R=None), dict(H=None)):
        assert f(**bad) == INVALID, bad
    for bad in (dict(K=508), dict(K=0), dict(K=65544, ldx=65544, ldr=65544, ldh=65544, ldq=65552), dict(ldx=504), dict(ldx=516),
                dict(ldr=500), dict(ldh=500), dict(ldq=504), dict(ldq=520), dict(layout=1, K=520, ldx=520, ldr=520, ldh=520)):
        assert f(**bad) == SHAPE, bad
    for bad in (dict(X=A + 2), dict(R=A + 8), dict(gamma=A + 4), dict(H=A + 8), dict(Xq=A + 8), dict(s=A + 2), dict(layout=1, s=A + 1)):
        assert f(**bad) == MISALIGNED, bad


def test_rows8(lib):
    q = lib.mq_quantize_rows8
    assert q(0, 512, 0, None, 512, None, 512, None, None) == OK
    assert q(4, 512, 2, A, 512, A, 512, A, None) == INVALID
    assert q(4, 512, 0, A, 510, A, 512, A, None) == SHAPE
    assert q(4, 512, 0, None, 512, A, 512, A, None) == INVALID
    assert q(4, 512, 0, A + 8, 512, A, 512, A, None) == MISALIGNED
    d = lib.mq_dequantize_act8
    assert d(0, 512, 0, None, 512, None, 0, None, 512, None) == OK
    assert d(4, 512, 0, A, 512, A, 2, A, 512, None) == INVALID
    assert d(4, 512, 3, A, 512, A, 0, A, 512, None) == INVALID
    assert d(4, 512, 0, A, 512, A, 0, A, 508, None) == SHAPE
    assert d(4, 512, 0, A, 512, A, 0, None, 512, None) == INVALID
    assert d(4, 512, 0, A, 512, A, 0, A + 2, 512, None) == MISALIGNED


def test_weight8(lib):
    assert lib.mq_weight8_bytes(17, 65) == 64 * 128 and lib.mq_weight8_bytes(65, 129) == 128 * 256
    assert lib.mq_weight8_bytes(0, 64) == 0 and lib.mq_weight8_bytes(16, 131057) == 0
    assert lib.mq_weight8_bytes(1 << 24, 131056) == (1 << 24) * 131072
    for f in (lambda N=16, K=64, W=A, ld=64, q=A: lib.mq_quantize_weight8(W, N, K, ld, q, A, None),
              lambda N=16, K=64, W=A, ld=64, q=A: lib.mq_repack_weight8(N, K, W, ld, q, None),
              lambda N=16, K=64, W=A, ld=64, q=A: lib.mq_unpack_weight8(N, K, q, W, ld, None)):
        assert f(N=-1) == INVALID and f(W=None) == INVALID and f(q=None) == INVALID
        assert f(N=0) == SHAPE and f(K=131057, ld=131057) == SHAPE and f(ld=63) == SHAPE
        assert f(q=A + 8) == MISALIGNED


def test_gemm_w8a8(lib):
    def f(M=4, N=32, K=64, X=A, ldx=64, sx=A, W=A, sw=A, type=0, bias=None, Y=A, ldy=32, ws=None, nb=0):
        return lib.mq_gemm_w8a8(M, N, K, X, ldx, sx, W, sw, type, bias, Y, ldy, ws, nb, None)
    assert f(M=0) == OK
    for bad in (dict(M=-1), dict(type=3), dict(X=None), dict(sx=None), dict(W=None), dict(sw=None), dict(Y=None)):
        assert f(**bad) == INVALID, bad
    for bad in (dict(N=0), dict(K=0), dict(K=131057, ldx=131072), dict(ldx=48), dict(ldx=72), dict(K=65, ldx=64), dict(ldy=31),
                dict(M=(1 << 24) + 1)):
        assert f(**bad) == SHAPE, bad
    for bad in (dict(X=A + 8), dict(sx=A + 2), dict(W=A + 8), dict(sw=A + 2), dict(bias=A + 1), dict(Y=A + 1), dict(type=2, Y=A + 2)):
        assert f(**bad) == MISALIGNED, bad
    for M, N, K in ((1, 128, 131056), (1, 4096, 4096), (16, 4096, 14336), (300, 1024, 28672)):
        need = lib.mq_gemm_w8a8_workspace_size(M, N, K)
        if need:
            assert f(M=M, N=N, K=K, ldx=131056, ldy=N, ws=None) == WORKSPACE
            assert f(M=M, N=N, K=K, ldx=131056, ldy=N, ws=A, nb=need - 1) == WORKSPACE


def cache(k=A, v=A, kp=A, vp=A, pages=8, page_size=16, heads=2, head_dim=64):
    from paper_2606_15652_amd.serving import _CacheStruct
    return _CacheStruct(k, v, kp, vp, pages, page_size, heads, head_dim)


BAD_CACHES = [(dict(k=None), INVALID), (dict(vp=None), INVALID), (dict(pages=-1), INVALID), (dict(pages=0), SHAPE),
              (dict(page_size=24), SHAPE), (dict(page_size=8), SHAPE), (dict(page_size=1 << 17), SHAPE), (dict(heads=0), SHAPE),
              (dict(heads=65536), SHAPE), (dict(head_dim=96), SHAPE), (dict(v=A + 8), MISALIGNED), (dict(kp=A + 4), MISALIGNED)]


def test_kv4(lib):
    assert lib.mq_kv4_code_bytes(4200, 256, 64, 128) == 4200 * 256 * 64 * 64
    assert lib.mq_kv4_code_bytes(0, 16, 1, 64) == 0

    def append(c=None, T=3, type=0, K=A, kt=128, kh=64, V=A, vt=128, vh=64, slots=A):
        c = cache() if c is None else c
        return lib.mq_kv4_append(C.addressof(c), T, type, K, kt, kh, V, vt, vh, slots, None)

    def read(c=None, T=3, type=0, K=A, kt=128, kh=64, V=A, vt=128, vh=64, slots=A):
        c = cache() if c is None else c
        return lib.mq_kv4_read(C.addressof(c), T, type, slots, K, kt, kh, V, vt, vh, None)
    for f in (append, read):
        assert f(T=0) == OK
        for bad, status in BAD_CACHES:
            assert f(c=cache(**bad)) == status, bad
        for bad in (dict(T=-1), dict(type=2), dict(K=None), dict(V=None), dict(slots=None)):
            assert f(**bad) == INVALID, bad
        for bad in (dict(kt=-8), dict(kh=4), dict(vt=130), dict(vh=-64)):
            assert f(**bad) == SHAPE, bad
        for bad in (dict(K=A + 8), dict(V=A + 2), dict(slots=A + 4)):
            assert f(**bad) == MISALIGNED, bad
    assert lib.mq_kv4_append(None, 1, 0, A, 8, 8, A, 8, 8, A, None) == INVALID


def test_attention_kv4(lib):
    def f(c=None, B=2, T=2, group=4, max_q=1, max_kv=64, type=0, Q=A, qt=512, qh=64, table=A, tp=4, lens=A, cu=None, scale=0.125,
          causal=1, O=A, ot=512, oh=64, ws=None, nb=0):
        c = cache() if c is None else c
        return lib.mq_attention_kv4(C.addressof(c), B, T, group, max_q, max_kv, type, Q, qt, qh, table, tp, lens, cu, scale, causal,
                                    O, ot, oh, ws, nb, None)
    assert f(B=0, T=0) == OK and f(T=0, cu=A) == OK and f(cu=A, max_q=0) == OK
    for bad, status in BAD_CACHES:
        assert f(c=cache(**bad)) == status, bad
    inf, nan = float("inf"), float("nan")
    for bad in (dict(B=-1), dict(T=-1), dict(T=3), dict(group=0), dict(max_q=-1), dict(max_kv=-1), dict(type=2), dict(Q=None),
                dict(table=None), dict(tp=-1), dict(lens=None), dict(scale=0.0), dict(scale=-1.0), dict(scale=inf), dict(scale=nan),
                dict(O=None)):
        assert f(**bad) == INVALID, bad
    for bad in (dict(max_kv=65), dict(group=1025), dict(qt=-8), dict(qh=60), dict(ot=4), dict(oh=-64)):
        assert f(**bad) == SHAPE, bad
    for bad in (dict(Q=A + 8), dict(O=A + 2), dict(table=A + 2), dict(lens=A + 1), dict(cu=A + 2)):
        assert f(**bad) == MISALIGNED, bad
    need = lib.mq_attention_kv4_workspace_size(1, 1, 2, 4, 64, 1, 1 << 20)
    assert need > 0
    long = dict(B=1, T=1, max_kv=1 << 20, tp=1 << 16)
    assert f(**long) == WORKSPACE and f(**long, ws=A, nb=need - 1) == WORKSPACE and f(**long, ws=A + 8, nb=need) == MISALIGNED


@pytest.mark.parametrize("B,H,group,max_q,max_kv", [(1, 8, 4, 1, 1003), (2, 8, 8, 1, 131072), (64, 8, 4, 1, 8191), (4, 8, 4, 2047, 4095),
                                                   (1, 1, 1, 1, 2 ** 31 - 65537), (128, 32, 1, 1, 100), (1, 1, 1, 1, 0)])
def test_attention_workspace_is_small(lib, B, H, group, max_q, max_kv):
    """Two parts of at most 16 columns for each workgroup that the chip holds, or one of 256, and where each sequence begins."""
    size = lib.mq_attention_kv4_workspace_size(B, B * max_q, H, group, 128, max_q, max_kv)
    assert size <= 256 * 256 * 130 * 4 + 4 * B + 32


def test_gemm_w8a8_rows_far_apart(lib):
    """The rows of a wave's loads span less than 2 GB, up to 16 rows (all in one wave) less than 4; what fits is refused
    for its output's address only, what does not before."""
    def f(M, ldx, K=128):
        return lib.mq_gemm_w8a8(M, 32, K, A, ldx, A, A, A, 0, None, A + 1, 32, None, 0, None)
    top = (1 << 31) - 16                                    # the largest leading dimension there is
    for M, ldx in ((1, top), (2, top), (3, top - 112), (16, 286331136), (33, 69273648), (1 << 24, 69273648)):
        assert f(M, ldx) == MISALIGNED, (M, ldx)
    for M, ldx in ((3, top), (16, 286331152), (33, 69273664), (1 << 24, 1 << 27)):
        assert f(M, ldx) == SHAPE, (M, ldx)


def test_attention_kv4_limits(lib):
    """Both sides of the limits that the launches have; what is within them is refused for its queries' address only."""
    def f(B=1, heads=8, group=4, max_q=1, max_kv=64):
        c = cache(heads=heads, page_size=65536)
        T = B * max_q
        return lib.mq_attention_kv4(C.addressof(c), B, T, group, max_q, max_kv, 0, A + 8, 512, 64, A, 1 << 15, A, A, 0.125, 1, A, 512, 64,
                                    None, 0, None)
    # long prompts: whatever the context's length
    for sizes in (dict(group=8, max_q=32768, max_kv=131072), dict(max_q=131072, max_kv=131072), dict(group=8, max_q=131072, max_kv=1 << 20),
                  dict(B=64, max_q=32768 // 64, max_kv=131072), dict(B=16, heads=64, group=1, max_q=8192, max_kv=1 << 17),
                  dict(heads=65535, group=1, max_q=32768, max_kv=4096)):
        assert f(**sizes) == MISALIGNED, sizes
    assert f(heads=65535, group=1, max_q=32769, max_kv=4096) == SHAPE
    # few columns, shared out step by step
    most = (1 << 31) - 65537
    assert f(heads=32, group=1, max_kv=most) == MISALIGNED and f(heads=33, group=1, max_kv=most) == SHAPE
    assert f(B=255, heads=65535, group=1, max_kv=64) == MISALIGNED and f(B=257, heads=65535, group=1, max_kv=64) == SHAPE
    assert f(B=1 << 24, heads=65535, group=1024, max_q=1 << 19, max_kv=most) == SHAPE
    assert lib.mq_attention_kv4_workspace_size(1 << 24, 1, 65535, 1, 64, 1, most) == 0


def test_attention_kv4_defaults_are_within_the_limits(lib):
    """The binding's own bounds, all rows of Q and the whole table: 64 prompts of 512 tokens, tables of 8192."""
    c = cache(heads=8, page_size=64)
    status = lib.mq_attention_kv4(C.addressof(c), 64, 64 * 512, 4, 64 * 512, 8192, 0, A + 8, 512, 64, A, 128, A, A, 0.125, 1, A, 512, 64,
                                  None, 0, None)
    assert status == MISALIGNED


def test_gemm_w8a8_workspace_alignment(lib):
    M, N, K = 64, 4096, 14336                               # splits of K
    need = lib.mq_gemm_w8a8_workspace_size(M, N, K)
    assert need > 0
    for off in (1, 4, 8):
        assert lib.mq_gemm_w8a8(M, N, K, A, K, A, A, A, 0, None, A, N, A + off, need, None) == MISALIGNED


# (M, N, K): output tile and splits of K, one at least for every kernel that the W8A8 product has
W8A8_TILES = [
    ((1, 14336, 4096), (16, 64, 1)), ((4, 8192, 8192), (16, 32, 1)), ((16, 1000, 512), (16, 16, 1)),
    ((32, 4096, 4096), (32, 32, 1)), ((19, 4099, 1000), (32, 32, 1)), ((17, 255, 64), (32, 16, 1)),
    ((130, 129, 14335), (64, 64, 4)), ((257, 1500, 8192), (64, 64, 2)), ((33, 512, 64), (64, 64, 1)),
    ((300, 1024, 28672), (128, 64, 4)), ((65, 3001, 8192), (128, 64, 4)), ((257, 4099, 14336), (128, 64, 2)), ((77, 25599, 640), (128, 64, 1)),
    ((700, 8201, 1000), (128, 128, 1)), ((2050, 4099, 513), (256, 256, 1)),
]


@pytest.mark.parametrize("shape,expect", W8A8_TILES, ids=[f"M{m}_N{n}_K{k}" for (m, n, k), _ in W8A8_TILES])
def test_gemm_w8a8_tile(lib, shape, expect):
    import paper_2606_15652_amd as mq
    assert mq.gemm_w8a8_tile(*shape) == expect
    M, N, _ = shape
    splits = expect[2]
    assert mq.gemm_w8a8_workspace_bytes(*shape) == (0 if splits == 1 else splits * M * -(-N // 64) * 64 * 4)


def test_gemm_w8a8_tile_validation(lib):
    r = C.byref(C.c_int(0))
    f = lib.mq_gemm_w8a8_tile
    assert f(0, 64, 64, r, r, r) == INVALID and f(1, 64, 64, r, r, None) == INVALID and f(1, 64, 64, None, r, r) == INVALID
    assert f(1, 0, 64, r, r, r) == SHAPE and f(1, 64, 131057, r, r, r) == SHAPE


def test_launches_past_32_bits_of_threads(lib):
    """Such launches are cut by the runtime without an error; what fits is refused for an address only."""
    norm = lambda M, K: lib.mq_rms_norm_quantize8(M, K, 0, A + 2, K, None, 0, A, 1e-5, None, 0, 0, A, K, A, None)      # noqa: E731
    rows = lambda M, K: lib.mq_quantize_rows8(M, K, 0, A + 2, K, A, K, A, None)                                        # noqa: E731
    values = lambda M, K: lib.mq_dequantize_act8(M, K, 0, A, K, A, 0, A + 2, K, None)                                  # noqa: E731
    for f in (norm, rows):
        assert f((1 << 22) - 1, 16384) == MISALIGNED and f(1 << 22, 16384) == SHAPE and f(1 << 24, 2048) == MISALIGNED
    assert values((1 << 24) - 1, 2048) == MISALIGNED and values(1 << 24, 2048) == SHAPE and values(1 << 22, 16384) == SHAPE
    c = cache(heads=64, head_dim=128)

    def append(T):
        return lib.mq_kv4_append(C.addressof(c), T, 0, A + 2, 0, 0, A, 0, 0, A, None)

    def read(T):
        return lib.mq_kv4_read(C.addressof(c), T, 0, A, A + 2, 0, 0, A, 0, 0, None)
    most = ((1 << 24) - 1) * 4 // 64 * 4                    # workgroups of four waves of four rows
    for f in (append, read):
        assert f(most) == MISALIGNED and f(most + 1) == SHAPE
    gemm = lambda M, N, K: lib.mq_gemm_w8a8(M, N, K, A, 16, A, A, A, 0, None, A + 1, N, A, 1 << 62, None)              # noqa: E731
    assert gemm(1 << 20, 65536, 16) == MISALIGNED and gemm(1 << 24, 1 << 24, 16) == SHAPE
