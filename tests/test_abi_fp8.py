"""Argument checks of the C calls in 8-bit floating point and of sampling, without a GPU: every call below fails its checks
or is empty, so the fake addresses are never used."""
import ctypes as C
import math

from test_abi import A, INVALID, MISALIGNED, OK, SHAPE, WORKSPACE, lib  # noqa: F401


def test_quantize_rows(lib):
    def f(M=4, K=512, type=0, X=A, ldx=512, Xq=A, ldq=512, s=A, lds=4):
        return lib.mq_quantize_rows_fp8(M, K, type, X, ldx, Xq, ldq, s, lds, None)
    assert f(M=0) == OK
    for bad in (dict(M=-1), dict(K=-8), dict(type=2), dict(type=-1), dict(X=None), dict(Xq=None), dict(s=None)):
        assert f(**bad) == INVALID, bad
    for bad in (dict(K=0), dict(K=510), dict(K=131064, ldx=131064, ldq=131072), dict(ldx=504), dict(ldx=516), dict(ldq=496), dict(ldq=520),
                dict(K=504, ldq=504), dict(lds=3), dict(M=(1 << 24) + 1, lds=1 << 25), dict(M=1 << 24, lds=1 << 24, K=131056, ldx=131056, ldq=131056)):
        assert f(**bad) == SHAPE, bad
    for bad in (dict(X=A + 8), dict(Xq=A + 8), dict(s=A + 2)):
        assert f(**bad) == MISALIGNED, bad


def test_weights(lib):
    assert lib.mq_weight_fp8_bytes(17, 65) == 64 * 128 and lib.mq_weight_fp8_bytes(65, 129) == 128 * 256
    assert lib.mq_weight_fp8_bytes(0, 64) == 0 and lib.mq_weight_fp8_bytes(16, 131057) == 0 and lib.mq_weight_fp8_bytes((1 << 24) + 1, 64) == 0
    assert lib.mq_weight_fp8_bytes(1 << 24, 131056) == (1 << 24) * 131072
    for f in (lambda N=16, K=64, W=A, ld=64, q=A: lib.mq_quantize_weight_fp8(W, N, K, ld, q, A, None),
              lambda N=16, K=64, W=A, ld=64, q=A: lib.mq_repack_weight_fp8(N, K, W, ld, q, None),
              lambda N=16, K=64, W=A, ld=64, q=A: lib.mq_unpack_weight_fp8(N, K, q, W, ld, None)):
        assert f(N=-1) == INVALID and f(W=None) == INVALID and f(q=None) == INVALID
        assert f(N=0) == SHAPE and f(K=131057, ld=131057) == SHAPE and f(ld=63) == SHAPE
        assert f(q=A + 8) == MISALIGNED
    assert lib.mq_quantize_weight_fp8(A, 16, 64, 64, A, None, None) == INVALID
    assert lib.mq_quantize_weight_fp8(A + 2, 16, 64, 64, A, A, None) == MISALIGNED
    assert lib.mq_repack_weight_fp8(1 << 24, 131056, A, 131056, A, None) == SHAPE       # 2^27 blocks of 1024 threads


def test_gemm(lib):
    def f(M=4, N=32, K=64, X=A, ldx=64, sx=A, lds=4, W=A, sw=A, type=0, bias=None, Y=A, ldy=32, ws=None, nb=0):
        return lib.mq_gemm_fp8(M, N, K, X, ldx, sx, lds, W, sw, type, bias, Y, ldy, ws, nb, None)
    assert f(M=0, lds=0) == OK
    for bad in (dict(M=-1), dict(type=3), dict(X=None), dict(sx=None), dict(W=None), dict(sw=None), dict(Y=None)):
        assert f(**bad) == INVALID, bad
    for bad in (dict(N=0), dict(K=0), dict(K=131057, ldx=131072), dict(ldx=48), dict(ldx=72), dict(K=65, ldx=64), dict(ldy=31), dict(lds=3),
                dict(M=(1 << 24) + 1, lds=1 << 25), dict(M=40, lds=40, ldx=70 << 20)):
        assert f(**bad) == SHAPE, bad
    for bad in (dict(X=A + 8), dict(sx=A + 2), dict(W=A + 8), dict(sw=A + 2), dict(bias=A + 1), dict(Y=A + 1), dict(type=2, Y=A + 2)):
        assert f(**bad) == MISALIGNED, bad
    split = 0
    for M, N, K in ((1, 128, 131056), (1, 4096, 4096), (33, 1024, 14336), (70, 300, 14336), (300, 1024, 28672)):
        need = lib.mq_gemm_fp8_workspace_size(M, N, K)
        r, c, s = C.c_int(), C.c_int(), C.c_int()
        assert lib.mq_gemm_fp8_tile(M, N, K, C.byref(r), C.byref(c), C.byref(s)) == OK
        assert (need > 0) == (s.value > 1)
        if need:
            split += 1
            assert f(M=M, N=N, K=K, ldx=131056, lds=M, ldy=N, ws=None) == WORKSPACE
            assert f(M=M, N=N, K=K, ldx=131056, lds=M, ldy=N, ws=A, nb=need - 1) == WORKSPACE
            assert f(M=M, N=N, K=K, ldx=131056, lds=M, ldy=N, ws=A + 8, nb=need) == MISALIGNED
    assert split
    assert lib.mq_gemm_fp8_workspace_size(0, 32, 64) == 0 and lib.mq_gemm_fp8_workspace_size(1 << 25, 32, 64) == 0
    assert lib.mq_gemm_fp8_tile(1, 32, 64, None, C.byref(r), C.byref(s)) == INVALID


def cache(k=A, v=A, ks=A, vs=A, pages=8, page_size=32, heads=2, head_dim=64):
    from paper_2606_15652_amd.fp8 import _CacheStruct8
    return _CacheStruct8(k, v, ks, vs, pages, page_size, heads, head_dim)


BAD_CACHES = [(dict(k=None), INVALID), (dict(vs=None), INVALID), (dict(pages=-1), INVALID), (dict(pages=0), SHAPE),
              (dict(page_size=48), SHAPE), (dict(page_size=16), SHAPE), (dict(page_size=1 << 17), SHAPE), (dict(heads=0), SHAPE),
              (dict(heads=65536), SHAPE), (dict(head_dim=96), SHAPE), (dict(v=A + 8), MISALIGNED), (dict(k=A + 4), MISALIGNED)]


def test_kv8(lib):
    assert lib.mq_kv8_code_bytes(4200, 256, 64, 128) == 4200 * 256 * 64 * 128
    assert lib.mq_kv8_code_bytes(0, 32, 1, 64) == 0

    def append(c=None, B=3, T=3, type=0, K=A, kt=128, kh=64, V=A, vt=128, vh=64, table=A, tp=4, lens=A, cu=A):
        c = cache() if c is None else c
        return lib.mq_kv8_append(C.addressof(c), B, T, type, K, kt, kh, V, vt, vh, table, tp, lens, cu, None)

    def read(c=None, T=3, type=0, K=A, kt=128, kh=64, V=A, vt=128, vh=64, slots=A):
        c = cache() if c is None else c
        return lib.mq_kv8_read(C.addressof(c), T, type, slots, K, kt, kh, V, vt, vh, None)
    for f in (append, read):
        assert f(T=0) == OK
        for bad, status in BAD_CACHES:
            assert f(c=cache(**bad)) == status, bad
        for bad in (dict(T=-1), dict(type=2), dict(K=None), dict(V=None)):
            assert f(**bad) == INVALID, bad
        for bad in (dict(kt=-8), dict(kh=4), dict(vt=130), dict(vh=-64)):
            assert f(**bad) == SHAPE, bad
        for bad in (dict(K=A + 8), dict(V=A + 2)):
            assert f(**bad) == MISALIGNED, bad
    assert read(slots=None) == INVALID and read(slots=A + 4) == MISALIGNED
    assert append(B=0, cu=A) == OK and append(B=0, T=0, cu=None) == OK
    for bad in (dict(B=-1), dict(tp=-1), dict(table=None), dict(lens=None), dict(cu=None, B=2)):
        assert append(**bad) == INVALID, bad
    for bad in (dict(table=A + 2), dict(lens=A + 2), dict(cu=A + 2)):
        assert append(**bad) == MISALIGNED, bad
    assert append(c=cache(heads=65535), B=1 << 20) == SHAPE
    assert lib.mq_kv8_append(None, 1, 1, 0, A, 8, 8, A, 8, 8, A, 1, A, None, None) == INVALID


def test_attention_kv8(lib):
    def f(c=None, B=2, T=2, group=4, max_q=1, max_kv=64, type=0, Q=A, qt=512, qh=64, table=A, tp=4, lens=A, cu=None, scale=0.125,
          causal=1, O=A, ot=512, oh=64, ws=None, nb=0):
        c = cache() if c is None else c
        return lib.mq_attention_kv8(C.addressof(c), B, T, group, max_q, max_kv, type, Q, qt, qh, table, tp, lens, cu, scale, causal,
                                    O, ot, oh, ws, nb, None)
    assert f(B=0, T=0) == OK and f(T=0, cu=A) == OK and f(cu=A, max_q=0) == OK
    for bad, status in BAD_CACHES:
        assert f(c=cache(**bad)) == status, bad
    for bad in (dict(B=-1), dict(T=-1), dict(T=3), dict(group=0), dict(max_q=-1), dict(max_kv=-1), dict(type=2), dict(Q=None),
                dict(table=None), dict(tp=-1), dict(lens=None), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.inf), dict(scale=math.nan),
                dict(O=None)):
        assert f(**bad) == INVALID, bad
    for bad in (dict(max_kv=129), dict(group=1025), dict(qt=-8), dict(qh=60), dict(ot=4), dict(oh=-64),
                dict(cu=A, max_q=1 << 30), dict(B=1 << 20, T=1 << 20, c=cache(heads=65535))):
        assert f(**bad) == SHAPE, bad
    for bad in (dict(Q=A + 8), dict(O=A + 2), dict(table=A + 2), dict(lens=A + 1), dict(cu=A + 2)):
        assert f(**bad) == MISALIGNED, bad
    need = lib.mq_attention_kv8_workspace_size(2, 2, 2, 4, 64, 1, 100000)
    assert need > 0
    long = dict(c=cache(page_size=65536), tp=2, max_kv=100000)
    assert f(**long) == WORKSPACE and f(**long, ws=A, nb=need - 1) == WORKSPACE and f(**long, ws=A + 8, nb=need) == MISALIGNED
    size = lib.mq_attention_kv8_workspace_size
    assert size(1, 1, 1, 1, 96, 1, 1000) == 0 and size(-1, 1, 1, 1, 64, 1, 1000) == 0 and size(1, -1, 1, 1, 64, 1, 1000) == 0
    # many queries over long contexts are taken
    assert f(c=cache(page_size=65536), tp=2, cu=A, B=1, T=131072, max_q=131072, max_kv=131072, table=None) == INVALID


def test_sample(lib):
    def f(rows=3, vocab=100, type=2, x=A, ldx=100, u=A, t=None, t1=1.0, k=None, k1=0, p=None, p1=1.0, m=None, m1=0.0, tokens=A, probs=A):
        return lib.mq_sample(rows, vocab, type, x, ldx, u, t, t1, k, k1, p, p1, m, m1, tokens, probs, None)
    assert f(rows=0) == OK and f(rows=0, t=A, t1=-1.0) == OK
    for bad in (dict(rows=-1), dict(vocab=-1), dict(type=3), dict(x=None), dict(u=None), dict(tokens=None), dict(probs=None), dict(t1=-1.0),
                dict(t1=math.nan), dict(p1=-0.5), dict(p1=math.nan), dict(m1=-0.5), dict(m1=math.nan)):
        assert f(**bad) == INVALID, bad
    for bad in (dict(vocab=0), dict(vocab=(1 << 20) + 1, ldx=1 << 21), dict(ldx=99), dict(rows=1 << 28)):
        assert f(**bad) == SHAPE, bad
    for bad in (dict(x=A + 2), dict(type=0, x=A + 1), dict(u=A + 2), dict(t=A + 2), dict(k=A + 2), dict(p=A + 1), dict(m=A + 2),
                dict(tokens=A + 4), dict(probs=A + 2)):
        assert f(**bad) == MISALIGNED, bad
