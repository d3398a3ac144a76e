"""Host-only checks of the cache, attention and adapter entry points: each call here fails validation (or has
nothing to do), so nothing is launched."""
import ctypes
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2609_39223_amd", "libqf.so")
QF_OK, QF_EINVAL, QF_ESHAPE, QF_EALIGN, QF_ENOTSUP = 0, 1, 2, 3, 4
I, P, F, Z = ctypes.c_int64, ctypes.c_void_p, ctypes.c_float, ctypes.c_size_t
A, B, C, D = P(256), P(512), P(768), P(1024)


class Cache(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("pages", "page", "H", "D")] + [("fmt", ctypes.c_int32)] + \
        [(n, ctypes.c_void_p) for n in ("k_codes", "k_scales", "v_codes", "v_scales", "k_S", "v_S")]


class Seqs(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int64), ("offsets", ctypes.c_void_p), ("lens", ctypes.c_void_p), ("table", ctypes.c_void_p),
                ("cols", ctypes.c_int64), ("max_len", ctypes.c_int64)]


class Adapters(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("n", "r", "N", "K")] + [(n, ctypes.c_void_p) for n in ("A", "B", "scale", "ranks")]


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(LIB):
        pytest.skip("libqf.so not built (run __graft_entry__.build())")
    import torch  # noqa: F401  (same HIP runtime as the GPU path)
    lib = ctypes.CDLL(LIB)
    lib.qf_last_error.restype = ctypes.c_char_p
    return lib


def cache(pages=8, page=16, H=2, D=128, fmt=1, k_codes=A, k_scales=B, v_codes=C, v_scales=D, k_S=A, v_S=B, **_):
    return Cache(pages, page, H, D, fmt, k_codes, k_scales, v_codes, v_scales, k_S, v_S)


def seqs(B_=4, offsets=A, lens=B, table=C, cols=2, max_len=32, **_):
    return Seqs(B_, offsets, lens, table, cols, max_len)


BAD_CACHE = [(dict(fmt=0), QF_EINVAL), (dict(fmt=3), QF_EINVAL), (dict(pages=-1), QF_ESHAPE), (dict(H=-1), QF_ESHAPE),
             (dict(page=8), QF_ENOTSUP), (dict(page=48), QF_ENOTSUP), (dict(page=2048), QF_ENOTSUP), (dict(page=0), QF_ENOTSUP),
             (dict(D=96), QF_ENOTSUP), (dict(D=512), QF_ENOTSUP), (dict(D=0), QF_ENOTSUP), (dict(H=1 << 14), QF_ENOTSUP),
             (dict(pages=1 << 31), QF_ENOTSUP), (dict(k_codes=None), QF_EINVAL), (dict(v_scales=None), QF_EINVAL),
             (dict(k_S=None), QF_EINVAL), (dict(v_S=None), QF_EINVAL), (dict(k_codes=P(8)), QF_EALIGN), (dict(v_scales=P(24)), QF_EALIGN),
             (dict(k_S=P(2)), QF_EALIGN), (dict(v_S=P(6)), QF_EALIGN)]
BAD_SEQS = [(dict(B_=-1), QF_ESHAPE), (dict(cols=-1), QF_ESHAPE), (dict(max_len=-1), QF_ESHAPE), (dict(max_len=1 << 30), QF_ENOTSUP),
            (dict(B_=1 << 28), QF_ENOTSUP), (dict(cols=1 << 31), QF_ENOTSUP), (dict(offsets=None), QF_ESHAPE),
            (dict(lens=None), QF_EINVAL), (dict(table=None), QF_EINVAL), (dict(lens=P(2)), QF_EALIGN), (dict(table=P(6)), QF_EALIGN),
            (dict(offsets=P(4)), QF_EALIGN)]


def calls(L, **kw):
    """The three calls with everything else valid (T = 6 rows)."""
    c, q = cache(**kw), seqs(**kw)
    T, ld, big = kw.get("T", 6), 2 * 128, Z(1 << 40)
    yield L.qf_kv_write(ctypes.byref(c), ctypes.byref(q), I(T), A, I(ld), B, I(ld), None)
    yield L.qf_kv_read(ctypes.byref(c), ctypes.byref(q), I(T), A, I(ld), B, I(ld), None)
    yield L.qf_kv_attention(ctypes.byref(c), ctypes.byref(q), I(T), A, I(8 * 128), I(8), F(1), I(0), B, I(8 * 128), None, P(4096), big, None)


@pytest.mark.parametrize("kw,status", BAD_CACHE + BAD_SEQS + [(dict(T=-1), QF_ESHAPE), (dict(T=1 << 28), QF_ENOTSUP)])
def test_refusals_of_every_call(L, kw, status):
    assert list(calls(L, **kw)) == [status] * 3, L.qf_last_error()


def test_nothing_to_do(L):
    assert list(calls(L, T=0)) == [QF_OK] * 3
    assert list(calls(L, B_=0)) == [QF_OK] * 3
    assert list(calls(L, fmt=2, k_S=None, v_S=None, T=0)) == [QF_OK] * 3
    c, q = cache(), seqs()
    assert L.qf_kv_read(ctypes.byref(c), ctypes.byref(q), I(6), None, I(0), None, I(0), None) == QF_OK
    for fn in (L.qf_kv_write, L.qf_kv_read):
        assert fn(None, ctypes.byref(q), I(6), A, I(256), B, I(256), None) == QF_EINVAL
        assert fn(ctypes.byref(c), None, I(6), A, I(256), B, I(256), None) == QF_EINVAL


def test_write_and_read_operands(L):
    c, q = cache(), seqs()
    for fn in (L.qf_kv_write, L.qf_kv_read):
        def call(K=A, ldk=256, V=B, ldv=256):
            return fn(ctypes.byref(c), ctypes.byref(q), I(6), K, I(ldk), V, I(ldv), None)
        assert call(ldk=248) == QF_ESHAPE and call(ldv=260) == QF_EALIGN and call(K=P(8)) == QF_EALIGN
    assert L.qf_kv_write(ctypes.byref(c), ctypes.byref(q), I(6), None, I(256), B, I(256), None) == QF_EINVAL


def test_attention_operands(L):
    c, n = cache(), Z()

    def call(Q=A, ldq=1024, Hq=8, window=0, O=B, ldo=1024, lse=None, ws=P(4096), nws=1 << 40, T=6, max_len=100000, cols=10000):
        q = seqs(max_len=max_len, cols=cols)
        return L.qf_kv_attention(ctypes.byref(c), ctypes.byref(q), I(T), Q, I(ldq), I(Hq), F(1), I(window), O, I(ldo), lse, ws, Z(nws), None)
    assert call(Hq=7) == QF_ESHAPE and call(Hq=-2) == QF_ESHAPE and call(window=-1) == QF_ESHAPE
    assert call(Hq=2 * 513, ldq=1 << 20, ldo=1 << 20) == QF_ENOTSUP and call(T=1 << 27) == QF_ENOTSUP
    assert call(Hq=0) == QF_OK
    assert call(Q=None) == QF_EINVAL and call(O=None) == QF_EINVAL and call(ldq=1016) == QF_ESHAPE and call(ldo=1028) == QF_EALIGN
    assert call(lse=P(8)) == QF_EALIGN and call(Q=P(8)) == QF_EALIGN
    assert call(nws=16) == QF_EINVAL and b"workspace" in L.qf_last_error()
    assert call(ws=None) == QF_EINVAL and call(ws=P(4100)) == QF_EALIGN
    size = L.qf_kv_attention_workspace_size
    q = seqs(max_len=100000, cols=10000)
    assert size(ctypes.byref(c), ctypes.byref(q), I(6), I(8), I(0), ctypes.byref(n)) == QF_OK and n.value > 0
    long = n.value
    assert size(ctypes.byref(c), ctypes.byref(q), I(6), I(8), I(300), ctypes.byref(n)) == QF_OK and n.value < long
    assert size(ctypes.byref(c), ctypes.byref(q), I(6), I(8), I(0), None) == QF_EINVAL
    assert size(ctypes.byref(c), ctypes.byref(q), I(6), I(9), I(0), ctypes.byref(n)) == QF_ESHAPE
    for w in ((1 << 30) - 1, 1 << 40, (1 << 63) - 1):               # windows longer than any sequence are none
        assert size(ctypes.byref(c), ctypes.byref(q), I(6), I(8), I(w), ctypes.byref(n)) == QF_OK and n.value == long
    q = seqs(max_len=200, cols=10000)                               # short sequences need none
    assert size(ctypes.byref(c), ctypes.byref(q), I(6), I(8), I(0), ctypes.byref(n)) == QF_OK and n.value == 0
    assert size(ctypes.byref(c), ctypes.byref(q), I(0), I(8), I(0), ctypes.byref(n)) == QF_OK and n.value == 0


def test_adapters(L):
    def call(n=3, r=16, N=32, K=64, fA=A, fB=B, scale=C, ranks=None, ids=D, M=5, X=A, ldx=64, base=B, ldb=32, Y=C, ldy=32, f32=0,
             ws=P(4096), nws=1 << 40):
        a = Adapters(n, r, N, K, fA, fB, scale, ranks)
        return L.qf_lora_rows(ctypes.byref(a), ids, I(M), X, I(ldx), base, I(ldb), Y, I(ldy), f32, ws, Z(nws), None)
    assert L.qf_lora_rows(None, D, I(5), A, I(64), None, I(0), C, I(32), 0, P(4096), Z(1 << 20), None) == QF_EINVAL
    assert call(M=0) == QF_OK and call(N=0) == QF_OK
    assert call(n=-1) == QF_ESHAPE and call(N=-1) == QF_ESHAPE and call(K=-8) == QF_ESHAPE and call(M=-1) == QF_ESHAPE
    assert call(r=0) == QF_ENOTSUP and call(r=12) == QF_ENOTSUP and call(r=264) == QF_ENOTSUP
    assert call(K=60, ldx=64) == QF_ESHAPE and call(f32=2) == QF_EINVAL
    assert call(M=1 << 24) == QF_ENOTSUP and call(N=1 << 30, ldb=1 << 30, ldy=1 << 30) == QF_ENOTSUP
    assert call(ids=None) == QF_EINVAL and call(X=None) == QF_EINVAL and call(Y=None) == QF_EINVAL
    assert call(fA=None) == QF_EINVAL and call(fB=None) == QF_EINVAL and call(scale=None) == QF_EINVAL
    assert call(fA=P(8)) == QF_EALIGN and call(fB=P(8)) == QF_EALIGN and call(ids=P(2)) == QF_EALIGN and call(ranks=P(3)) == QF_EALIGN
    assert call(ldx=56) == QF_ESHAPE and call(ldx=68) == QF_EALIGN and call(ldb=24) == QF_ESHAPE and call(ldy=36) == QF_EALIGN
    assert call(base=C, ldb=40) == QF_EINVAL and b"another row stride" in L.qf_last_error()
    assert call(nws=8) == QF_EINVAL and call(ws=None) == QF_EINVAL and call(ws=P(4100)) == QF_EALIGN
    n = Z()
    a = Adapters(3, 16, 32, 64, A, B, C, None)
    assert L.qf_lora_rows_workspace_size(ctypes.byref(a), I(5), ctypes.byref(n)) == QF_OK and n.value >= 5 * 16 * 4
    assert L.qf_lora_rows_workspace_size(ctypes.byref(a), I(5), None) == QF_EINVAL
