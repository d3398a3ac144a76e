"""GPU parity of the 4-bit cache (written, read back: bit for bit) and of the attention over it against FP64.

Bound of the attention, with u = 2^-23 (the matrix cores' and exponents' roundings need not be to nearest,
so a whole step each): a score is a sum of D products, each exact, then one product with its factor and one
addition, both rounded: |dz| <= (D + 8) u A + 8 u |z| with A the row's largest |scale| sum |q||k| (>= |z|), so e =
(D + 16) u A; NVFP4 queries lose less than 2^-38 of their largest element, below u A.  A probability is off by
e + 2 u relative and by half a step of FP16, 2^-11 relative, or absolutely by 2^-25 in units of 2^-14 of a
reference at most twice the largest: 2^-38 of that.  Rescalings are exact powers of two.  FP32 sums over n
tokens in chains of matrix products, 4 waves and the pieces: (n / 32 + 64) u relative to the sum of
magnitudes.  The normalizer is off by e + (n / 4 + 64) u relative.  bf16 output: 2^-8 relative."""
import numpy as np
import pytest

import workloads
from oracle import serving as sv
from tests import kv_cases as kc
from tests.helpers import bf16_to_f64, from_dev, to_dev

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
U = 2.0 ** -23
BLOCK = kc.BLOCK


@pytest.fixture(scope="module")
def qf():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_39223_amd as qf
    qf.lib()
    return qf


def _wide(x, pad=8, fill=0x7FC0):
    """x's rows in a wider tensor whose other columns hold NaN."""
    w = np.full((x.shape[0], x.shape[1] + pad), fill, np.uint16)
    w[:, :x.shape[1]] = x
    return to_dev(w)[:, :x.shape[1]]


def _cache(qf, fmt, k, v):
    d = lambda a: None if a is None else to_dev(a)  # noqa: E731
    return qf.kv_cache(fmt, d(k[0]), d(k[1]), d(v[0]), d(v[1]), d(k[2]), d(v[2]))


def _seqs(qf, lens, table, offsets=None, max_len=None):
    return qf.kv_sequences(to_dev(np.asarray(lens, np.int32)), to_dev(table), None if offsets is None else to_dev(offsets), max_len)


# ------------------------------------------------------------------------------- the cache
CACHES = [("nvfp4", 1, 64, 16), ("nvfp4", 8, 128, 64), ("nvfp4", 3, 256, 32), ("mxfp4", 1, 64, 1024), ("mxfp4", 5, 128, 16),
          ("mxfp4", 2, 256, 128)]


@pytest.mark.parametrize("fmt,H,D,page", CACHES)
@pytest.mark.parametrize("new", [None, [1, 0, 7, 33, 2], [40, 3, 0, 0, 129]])
def test_write_and_read(qf, fmt, H, D, page, new):
    """Rows into pages of random order; a bad page, a position below zero and one past the table are not kept;
    what belongs to nobody, and all other bytes, stay as they were."""
    rng = np.random.default_rng(H * D + page)
    B = 5
    counts = [1] * B if new is None else new
    n = sum(counts)
    T = n if new is None else n + 3
    lens = [c + int(rng.integers(0, 50)) for c in counts]
    lens[1], lens[2] = counts[1], counts[2] - 1                   # (the latter's first row is at -1)
    cols = max(lens) // page + 1
    pages = B * cols + 2
    table = kc.table(rng, B, cols, pages)
    bad = (lens[3] - 1) // page
    table[3, bad] = [-1, pages, 1 << 30, -(1 << 31)][int(rng.integers(0, 4))]
    lens[4] = cols * page + 1                                     # its last row is past the table
    offsets = None if new is None else kc.offsets_of(new)
    x = [workloads.normal_bf16(rng, (T, H * D)) for _ in range(2)]
    x[0][:, 5] = 0x8000
    if T > 3:
        x[1][1] = 0                                               # blocks of zeros
    g = [np.abs(bf16_to_f64(a)).max() * (0.3 + rng.random(H)) for a in x]   # (some heads saturate)
    g = [a.astype(np.float32) for a in g]
    old = [kc.pool(rng, fmt, pages, H, page, D) for _ in range(2)]
    ref = [sv.quantize_heads(a, H, fmt, b) for a, b in zip(x, g)]
    old = [(o[0], o[1], r[2]) for o, r in zip(old, ref)]
    cache, seqs = _cache(qf, fmt, *old), _seqs(qf, lens, table, offsets)
    qf.kv_write(cache, seqs, _wide(x[0]), _wide(x[1], 16))
    where = sv.places(offsets, lens, table, page, pages, T)
    assert None in where
    got = [from_dev(t) for t in cache._tensors[:4]]
    for i in range(2):
        codes, scales = sv.write(old[i][0], old[i][1], where, ref[i][0], ref[i][1])
        assert np.array_equal(got[2 * i], codes) and np.array_equal(got[2 * i + 1], scales)
    # and back
    out = [torch.full((T, H * D + 8), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    qf.kv_read(cache, seqs, out[0][:, :H * D], out[1][:, :H * D])
    one = torch.full((T, H * D), 7.0, dtype=torch.bfloat16, device="cuda")
    qf.kv_read(cache, seqs, V=one)
    for i in range(2):
        o = from_dev(out[i].view(torch.int16))
        assert bool((out[i][:, H * D:] == 7).all())
        for t, w in enumerate(where):
            want = np.full(H * D, 0x40E0, np.uint16) if w == "nobody" else np.zeros(H * D, np.uint16) if w is None else ref[i][3][t].reshape(-1)
            assert np.array_equal(o[t, :H * D], want), (i, t, w)
    assert torch.equal(one, out[1][:, :H * D])


@pytest.mark.parametrize("fmt", ["nvfp4", "mxfp4"])
def test_write_non_finite(qf, fmt):
    """A NaN makes its block read as NaN; an infinity too in MXFP4, the largest value in NVFP4; other blocks
    are as without it."""
    rng = np.random.default_rng(3)
    H, D, page = 2, 64, 16
    x = workloads.normal_bf16(rng, (2, H * D))
    clean = x.copy()
    x[0, 3], x[1, 70], x[1, 100] = 0x7FC1, 0x7F80, 0xFF80
    S = np.array([0.002, 0.003], np.float32) if fmt == "nvfp4" else None
    out = []
    for a in (x, clean):
        z = np.zeros((2, H, page, D // 2), np.uint8), np.zeros((2, H, page, D // BLOCK[fmt]), np.uint8), S
        cache, seqs = _cache(qf, fmt, z, z), _seqs(qf, [1, 5], np.array([[0], [1]], np.int32))
        qf.kv_write(cache, seqs, to_dev(a), to_dev(a))
        K = torch.empty(2, H * D, dtype=torch.bfloat16, device="cuda")
        qf.kv_read(cache, seqs, K)
        out.append(K.double().cpu().numpy())
    B = BLOCK[fmt]
    block = lambda c: slice(c // B * B, c // B * B + B)  # noqa: E731
    assert np.isnan(out[0][0, block(3)]).all()
    touched = np.zeros((2, H * D), bool)
    touched[0, block(3)] = touched[1, block(70)] = touched[1, block(100)] = True
    assert np.array_equal(out[0][~touched], out[1][~touched])
    if fmt == "mxfp4":
        assert np.isnan(out[0][1, block(70)]).all() and np.isnan(out[0][1, block(100)]).all()
    else:
        top = 448 * 6 * float(S[1])
        assert abs(out[0][1, 70] - top) <= 2.0 ** -8 * top and abs(out[0][1, 100] + top) <= 2.0 ** -8 * top


# ---------------------------------------------------------------------------- the attention
def _check(got_o, got_l, ref, n, D):
    O, lse, big, wv, svv = ref
    some = ~np.isnan(lse) & (lse > -np.inf)
    e = (D + 16) * U * big
    bound = (2 * e + 2.0 ** -11 + (n / 2 + 192) * U)[..., None] * wv + 2.0 ** -37 * svv + 2.0 ** -8 * np.abs(O) + 1e-40
    assert np.all(np.abs(got_o - O)[some] <= bound[some]), float((np.abs(got_o - O) / bound)[some].max())
    lbound = e + (n / 4 + 80) * U + 4 * U * np.abs(np.where(some, lse, 0))
    assert np.all(np.abs(got_l[some] - lse[some]) <= lbound[some]), float((np.abs(got_l[some] - lse[some]) / lbound[some]).max())
    empty = lse == -np.inf
    assert np.all(got_o[empty] == 0) and np.all(got_l[empty] == -np.inf)
    nobody = np.isnan(lse)
    assert np.all(got_o[nobody] == 7) and np.all(got_l[nobody] == 7)


def _attend(qf, cache, seqs, q, H, D, Hq, scale=None, window=0, T=None):
    T = q.shape[0]
    O = torch.full((T, Hq * D + 8), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((T, Hq), 7.0, device="cuda")
    ws = qf.kv_attention_workspace(cache, seqs, T, Hq, window=window)
    ws.fill_(0xFF)
    qf.kv_attention(cache, seqs, q, O[:, :Hq * D], ws, scale=scale, window=window, lse=lse)
    assert bool((O[:, Hq * D:] == 7).all())
    again = torch.full_like(O, 7.0)
    qf.kv_attention(cache, seqs, q, again[:, :Hq * D], ws, scale=scale, window=window)
    assert torch.equal(O.view(torch.int16), again.view(torch.int16))
    return O[:, :Hq * D].double().cpu().numpy().reshape(T, Hq, D), lse.double().cpu().numpy()


def _run(qf, fmt, lens, new, H, G, D, page, window=0, scale=None, max_len=None, seed=0, extra=0, spoil=None):
    rng = np.random.default_rng(seed)
    B = len(lens)
    cols = max(1, -(-max(lens) // page))
    pages = B * cols + 1
    table = kc.table(rng, B, cols, pages)
    offsets = None if new is None else kc.offsets_of(new)
    T = (B if new is None else sum(new)) + extra
    k, v = kc.pool(rng, fmt, pages, H, page, D), kc.pool(rng, fmt, pages, H, page, D)
    if spoil is not None:
        spoil(table, k, v)
    Hq = H * G
    qh = workloads.normal_bf16(rng, (T, Hq * D))
    cache, seqs = _cache(qf, fmt, k, v), _seqs(qf, lens, table, offsets, max_len)
    o, l = _attend(qf, cache, seqs, _wide(qh), H, D, Hq, scale, window)
    K, V = sv.values(*k, fmt), sv.values(*v, fmt)
    ref = sv.attention(bf16_to_f64(qh).reshape(T, Hq, D), K, V, offsets, lens, table, D ** -0.5 if scale is None else scale,
                       window, max_len)
    if offsets is not None:                                        # rows of nobody
        for a in ref[:2]:
            a[int(offsets[-1]):] = np.nan
    _check(o, l, ref, max(lens), D)
    return o, l


LENS = [[1], [16], [17, 63, 64], [65, 2, 255], [256, 257, 0, 1], [1000, 31, 513]]


@pytest.mark.parametrize("fmt", ["nvfp4", "mxfp4"])
@pytest.mark.parametrize("D,page", [(64, 16), (128, 32), (256, 64)])
@pytest.mark.parametrize("lens", LENS)
def test_decode(qf, fmt, D, page, lens):
    _run(qf, fmt, lens, None, 2, 4, D, page, seed=len(lens) + D)


@pytest.mark.parametrize("fmt", ["nvfp4", "mxfp4"])
@pytest.mark.parametrize("G", [1, 3, 5, 16, 17, 40])
def test_heads(qf, fmt, G):
    _run(qf, fmt, [70, 5, 300], None, 3, G, 64, 16, seed=G)
    _run(qf, fmt, [70, 5, 300], [9, 5, 2], 1, G, 128, 16, seed=G)


@pytest.mark.parametrize("fmt,D", [("nvfp4", 64), ("nvfp4", 128), ("nvfp4", 256), ("mxfp4", 64), ("mxfp4", 128), ("mxfp4", 256)])
@pytest.mark.parametrize("lens,new", [([100], [100]), ([70, 130, 40], [5, 1, 40]), ([20, 3, 90, 0], [33, 4, 0, 0]),
                                      ([300, 0, 64], [70, 0, 64]), ([1, 1], [1, 1]), ([400], [2])])
@pytest.mark.parametrize("window", [0, 24])
def test_several_new_tokens(qf, fmt, D, lens, new, window):
    """Causal rows, more new tokens than the sequence has (rows below position zero see nothing), rows of
    nobody at the end, a sliding window."""
    _run(qf, fmt, lens, new, 2, 3, D, 16, window=window, seed=sum(lens), extra=2)


@pytest.mark.parametrize("fmt", ["nvfp4", "mxfp4"])
@pytest.mark.parametrize("window", [1, 2, 63, 64, 65, 100, 5000])
def test_windows(qf, fmt, window):
    _run(qf, fmt, [333, 64, 90], None, 2, 2, 64, 32, window=window, seed=window)


def test_window_of_any_size(qf):
    """Windows longer than any sequence equal none, to the largest that the type holds."""
    want = _run(qf, "nvfp4", [3000, 90], None, 1, 2, 64, 32, seed=3)
    for window in (3000, 1 << 31, (1 << 63) - 1):
        got = _run(qf, "nvfp4", [3000, 90], None, 1, 2, 64, 32, window=window, seed=3)
        assert window == 3000 or all(np.array_equal(a, b) for a, b in zip(want, got))


@pytest.mark.parametrize("fmt", ["nvfp4", "mxfp4"])
def test_long(qf, fmt):
    """Pieces that meet in the merge, pages of 16 (more than 64 a wave), an odd end, a sequence far shorter."""
    _run(qf, fmt, [20011, 37, 1030], None, 1, 4, 64, 16, seed=1)
    _run(qf, fmt, [30007], [3], 1, 5, 128, 64, seed=2)
    _run(qf, fmt, [9001, 200], [40, 7], 1, 2, 64, 16, seed=3, window=8000)
    _run(qf, fmt, [70001], None, 1, 2, 256, 1024, seed=4)


@pytest.mark.parametrize("fmt,D,page", [("nvfp4", 64, 16), ("nvfp4", 128, 64), ("mxfp4", 64, 128), ("mxfp4", 128, 16), ("mxfp4", 256, 32)])
@pytest.mark.parametrize("window", [0, 700])
def test_pieces_of_prompts(qf, fmt, D, page, window):
    """Many new tokens behind many cached ones: every wave's share, more than 64 tiles a piece, row tiles that
    are not full, a sequence that is all new and one without new tokens."""
    _run(qf, fmt, [700, 131, 64, 1500], [300, 131, 0, 257], 1, 4, D, page, window=window, seed=30, extra=3)
    _run(qf, fmt, [5000], [70], 2, 3, D, page, window=window, seed=31)
    _run(qf, fmt, [200, 333], [200, 333], 1, 16, D, page, window=window, seed=32)


@pytest.mark.parametrize("fmt", ["nvfp4", "mxfp4"])
@pytest.mark.parametrize("scale", [0.0, -0.3, 1.0, 1e-30, 6.0])
def test_scales(qf, fmt, scale):
    _run(qf, fmt, [150, 3], None, 2, 2, 64, 16, scale=scale, seed=5)


@pytest.mark.parametrize("fmt", ["nvfp4", "mxfp4"])
def test_max_len(qf, fmt):
    """The bound may be larger than any length; tokens from it on are not seen."""
    _run(qf, fmt, [150, 3], None, 2, 2, 64, 16, max_len=100000, seed=6)
    _run(qf, fmt, [150, 3, 40], None, 2, 2, 64, 16, max_len=100, seed=6)


@pytest.mark.parametrize("fmt", ["nvfp4", "mxfp4"])
def test_many_sequences(qf, fmt):
    """More sequences than one step of the search takes, some without new tokens."""
    rng = np.random.default_rng(8)
    new = [int(v) for v in rng.integers(0, 4, 300)]
    _run(qf, fmt, [n + int(rng.integers(0, 20)) for n in new], new, 1, 4, 64, 16, seed=9, extra=1)
    _run(qf, fmt, [int(v) for v in rng.integers(0, 40, 150)], None, 1, 2, 64, 16, seed=9)


@pytest.mark.parametrize("B", [1, 2, 62, 63, 64, 65, 128])
@pytest.mark.parametrize("many", [4, 60])
def test_numbers_of_sequences(qf, B, many):
    """Around one wave of sequences, the first and last without new tokens or with the most."""
    for ends in (0, many):
        rng = np.random.default_rng(B + ends)
        new = [int(v) for v in rng.integers(0, many, B)]
        new[0], new[-1] = ends, many - ends
        _run(qf, "nvfp4", [n + int(rng.integers(0, 30)) for n in new], new, 1, 4, 64, 16, seed=B, extra=1)


@pytest.mark.parametrize("fmt", ["nvfp4", "mxfp4"])
@pytest.mark.parametrize("new", [None, [20, 1, 40], [100, 16, 150]])
def test_bad_pages(qf, fmt, new):
    """Tokens of a page that is none are not seen."""
    def spoil(table, k, v):
        table[0, 1], table[1, 0], table[2, 2] = -1, table.max() + 100, 1 << 30
    _run(qf, fmt, [100, 16, 150], new, 2, 2, 64, 16, seed=10, spoil=spoil)

    def all_bad(table, k, v):
        table[:] = -5
    _run(qf, fmt, [100, 16, 150], new, 2, 2, 64, 16, seed=10, spoil=all_bad)


@pytest.mark.parametrize("fmt", ["nvfp4", "mxfp4"])
@pytest.mark.parametrize("new,window", [(None, 0), ([9, 30], 0), ([9, 30], 13), (None, 20), ([60, 50], 0), ([60, 50], 13)])
def test_nan_scales(qf, fmt, new, window):
    """Keys and values with NaN scales behind a sequence's end or outside the window are not seen; the ones
    that a row sees make it NaN (a value's block: those outputs alone), and no row before them."""
    rng = np.random.default_rng(12)
    H, G, D, page, B = 2, 3, 128, 16, 2
    lens, cols = [75, 50], 6
    table = kc.table(rng, B, cols, B * cols)
    offsets = None if new is None else kc.offsets_of(new)
    T = B if new is None else sum(new)
    k, v = kc.pool(rng, fmt, B * cols, H, page, D), kc.pool(rng, fmt, B * cols, H, page, D)
    nan = 0x7F if fmt == "nvfp4" else 0xFF

    def at(b, pos):
        return table[b, pos // page], pos % page
    for b in range(B):
        for pos in range(lens[b], cols * page):                     # behind the end: all of it
            p, o = at(b, pos)
            k[1][p, :, o], v[1][p, :, o] = nan, nan
    p, o = at(0, 70)                                                # seen by sequence 0's last rows
    v[1][p, 1, o, 2] = nan
    p, o = at(1, 45)
    k[1][p, 0, o, 1] = nan
    p, o = at(0, 3)                                                 # outside a window
    if window:
        k[1][p, :, o], v[1][p, :, o] = nan, nan
    Hq = H * G
    qh = workloads.normal_bf16(rng, (T, Hq * D))
    o_, l_ = _attend(qf, _cache(qf, fmt, k, v), _seqs(qf, lens, table, offsets), to_dev(qh), H, D, Hq, None, window)
    K, V = sv.values(*k, fmt), sv.values(*v, fmt)
    ref = sv.attention(bf16_to_f64(qh).reshape(T, Hq, D), K, V, offsets, lens, table, D ** -0.5, window)
    assert np.isnan(ref[0]).any() and np.isfinite(ref[0]).any()
    assert np.array_equal(np.isnan(o_), np.isnan(ref[0])) and np.array_equal(np.isnan(l_), np.isnan(ref[1]))
    fine = ~np.isnan(ref[0])
    assert np.all(np.abs(o_ - ref[0])[fine] <= 1e-2 * ref[3][fine] + 1e-30)


def test_values_of_any_scale(qf):
    """MXFP4 values far outside FP16's range, beside ordinary ones, and blocks of zeros under code 0."""
    def spoil(table, k, v):
        rng = np.random.default_rng(1)
        v[1][:] = rng.choice([127, 60, 100, 106, 107, 134, 135, 180, 200], v[1].shape)
        k[1][:, :, :, 0] = 30
    _run(qf, "mxfp4", [150, 33, 64], None, 2, 2, 64, 16, seed=13, spoil=spoil)
    _run(qf, "mxfp4", [150, 33, 64], [20, 3, 64], 2, 3, 128, 16, seed=13, spoil=spoil)
    _run(qf, "mxfp4", [80], [7], 1, 2, 256, 16, seed=13, spoil=spoil)
    _run(qf, "mxfp4", [150, 133], [120, 90], 2, 3, 128, 16, seed=13, spoil=spoil)
    _run(qf, "mxfp4", [150, 133], [120, 90], 1, 5, 64, 32, seed=13, spoil=spoil)

    def tiny(table, k, v):
        v[1][:] = 20
    _run(qf, "mxfp4", [150, 33], None, 2, 2, 64, 16, seed=14, spoil=tiny)

    def zero(table, k, v):
        v[1][..., 0], v[0][..., :16] = 0, 0
    _run(qf, "mxfp4", [150, 33], None, 2, 2, 64, 16, seed=14, spoil=zero)


@pytest.mark.parametrize("fmt", ["nvfp4", "mxfp4"])
def test_queries_of_any_size(qf, fmt):
    """Large, tiny and mixed queries; zeros; a NaN or infinity makes its row NaN and no other."""
    rng = np.random.default_rng(15)
    H, G, D, page, lens = 1, 4, 64, 16, [90, 40, 17]
    table = kc.table(rng, 3, 6, 20)
    k, v = kc.pool(rng, fmt, 20, H, page, D), kc.pool(rng, fmt, 20, H, page, D)
    cache, seqs = _cache(qf, fmt, k, v), _seqs(qf, lens, table)
    K, V = sv.values(*k, fmt), sv.values(*v, fmt)
    for size in (1e30, 1e-30, 2.0 ** -130, 0.0):
        qh = workloads.normal_bf16(rng, (3, H * G * D), size) if size > 1e-37 else np.full((3, H * G * D), 3 if size else 0x8000, np.uint16)
        q = bf16_to_f64(qh).reshape(3, H * G, D)
        scale = 0.1 / max(size, 1e-36)
        o, l = _attend(qf, cache, seqs, to_dev(qh), H, D, H * G, scale)
        _check(o, l, sv.attention(q, K, V, None, lens, table, float(np.float32(scale))), 90, D)
    qh = workloads.normal_bf16(rng, (3, H * G * D))
    qh[:, 7] = 0x7F00                                              # one element 2^127
    q = bf16_to_f64(qh).reshape(3, H * G, D)
    o, l = _attend(qf, cache, seqs, to_dev(qh), H, D, H * G, 2.0 ** -126)
    _check(o, l, sv.attention(q, K, V, None, lens, table, 2.0 ** -126), 90, D)
    qh = workloads.normal_bf16(rng, (3, H * G * D))
    clean, _ = _attend(qf, cache, seqs, to_dev(qh), H, D, H * G)
    qh[0, 5], qh[1, D + 9], qh[2, 3 * D] = 0x7FC0, 0x7F80, 0xFF80
    o, l = _attend(qf, cache, seqs, to_dev(qh), H, D, H * G)
    for t, h in ((0, 0), (1, 1), (2, 3)):
        assert np.isnan(o[t, h]).all() and np.isnan(l[t, h])
        o[t, h] = clean[t, h]
    assert np.array_equal(o, clean)


def test_one_large_score(qf):
    """Scores hundreds apart, the largest first, last or in the middle: nothing overflows, and rows of equal
    scores average."""
    D, page, n = 64, 16, 600
    codes = np.zeros((40, 1, page, D // 2), np.uint8)
    scales = np.full((40, 1, page, D // 32), 127, np.uint8)
    table = np.arange(40, dtype=np.int32)[None]
    vc = np.random.default_rng(0).integers(0, 256, codes.shape).astype(np.uint8)
    qh = np.full((1, D), 0x4200, np.uint16)                        # 32
    for where in (0, 63, 64, 300, 599, None):
        kk = codes.copy()
        if where is not None:
            kk[where // page, 0, where % page] = 0x55              # 3 everywhere: score 768
        k, v = (kk, scales, None), (vc, scales, None)
        o, l = _attend(qf, _cache(qf, "mxfp4", k, v), _seqs(qf, [n], table), to_dev(qh), 1, D, 1)
        K, V = sv.values(*k, "mxfp4"), sv.values(*v, "mxfp4")
        _check(o, l, sv.attention(bf16_to_f64(qh).reshape(1, 1, D), K, V, None, [n], table, D ** -0.5), n, D)


def test_cache_past_4_gib(qf):
    """Pages whose bytes lie past 2^32: written, read back and attended to."""
    H, D, page = 8, 128, 1024
    pages = (1 << 32) // (H * page * D // 2) + 3                   # codes of 4 GiB and a little
    kcodes = torch.zeros(pages, H, page, D // 2, dtype=torch.uint8, device="cuda")
    kscales = torch.zeros(pages, H, page, D // 32, dtype=torch.uint8, device="cuda")
    cache = qf.kv_cache("mxfp4", kcodes, kscales, kcodes.clone(), kscales.clone())
    rng = np.random.default_rng(0)
    x = workloads.normal_bf16(rng, (20, H * D))
    seqs = _seqs(qf, [20], np.array([[pages - 1]], np.int32), np.array([0, 20], np.int64))
    qf.kv_write(cache, seqs, to_dev(x), to_dev(x))
    K = torch.empty(20, H * D, dtype=torch.bfloat16, device="cuda")
    qf.kv_read(cache, seqs, K)
    ref = sv.quantize_heads(x, H, "mxfp4")
    assert np.array_equal(from_dev(K.view(torch.int16)), ref[3].reshape(20, -1))
    xh = bf16_to_f64(ref[3].reshape(20, H * D)).reshape(1, 20, H, D).transpose(0, 2, 1, 3)
    o, l = _attend(qf, cache, seqs, to_dev(x), H, D, H)
    want = sv.attention(bf16_to_f64(x).reshape(20, H, D), xh, xh, np.array([0, 20]), [20], np.zeros((1, 1), np.int32), D ** -0.5, max_len=20)
    # (page 20 of the reference holds the 20 tokens alone)
    _check(o, l, want, 20, D)


# --------------------------------------------------------------- streams, graphs, devices
@pytest.mark.parametrize("fmt", ["nvfp4", "mxfp4"])
def test_graph_of_a_growing_sequence(qf, fmt):
    """One captured step (write, attend) replayed while lens and the table's contents change between the
    replays, against eager calls on the same cache; max_len bounds what the graph provides for."""
    rng = np.random.default_rng(20)
    H, G, D, page, B, cols = 2, 4, 64, 16, 3, 80
    table = kc.table(rng, B, cols, B * cols)
    k, v = kc.pool(rng, fmt, B * cols, H, page, D), kc.pool(rng, fmt, B * cols, H, page, D)
    caches = [_cache(qf, fmt, k, v) for _ in range(2)]
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    seqs = qf.kv_sequences(lens, to_dev(table), max_len=cols * page)
    x = [torch.empty(B, w, dtype=torch.bfloat16, device="cuda") for w in (H * D, H * D, H * G * D)]
    out = [torch.zeros(B, H * G * D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    lse = [torch.zeros(B, H * G, device="cuda") for _ in range(2)]
    ws = [qf.kv_attention_workspace(caches[0], seqs, B, H * G) for _ in range(2)]

    def step(i):
        qf.kv_write(caches[i], seqs, x[0], x[1])
        qf.kv_attention(caches[i], seqs, x[2], out[i], ws[i], lse=lse[i])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for a in x:
            a.normal_()
        lens.fill_(1)
        step(0)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(0)
    for n in (1, 2, 16, 17, 300, 1200, 40):
        for a in x:
            a.normal_()
        lens.copy_(torch.tensor([n, max(1, n // 3), n], dtype=torch.int32))
        graph.replay()
        step(1)
        torch.cuda.synchronize()
        assert torch.equal(out[0], out[1]) and torch.equal(lse[0], lse[1])
    for a, b in zip(caches[0]._tensors[:4], caches[1]._tensors[:4]):
        assert torch.equal(a, b)


def test_two_streams(qf):
    """Two calls at once, each with its own workspace, equal the same calls one after the other."""
    rng = np.random.default_rng(21)
    H, G, D, page, cols = 2, 4, 128, 16, 200
    sets = []
    for i in range(2):
        table = kc.table(rng, 2, cols, 2 * cols)
        k, v = kc.pool(rng, "nvfp4", 2 * cols, H, page, D), kc.pool(rng, "nvfp4", 2 * cols, H, page, D)
        cache, seqs = _cache(qf, "nvfp4", k, v), _seqs(qf, [3000, 1700 + i], table)
        q = to_dev(workloads.normal_bf16(rng, (2, H * G * D)))
        sets.append((cache, seqs, q, qf.kv_attention_workspace(cache, seqs, 2, H * G)))
    want = []
    for c, s, q, ws in sets:
        want.append(torch.empty_like(q))
        qf.kv_attention(c, s, q, want[-1], ws)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [torch.empty_like(w) for w in want]
    for _ in range(10):
        for (c, s, q, ws), st, g in zip(sets, streams, got):
            with torch.cuda.stream(st):
                qf.kv_attention(c, s, q, g, ws)
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b)


def test_python_refusals(qf):
    c = torch.zeros(2, 1, 16, 32, dtype=torch.uint8, device="cuda")
    s = torch.zeros(2, 1, 16, 2, dtype=torch.uint8, device="cuda")
    cache = qf.kv_cache("mxfp4", c, s, c, s)
    with pytest.raises(ValueError):
        qf.kv_cache("nvfp4", c, s, c, s)                           # no S, scales of the other format
    with pytest.raises(ValueError):
        qf.kv_cache("mxfp4", c, s[:1], c, s)
    with pytest.raises(TypeError):
        qf.kv_cache("mxfp4", c.int(), s, c, s)
    lens, table = torch.ones(2, dtype=torch.int32, device="cuda"), torch.zeros(2, 1, dtype=torch.int32, device="cuda")
    with pytest.raises(TypeError):
        qf.kv_sequences(lens.long(), table)
    with pytest.raises(ValueError):
        qf.kv_sequences(lens[:1], table)
    with pytest.raises(ValueError):
        qf.kv_sequences(lens, table, max_len=-3)
    seqs = qf.kv_sequences(lens, table)
    x = torch.zeros(2, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError):
        qf.kv_write(cache, seqs, x, x[:1])
    with pytest.raises(ValueError):
        qf.kv_write(cache, seqs, x[:, :32], x)
    with pytest.raises(qf.QFError):
        qf.kv_write(cache, seqs, x[:1], x[:1])                     # one row for two sequences
    with pytest.raises(ValueError):
        qf.kv_attention(cache, seqs, x, x[:, :32].contiguous(), torch.empty(256, dtype=torch.uint8, device="cuda"))
    with pytest.raises(qf.QFError):
        qf.kv_attention(cache, seqs, x, x.clone(), torch.empty(256, dtype=torch.uint8, device="cuda"), window=-1)
