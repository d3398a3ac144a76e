"""GPU parity of the products of few rows with packed weights, dense and per expert, against the
FP64 decode of the same codes.

Bound: a sum of K exact products of bf16 values in binary32, in chains of at most 32 terms (one
MFMA) + K / 128 steps of one wave x 4 + 8 waves, each addition rounding a partial sum no larger than
sum |x| |w|: D u sum |x| |w| with D = 32 + K / 32 + 8 and u = 2^-23 (the matrix cores' additions
need not round to nearest); two more roundings for the block and tensor scales.  Q4_K sums
(16 + q) x and x: |w| there counts as |d s6| (16 + q) + |dmin m6 + 16 d s6|.  A bf16 result adds
2^-8 relative, FP32 2^-24."""
import numpy as np
import pytest

import workloads
from oracle import experts as ox
from tests import matvec_cases
from tests.helpers import bf16_to_f64, from_dev, to_dev

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

BLOCK = {"nvfp4": 16, "mxfp4": 32, "q4k": 256}


@pytest.fixture(scope="module")
def qf():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_39223_amd as qf
    qf.lib()
    return qf


def _codes(rng, fmt, R, K, E=1):
    """Arbitrary codes under arbitrary scales of a realistic range."""
    if fmt == "q4k":
        c = rng.integers(0, 256, (R, K // 256, 144)).astype(np.uint8)
        half = (rng.random((R, K // 256, 2)) * 0.01).astype(np.float16)
        c[..., :4] = half.view(np.uint8).reshape(R, K // 256, 4)
        return c, None, None
    codes = rng.integers(0, 256, (R, K // 2)).astype(np.uint8)
    if fmt == "nvfp4":
        return codes, rng.integers(0, 0x7F, (R, K // 16)).astype(np.uint8), (rng.random(E) * 1e-3 + 1e-5).astype(np.float32)
    return codes, rng.integers(100, 130, (R, K // 32)).astype(np.uint8), None


def _magnitude(fmt, codes, W):
    if fmt != "q4k":
        return np.abs(W)
    zero_q = codes.copy()
    zero_q[..., 16:] = 0
    off = np.abs(ox.decode(fmt, zero_q))                          # dmin m6
    one_q = zero_q.copy()
    one_q[..., 16:] = 0x11
    step = np.abs(ox.decode(fmt, one_q) + off)                    # d s6
    return np.abs(W) + off + 16 * step + off + 16 * step


def _bound(x, W, mag, K, f32):
    ref = x @ W.T
    return ref, ((32 + K / 32 + 8) * 2.0 ** -23 + 2.0 ** -22) * (np.abs(x) @ mag.T) + (2.0 ** -24 if f32 else 2.0 ** -8) * np.abs(ref)


def _weight(qf, fmt, N, K, codes, scales, S, E=None):
    return qf.packed_weight(fmt, N, K, to_dev(codes), None if scales is None else to_dev(scales),
                            None if S is None else to_dev(S), E=E)


def _out(R, N, f32, pad=8):
    cols = (N + 7) // 8 * 8 + pad
    return torch.full((R, cols), 7.0, dtype=torch.float32 if f32 else torch.bfloat16, device="cuda")


SHAPES = [(1, 1, 256), (1, 16, 512), (1, 4096, 256), (2, 37, 768), (5, 1000, 1024), (16, 129, 2304), (17, 64, 768),
          (33, 40, 1024), (64, 257, 4096), (3, 24, 256 * 9), (1, 9000, 256), (40, 17000, 256)]
FP4_SHAPES = [(1, 8, 32), (3, 20, 96), (7, 33, 160), (16, 50, 1056), (50, 9, 4000)]
ODD_SHAPES = [(1, 8, 16), (2, 17, 48), (9, 33, 272), (33, 20, 1040 + 16), (64, 40, 4080)]


@pytest.mark.parametrize("fmt,M,N,K", [(f, *s) for f in ("nvfp4", "mxfp4", "q4k") for s in SHAPES]
                         + [(f, *s) for f in ("nvfp4", "mxfp4") for s in FP4_SHAPES]
                         + [("nvfp4", *s) for s in ODD_SHAPES])
@pytest.mark.parametrize("f32", [False, True])
def test_dense(qf, fmt, M, N, K, f32):
    rng = np.random.default_rng(M * N + K)
    codes, scales, S = _codes(rng, fmt, N, K)
    xh = workloads.normal_bf16(rng, (M, K))
    wide = np.full((M, (K + 7) // 8 * 8 + 16), 0x7FC0, np.uint16)
    wide[:, :K] = xh
    full = _out(M, N, f32)
    weight = _weight(qf, fmt, N, K, codes, scales, S)
    qf.packed_matvec(weight, to_dev(wide)[:, :K], full[:, :N])
    W = ox.decode(fmt, codes, scales, None if S is None else S[0])
    ref, bound = _bound(bf16_to_f64(xh), W, _magnitude(fmt, codes, W), K, f32)
    got = full[:, :N].double().cpu().numpy()
    assert np.all(np.abs(got - ref) <= bound), float((np.abs(got - ref) / bound).max())
    assert bool((full[:, N:] == 7).all())
    again = _out(M, N, f32)
    qf.packed_matvec(weight, to_dev(wide)[:, :K], again[:, :N])
    assert torch.equal(full, again)


@pytest.mark.parametrize("fmt", ["nvfp4", "mxfp4", "q4k"])
def test_codes_of_the_quantizers(qf, fmt):
    """A weight quantized by the library, one token: near the layer's product on W_hat."""
    rng = np.random.default_rng(4)
    N, K = 96, 512
    W, x = to_dev(workloads.normal_bf16(rng, (N, K), 0.02)), workloads.normal_bf16(rng, (1, K))
    hat = torch.empty(N, K, dtype=torch.int16, device="cuda")
    if fmt == "q4k":
        codes, scales, S = torch.empty(N, K // 256, 144, dtype=torch.uint8, device="cuda"), None, None
        qf.fakequant_q4k(W, codes, hat)
    else:
        codes = torch.empty(N, K // 2, dtype=torch.uint8, device="cuda")
        scales, S = torch.empty(N, K // BLOCK[fmt], dtype=torch.uint8, device="cuda"), None
        if fmt == "nvfp4":
            S = torch.empty(1, device="cuda")
            qf.fakequant_nvfp4(W, torch.empty(1, device="cuda"), qf.AMAX_COMPUTE, S, codes, scales, hat)
        else:
            qf.fakequant_mxfp4(W, codes, scales, hat)
    Y = torch.empty(1, N, device="cuda")
    qf.packed_matvec(qf.packed_weight(fmt, N, K, codes, scales, S), to_dev(x), Y)
    Wh, xf = bf16_to_f64(from_dev(hat)), bf16_to_f64(x)
    assert np.all(np.abs(from_dev(Y) - xf @ Wh.T) <= (2.0 ** -8 * 1.01 + 1e-4) * (np.abs(xf) @ np.abs(Wh).T))


def test_non_finite(qf):
    rng = np.random.default_rng(6)
    N, K = 40, 512
    for fmt, bad in (("nvfp4", 0x7F), ("mxfp4", 0xFF)):
        codes, scales, S = _codes(rng, fmt, N, K)
        scales[5, 3] = bad
        x = workloads.normal_bf16(rng, (2, K))
        Y = torch.empty(2, N, device="cuda")
        qf.packed_matvec(_weight(qf, fmt, N, K, codes, scales, S), to_dev(x), Y)
        nan = torch.isnan(Y)
        assert bool(nan[:, 5].all()) and int(nan.sum()) == 2
        x[0, 100] = 0x7F80                                         # an infinite activation: its row alone
        codes, scales, S = _codes(rng, fmt, N, K)
        codes[:, 50] |= 0x11                                       # (under weights that are not zero)
        scales[:, 100 // BLOCK[fmt]] = np.maximum(scales[:, 100 // BLOCK[fmt]], 1)
        qf.packed_matvec(_weight(qf, fmt, N, K, codes, scales, S), to_dev(x), Y)
        assert not bool(torch.isfinite(Y[0]).any()) and bool(torch.isfinite(Y[1]).all())


def test_no_rows_no_columns_no_depth(qf):
    rng = np.random.default_rng(7)
    codes, scales, S = _codes(rng, "nvfp4", 16, 64)
    qf.packed_matvec(_weight(qf, "nvfp4", 16, 64, codes, scales, S), torch.empty(0, 64, dtype=torch.bfloat16, device="cuda"),
                     torch.empty(0, 16, device="cuda"))
    z = torch.empty(0, dtype=torch.uint8, device="cuda")
    Y = torch.full((3, 16), 7.0, device="cuda")
    qf.packed_matvec(qf.packed_weight("mxfp4", 16, 0, z, z), torch.empty(3, 0, dtype=torch.bfloat16, device="cuda"), Y)
    assert bool((Y == 0).all())


def _grouped(rng, counts):
    off = np.zeros(len(counts) + 1, np.int64)
    off[1:] = np.cumsum(counts)
    return off


@pytest.mark.parametrize("fmt,N,K,counts", [
    ("nvfp4", 64, 256, [1]), ("nvfp4", 40, 272, [0, 3, 0, 17, 1, 0]), ("mxfp4", 33, 96, [5, 0, 70, 1]),
    ("q4k", 24, 512, [2, 0, 33, 16]), ("nvfp4", 16, 128, [0] * 129 + [4]), ("mxfp4", 16, 64, [1] * 300),
    ("nvfp4", 272, 512, [20] * 5), ("q4k", 48, 256, [40, 9, 0, 64, 65]), ("mxfp4", 17, 32, [0, 0, 0])])
@pytest.mark.parametrize("f32", [False, True])
def test_grouped(qf, fmt, N, K, counts, f32):
    rng = np.random.default_rng(N + K + len(counts))
    E, off = len(counts), _grouped(rng, counts)
    R, live = int(off[-1]) + 3, int(off[-1])                       # three rows of no expert
    codes, scales, S = _codes(rng, fmt, E * N, K, E)
    div, M = 3, 29
    rows = rng.integers(0, M * div, R).astype(np.int32)
    rows[live:] = -1
    if live > 2:
        rows[1], rows[2] = -1, M * div + 5                         # X rows that do not exist
    xh = workloads.normal_bf16(rng, (M, K))
    full = _out(R, N, f32)
    weight = _weight(qf, fmt, N, K, codes, scales, S, E=E)
    qf.packed_matvec_grouped(weight, to_dev(off), to_dev(xh), full[:, :N], rows=to_dev(rows), rows_div=div)
    x = np.zeros((R, K))
    ok = (rows >= 0) & (rows < M * div)
    x[ok] = bf16_to_f64(xh)[rows[ok] // div]
    got = full[:, :N].double().cpu().numpy()
    for e in range(E):
        a, b = off[e], off[e + 1]
        if a == b:
            continue
        part = slice(e * N, (e + 1) * N)
        W = ox.decode(fmt, codes[part], None if scales is None else scales[part], None if S is None else S[e])
        ref, bound = _bound(x[a:b], W, _magnitude(fmt, codes[part], W), K, f32)
        assert np.all(np.abs(got[a:b] - ref) <= bound), e
    assert bool((full[live:] == 7).all()) and bool((full[:, N:] == 7).all())
    # rows in expert order already
    if live:
        xg = np.zeros((R, K), np.uint16)
        xg[ok] = xh[rows[ok] // div]
        same = _out(R, N, f32)
        qf.packed_matvec_grouped(weight, to_dev(off), to_dev(xg), same[:, :N])
        assert torch.equal(full, same)


@pytest.mark.parametrize("fmt,N,K,counts", [
    ("nvfp4", 48, 1072, [9, 16, 17, 0, 8, 40]), ("mxfp4", 80, 1184, [12, 1, 33, 16, 9, 25]),
    ("mxfp4", 32, 512, [1] * 20 + [15] * 12), ("nvfp4", 33, 1536, [0] * 30 + [10, 64]),
    ("nvfp4", 4112, 1024, [10, 11, 30]), ("mxfp4", 8208, 2048, [16, 9, 0, 24])])
def test_grouped_many_rows(qf, fmt, N, K, counts):
    """Experts of 9 to 16 rows a group over whole slices, a tail of k, and codes copied in words."""
    test_grouped(qf, fmt, N, K, counts, False)
    test_grouped(qf, fmt, N, K, counts, True)


def test_grouped_offsets_out_of_range_and_no_x(qf):
    """Offsets that leave 0 .. R are cut to it; no X rows at all: zeros."""
    rng = np.random.default_rng(3)
    codes, scales, S = _codes(rng, "mxfp4", 32, 64)
    weight = _weight(qf, "mxfp4", 16, 64, codes, scales, S, E=2)
    x = workloads.normal_bf16(rng, (6, 64))
    Y = _out(6, 16, True)
    qf.packed_matvec_grouped(weight, torch.tensor([-4, 3, 900], device="cuda"), to_dev(x), Y[:, :16])
    W = ox.decode("mxfp4", codes, scales)
    ref = np.concatenate([bf16_to_f64(x)[:3] @ W[:16].T, bf16_to_f64(x)[3:] @ W[16:].T])
    assert np.allclose(from_dev(Y[:, :16]), ref, rtol=1e-4, atol=1e-4 * np.abs(ref).max())
    qf.packed_matvec_grouped(weight, torch.tensor([0, 3, 6], device="cuda"), torch.empty(0, 64, dtype=torch.bfloat16, device="cuda"),
                             Y[:, :16])
    assert bool((Y[:, :16] == 0).all())


def test_weights_past_32_bits_of_bytes(qf):
    """Experts whose codes start past 2^32 bytes (5 GB of NVFP4 codes)."""
    E, N, K = 320, 4096, 8192
    g = torch.Generator(device="cuda").manual_seed(1)
    codes = torch.randint(0, 256, (N, K // 2), generator=g, device="cuda", dtype=torch.uint8).repeat(E, 1)
    scales = torch.randint(40, 80, (E * N, K // 16), generator=g, device="cuda", dtype=torch.uint8)
    S = torch.rand(E, generator=g, device="cuda") + 0.5
    off = torch.zeros(E + 1, dtype=torch.int64, device="cuda")
    off[E - 1:] = 1
    off[E] = 3
    x = torch.randn(3, K, generator=g, device="cuda").to(torch.bfloat16)
    Y = torch.empty(3, N, device="cuda")
    qf.packed_matvec_grouped(qf.packed_weight("nvfp4", N, K, codes, scales, S, E=E), off, x, Y)
    pick = [0, 1, 77, N - 1]
    for r, e in ((0, E - 2), (1, E - 1), (2, E - 1)):
        W = ox.decode("nvfp4", from_dev(codes[[e * N + p for p in pick]]), from_dev(scales[[e * N + p for p in pick]]), float(S[e]))
        ref, bound = _bound(x[r:r + 1].double().cpu().numpy(), W, np.abs(W), K, True)
        assert np.all(np.abs(from_dev(Y[r:r + 1, pick]) - ref) <= bound)


def test_in_a_graph_and_on_a_side_stream(qf):
    rng = np.random.default_rng(12)
    E, N, K, R = 6, 80, 512, 24
    codes, scales, S = _codes(rng, "nvfp4", E * N, K, E)
    weight = _weight(qf, "nvfp4", N, K, codes, scales, S, E=E)
    off = torch.empty(E + 1, dtype=torch.int64, device="cuda")
    X = torch.empty(R, K, dtype=torch.bfloat16, device="cuda")
    Y = torch.empty(R, N, dtype=torch.bfloat16, device="cuda")

    def load(seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        X.copy_(torch.randn(R, K, generator=g, device="cuda"))
        off.copy_(torch.cat([torch.zeros(1), torch.randint(0, R + 1, (E - 1,), generator=g, device="cuda").cpu().sort().values,
                             torch.full((1,), R)]).long())

    load(0)
    qf.packed_matvec_grouped(weight, off, X, Y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        qf.packed_matvec_grouped(weight, off, X, Y)
    for seed in (1, 2, 3, 1):
        load(seed)
        qf.packed_matvec_grouped(weight, off, X, Y)
        torch.cuda.synchronize()
        want = Y.clone()
        Y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(Y, want), seed
        Y.zero_()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            qf.packed_matvec_grouped(weight, off, X, Y)
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        assert torch.equal(Y, want), seed


def test_refusals(qf):
    rng = np.random.default_rng(2)
    codes, scales, S = _codes(rng, "nvfp4", 16, 64)
    weight = _weight(qf, "nvfp4", 16, 64, codes, scales, S)
    X, Y = torch.zeros(65, 64, dtype=torch.bfloat16, device="cuda"), torch.full((65, 16), 7.0, device="cuda")
    with pytest.raises(qf.QFError, match="QF_ENOTSUP"):
        qf.packed_matvec(weight, X, Y)
    with pytest.raises(qf.QFError, match="tensor scales"):
        qf.packed_matvec(qf.packed_weight("nvfp4", 16, 64, to_dev(codes), to_dev(scales)), X[:1], Y[:1])
    with pytest.raises(qf.QFError, match="QF_EALIGN"):
        qf.packed_matvec(qf.packed_weight("mxfp4", 4, 32, to_dev(codes).view(-1)[8:], to_dev(scales)), X[:1, :32], Y[:1, :4])
    with pytest.raises(qf.QFError, match="QF_ESHAPE"):
        qf.packed_matvec(qf.packed_weight("q4k", 16, 64, to_dev(codes)), X[:1], Y[:1])
    with pytest.raises(ValueError):
        qf.packed_weight("nvfp4", 17, 64, to_dev(codes), to_dev(scales), to_dev(S))
    with pytest.raises(ValueError):
        qf.packed_matvec(weight, X[:1, :32], Y[:1])
    with pytest.raises(ValueError):
        qf.packed_matvec_grouped(weight, torch.zeros(3, dtype=torch.int64, device="cuda"), X, Y)
    with pytest.raises(qf.QFError, match="QF_EINVAL"):
        qf.packed_matvec_grouped(weight, torch.zeros(2, dtype=torch.int64, device="cuda"), X, Y, rows_div=0)
    torch.cuda.synchronize()
    assert bool((Y == 7).all())


def test_more_row_groups_than_one_launch_holds(qf):
    """33000 rows of 2^20 columns need more workgroups than a grid may have: several launches.  Every
    row is one of 64 rows of X, whose products a dense call gives (same sums in the same order: one
    wave a tile in both, and one MFMA deep)."""
    N, K, M, R = 1 << 20, 32, 64, 33000
    g = torch.Generator(device="cuda").manual_seed(8)
    codes = torch.randint(0, 256, (N, K // 2), generator=g, device="cuda", dtype=torch.uint8)
    scales = torch.randint(110, 130, (N, K // 32), generator=g, device="cuda", dtype=torch.uint8)
    x = torch.randn(M, K, generator=g, device="cuda").to(torch.bfloat16)
    rows = torch.randint(0, M, (R,), generator=g, device="cuda", dtype=torch.int32)
    want = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    qf.packed_matvec(qf.packed_weight("mxfp4", N, K, codes, scales), x, want)
    Y = torch.full((R, N), 7.0, dtype=torch.bfloat16, device="cuda")
    off = torch.tensor([0, R - 2], device="cuda")
    qf.packed_matvec_grouped(qf.packed_weight("mxfp4", N, K, codes, scales, E=1), off, x, Y, rows=rows)
    for r in range(0, R - 2, 1000):
        end = min(r + 1000, R - 2)
        assert torch.equal(Y[r:end], want[rows[r:end].long()]), r
    assert bool((Y[R - 2:] == 7).all())


def test_more_columns_than_one_launch_holds(qf):
    """64 rows of 2^29 + 40 columns: three row groups in one launch, the fourth in another.  The weight
    is one of 2^20 rows over and over, whose products a call of its own gives."""
    n, K, M, times = 1 << 20, 32, 64, 512
    g = torch.Generator(device="cuda").manual_seed(9)
    codes = torch.randint(0, 256, (n, K // 2), generator=g, device="cuda", dtype=torch.uint8)
    scales = torch.randint(110, 130, (n, K // 32), generator=g, device="cuda", dtype=torch.uint8)
    x = torch.randn(M, K, generator=g, device="cuda").to(torch.bfloat16)
    want = torch.empty(M, n, dtype=torch.bfloat16, device="cuda")
    qf.packed_matvec(qf.packed_weight("mxfp4", n, K, codes, scales), x, want)
    N = n * times + 40
    all_codes = torch.cat([codes.repeat(times, 1), codes[:40]])
    all_scales = torch.cat([scales.repeat(times, 1), scales[:40]])
    Y = torch.full((M, N), 7.0, dtype=torch.bfloat16, device="cuda")
    qf.packed_matvec(qf.packed_weight("mxfp4", N, K, all_codes, all_scales), x, Y)
    for i in range(times):
        assert torch.equal(Y[:, i * n:(i + 1) * n], want), i
    assert torch.equal(Y[:, times * n:], want[:, :40])


@pytest.mark.parametrize("fmt,instance,rows,N,K", matvec_cases.VARIANTS)
def test_every_instance_of_the_kernel(qf, fmt, instance, rows, N, K):
    """All columns against FP64 on the decode; the weight's rows are 2053 different ones over and over."""
    rng = np.random.default_rng(N + K)
    grouped, E, R = matvec_cases.sizes(rows)
    P, M, div = 2053, 29 if grouped else R, 3
    codes, scales, S = _codes(rng, fmt, P, K, E)
    W = ox.decode(fmt, codes, scales, None if S is None else 1.0)
    mag = torch.from_numpy(_magnitude(fmt, codes, W)).cuda()
    W = torch.from_numpy(W).cuda()
    pick = torch.arange(E * N, device="cuda") % P
    weight = qf.packed_weight(fmt, N, K, to_dev(codes)[pick], None if scales is None else to_dev(scales)[pick],
                              None if S is None else to_dev(S), E=E if grouped else None)
    xh = workloads.normal_bf16(rng, (M, K))
    wide = np.full((M, (K + 7) // 8 * 8 + 16), 0x7FC0, np.uint16)
    wide[:, :K] = xh
    X, xf = to_dev(wide)[:, :K], torch.from_numpy(bf16_to_f64(xh)).cuda()
    if grouped:
        off = _grouped(rng, rows)
        of = rng.integers(0, M * div, R).astype(np.int32)
        of[1] = -1
        xf = torch.cat([xf, torch.zeros(1, K, dtype=torch.float64, device="cuda")])
        x = xf[torch.from_numpy(np.where(of < 0, M, of // div)).cuda().long()]
    else:
        off, x = [0, R], xf
    for f32 in (True, False):
        full = _out(R, N, f32)
        if grouped:
            qf.packed_matvec_grouped(weight, to_dev(off), X, full[:, :N], rows=to_dev(of), rows_div=div)
        else:
            qf.packed_matvec(weight, X, full[:, :N])
        for e in range(E):
            a, b = int(off[e]), int(off[e + 1])
            if a == b:
                continue
            p, s = pick[e * N:(e + 1) * N], 1.0 if S is None else float(S[e])
            ref, most = x[a:b] @ W[p].t().contiguous() * s, x[a:b].abs() @ mag[p].t().contiguous() * s
            bound = ((32 + K / 32 + 8) * 2.0 ** -23 + 2.0 ** -22) * most + (2.0 ** -24 if f32 else 2.0 ** -8) * ref.abs()
            assert bool(((full[a:b, :N].double() - ref).abs() <= bound).all()), (e, f32)
        assert bool((full[:, N:] == 7).all()) and bool((full[int(off[-1]):] == 7).all())


@pytest.mark.parametrize("fmt,K", [("nvfp4", 1056), ("nvfp4", 1072), ("mxfp4", 1056)])
def test_nan_scales_in_every_form(qf, fmt, K):
    """A scale code that is NaN, in a whole slice or in the k past it, under codes that are zero too: its
    weight row's outputs are NaN and no others, for few rows, up to 16, and experts of 9 to 16."""
    rng = np.random.default_rng(K)
    N, bad = 70, {"nvfp4": (0x7F, 0xFF), "mxfp4": (0xFF, 0xFF)}[fmt]
    codes, scales, S = _codes(rng, fmt, 2 * N, K, 2)
    codes[:, ::3] = 0
    n, last = 5, scales.shape[1] - 1
    scales[n, 3], scales[33, last], scales[N + 64, 0] = bad[0], bad[0], bad[1]
    codes[n, 3 * BLOCK[fmt] // 2:4 * BLOCK[fmt] // 2] = 0
    want = np.zeros((2, N), bool)
    want[0, [n, 33]], want[1, 64] = True, True
    want = torch.from_numpy(want).cuda()
    for M in (2, 7, 16, 40):
        x = to_dev(workloads.normal_bf16(rng, (M, K)))
        Y = _out(M, N, True)[:, :N]
        qf.packed_matvec(_weight(qf, fmt, N, K, codes[:N], scales[:N], None if S is None else S[:1]), x, Y)
        assert torch.equal(torch.isnan(Y), want[:1].expand(M, N)), M
    for counts in ([1, 2], [4, 5], [16, 11], [40, 20]):
        R = sum(counts)
        x = to_dev(workloads.normal_bf16(rng, (R, K)))
        Y = _out(R, N, True)[:, :N]
        qf.packed_matvec_grouped(_weight(qf, fmt, N, K, codes, scales, S, E=2), to_dev(_grouped(rng, counts)), x, Y)
        assert torch.equal(torch.isnan(Y), want[torch.tensor([0] * counts[0] + [1] * counts[1], device="cuda")]), counts


def test_q4k_activations_of_every_size(qf):
    """Every finite activation has the definition's product, however near the type's largest it is, where
    that is finite: d and dmin of 2^-24 or thrice it, so that it always is (2^128 x 3 x 2^-24 x 63 x 16 x
    1280 < 2^127), while 16 sum x and sums of s6 (16 + q) x are far from it.  Activations of 2^-120 too: the
    bound then has what sums kept to multiples of 2^-149 / 2^18 can be off by, once an addition, s6 or m6
    times, twice."""
    rng = np.random.default_rng(21)
    N, K, M = 40, 1280, 9
    codes, _, _ = _codes(rng, "q4k", N, K)
    half = ((1 + 2 * rng.integers(0, 2, (N, K // 256, 2))) * 2.0 ** -24).astype(np.float16)
    codes[..., :4] = half.view(np.uint8).reshape(N, K // 256, 4)
    codes[7, 1, 4:] = 0xFF                                         # the largest scales, mins and codes
    x = workloads.normal_bf16(rng, (M, K))
    x[0] = 0x7F7F                                                  # the largest, all of one sign
    x[1] = np.where(rng.random(K) < 0.5, 0x7F7F, 0xFF7F)
    x[2] = (x[2] & 0x807F) | 0x7F00                                # 2^127 to 2^128
    x[3] = (x[3] & 0x807F) | 0x7880                                # 2^114 to 2^115
    x[4, ::2] = 0x7F7F                                             # beside ordinary ones
    x[5] = (x[5] & 0x807F) | 0x2000                                # 2^-63 to 2^-62
    x[6] = (x[6] & 0x807F) | 0x0380                                # 2^-120 to 2^-119
    for big in (False, True):
        if big:                                                    # steps of 2^14 for the small ones alone
            codes[..., :4] = np.full((N, K // 256, 2), 2.0 ** 14, np.float16).view(np.uint8).reshape(N, K // 256, 4)
            x[:5] = 0
        W = ox.decode("q4k", codes)
        Y = torch.empty(M, N, device="cuda")
        qf.packed_matvec(qf.packed_weight("q4k", N, K, to_dev(codes)), to_dev(x), Y)
        ref, bound = _bound(bf16_to_f64(x), W, _magnitude("q4k", codes, W), K, True)
        assert np.abs(ref).max() < 3.4e38
        step = 2.0 ** 14 if big else 3 * 2.0 ** -24
        bound += 2 * (32 + K / 32 + 8) * 63 * step * 2.0 ** (18 - 149) + 2.0 ** -149
        off = ~(np.abs(from_dev(Y) - ref) <= bound)
        assert not off.any(), (big, np.argwhere(off)[:4].tolist())
