"""GPU parity of the adapters of many requests against FP64.

Bound, u = 2^-23 (sums of the matrix cores need not round to nearest): z sums K exact products in chains of
K / 32 steps, 4 waves and up to 16 slices, z's two bf16 halves leave 2^-17 of it, the second product sums 2 r
terms, and base is added once: ((K / 32 + r / 8 + 64) u + 2^-16) |scale| sum |b| sum |a||x| + u |Y|.  A bf16 result
adds 2^-8 relative, FP32 2^-24."""
import numpy as np
import pytest

import workloads
from oracle import serving as sv
from tests.helpers import bf16_to_f64, to_dev

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
U = 2.0 ** -23


@pytest.fixture(scope="module")
def qf():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_39223_amd as qf
    qf.lib()
    return qf


def _wide(x, pad=8):
    w = np.full((x.shape[0], (x.shape[1] + 7) // 8 * 8 + pad), 0x7FC0, np.uint16)
    w[:, :x.shape[1]] = x
    return to_dev(w)[:, :x.shape[1]].view(torch.bfloat16)


def _case(rng, M, n, r, K, N, ids=None, ranks=None):
    A, B = workloads.normal_bf16(rng, (n * r, K), K ** -0.5), workloads.normal_bf16(rng, (n * N, r), 0.05)
    return {"A": A.reshape(n, r, K), "B": B.reshape(n, N, r), "scale": (rng.standard_normal(n) * 2).astype(np.float32),
            "X": workloads.normal_bf16(rng, (M, K)), "base": workloads.normal_bf16(rng, (M, N)),
            "ids": (rng.integers(-1, n + 1, M) if ids is None else np.asarray(ids)).astype(np.int32),
            "ranks": None if ranks is None else np.asarray(ranks, np.int32)}


def _ref(c, base=True):
    f = bf16_to_f64
    return sv.lora_rows(c["ids"], f(c["X"]), f(c["A"]), f(c["B"]), c["scale"].astype(np.float64), f(c["base"]) if base else None,
                        c["ranks"])


def _check(got, ref, mag, r, K, f32):
    bound = ((K / 32 + r / 8 + 64) * U + 2.0 ** -16) * mag + (U + (2.0 ** -24 if f32 else 2.0 ** -8)) * np.abs(ref) + 1e-38
    assert np.all(np.abs(got - ref) <= bound), float((np.abs(got - ref) / bound).max())


def _run(qf, c, f32=False, inplace=False, base=True, pad=8):
    n, r, K = c["A"].shape
    M, N = c["base"].shape
    bf = lambda a: to_dev(a).view(torch.bfloat16)  # noqa: E731
    a = qf.adapters(bf(c["A"]), bf(c["B"]), to_dev(c["scale"]), None if c["ranks"] is None else to_dev(c["ranks"]))
    ws = qf.lora_rows_workspace(a, M)
    ws.fill_(0xFF)
    b = _wide(c["base"])
    b = b.float() if f32 else b
    cols = (N + 7) // 8 * 8 + pad
    full = torch.full((M, cols), 7.0, dtype=torch.float32 if f32 else torch.bfloat16, device="cuda")
    Y = full[:, :N]
    if f32:
        wide = torch.full((M, cols), float("nan"), device="cuda")
        wide[:, :N] = b
        b = wide[:, :N]
    if inplace:
        Y.copy_(b)
        b = Y
    args = (a, to_dev(c["ids"]), _wide(c["X"]), Y, ws)
    qf.lora_rows(*args, base=b if base else None)
    assert bool((full[:, N:] == 7).all())
    first = Y.clone()
    if not inplace:
        qf.lora_rows(*args, base=b if base else None)
        assert np.array_equal(first.float().cpu().numpy(), Y.float().cpu().numpy(), equal_nan=True)
    return first.double().cpu().numpy()


SHAPES = [(1, 1, 8, 8, 8), (1, 3, 16, 256, 100), (5, 2, 24, 1000, 37), (16, 16, 16, 512, 256), (17, 4, 8, 264, 513), (33, 40, 64, 1032, 72),
          (61, 24, 128, 4096, 200), (64, 1, 256, 136, 1000), (300, 5, 40, 520, 264), (1000, 9, 32, 128, 65)]


@pytest.mark.parametrize("M,n,r,K,N", SHAPES)
@pytest.mark.parametrize("f32", [False, True])
def test_shapes(qf, M, n, r, K, N, f32):
    c = _case(np.random.default_rng(M * N), M, n, r, K, N)
    for kw in ({}, {"inplace": True}):
        _check(_run(qf, c, f32, **kw), *_ref(c), r, K, f32)
    _check(_run(qf, c, f32, base=False), *_ref(c, False), r, K, f32)


@pytest.mark.parametrize("order", ["runs", "mixed", "one", "none", "far"])
@pytest.mark.parametrize("M", [1, 40, 500])
def test_orders(qf, order, M):
    rng = np.random.default_rng(M)
    n, r, K, N = 7, 16, 320, 130
    ids = {"runs": np.arange(M) * n // M, "mixed": rng.integers(0, n, M), "one": np.full(M, 3), "none": np.full(M, -1),
           "far": rng.choice([n, 1 << 30, -(1 << 31), (1 << 31) - 1, 2], M)}[order]
    c = _case(rng, M, n, r, K, N, ids)
    for kw in ({}, {"inplace": True}):
        _check(_run(qf, c, **kw), *_ref(c), r, K, False)


def test_ranks(qf):
    """Adapters of lower rank than they are stored with, down to none: what lies in the rest is not used."""
    rng = np.random.default_rng(5)
    n, r, K, N, M = 6, 40, 256, 80, 70
    c = _case(rng, M, n, r, K, N, ranks=[40, 1, 0, 8, 33, 1000])
    for a, k in enumerate([40, 1, 0, 8, 33, 40]):
        c["A"][a, k:], c["B"][a, :, k:] = 0x7FC0, 0x7F80
    clean = {**c, "A": np.where(c["A"] == 0x7FC0, 0, c["A"]).astype(np.uint16), "B": np.where(c["B"] == 0x7F80, 0, c["B"]).astype(np.uint16)}
    _check(_run(qf, c), *_ref(clean), r, K, False)
    c["ranks"][3] = -4
    clean["ranks"] = c["ranks"]
    _check(_run(qf, c, f32=True), *_ref(clean), r, K, True)


def test_non_finite_rows_and_adapters(qf):
    """A NaN in a row stays in it, one in an adapter in its rows, an infinity gives one or a NaN there."""
    rng = np.random.default_rng(6)
    M, n, r, K, N = 40, 4, 16, 256, 64
    c = _case(rng, M, n, r, K, N, rng.integers(0, n - 1, M))
    clean = _run(qf, c)
    c["X"][7, 100], c["X"][20, 3] = 0x7FC0, 0x7F80
    c["A"][n - 1] = 0x7FC0                                         # (nobody's)
    got = _run(qf, c)
    assert np.isnan(got[7]).all() and not np.isfinite(got[20]).any()
    rest = np.delete(np.arange(M), [7, 20])
    assert np.array_equal(got[rest], clean[rest])
    c = _case(rng, M, n, r, K, N, rng.integers(0, n, M))
    clean = _run(qf, c)
    c["B"][1, 5, 3] = 0x7FC0
    got = _run(qf, c)
    bad = np.zeros((M, N), bool)
    bad[c["ids"] == 1, 5] = True
    assert np.array_equal(np.isnan(got), bad) and np.array_equal(got[~bad], clean[~bad])


@pytest.mark.parametrize("M", [5, 80])
def test_sums_next_to_the_largest_float(qf, M):
    """s z between the largest bf16 and the largest FP32 value, of either sign, is still finite times a small B."""
    c = _case(np.random.default_rng(9), M, 1, 8, 8, 24, np.zeros(M))
    bf = lambda v: int(np.float32(v).view(np.uint32)) >> 16  # noqa: E731
    c["X"][:], c["A"][:], c["base"][:], c["scale"][:] = 0, 0, 0, 1
    c["X"][:, 0], c["X"][:, 1], c["A"][:, 0, :2] = bf(2.0 ** 127 * (2 - 2.0 ** -7)), bf(1.5 * 2.0 ** 119), bf(1)
    c["X"][1::2, :2] |= 0x8000
    c["B"][:] = bf(2.0 ** -20)
    got, ref = _run(qf, c), _ref(c)
    assert np.abs(ref[0]).min() > 2.0 ** 107
    _check(got, *ref, 8, 8, False)


@pytest.mark.parametrize("M,n,r,K,N", [(100, 9000, 8, 8, 8), (70000, 3, 8, 8, 8), (200, 2, 256, 72, 40), (129, 1, 24, 40, 300),
                                       (200, 3, 24, 2056, 40), (150, 2, 32, 4168, 264), (90, 20, 32, 1024, 64), (130, 4, 16, 2312, 72)])
def test_many_rows_or_adapters(qf, M, n, r, K, N):
    """More adapters or rows than are put in order first, the widest rank, two and three groups of rows of one adapter,
    sums long enough for every loop, with odd ends."""
    c = _case(np.random.default_rng(M + n), M, n, r, K, N)
    _check(_run(qf, c), *_ref(c), r, K, False)
    _check(_run(qf, c, f32=True, inplace=True), *_ref(c), r, K, True)


@pytest.mark.parametrize("M", [3, 90])
def test_nothing_to_sum(qf, M):
    """K = 0, or no adapters at all: base alone."""
    rng = np.random.default_rng(10)
    bf = lambda a: to_dev(a).view(torch.bfloat16)  # noqa: E731
    base, ids = workloads.normal_bf16(rng, (M, 40)), to_dev(rng.integers(-1, 3, M).astype(np.int32))
    for n, K in ((2, 0), (0, 64), (0, 0)):
        e = lambda *s: torch.empty(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
        a = qf.adapters(e(n, 8, K), e(n, 40, 8).fill_(1), torch.ones(n, device="cuda"))
        ws = qf.lora_rows_workspace(a, M)
        ws.fill_(0xFF)
        Y = e(M, 40).fill_(7)
        qf.lora_rows(a, ids, e(M, K), Y, ws, base=bf(base))
        assert torch.equal(Y, bf(base))


def test_no_adapters_and_no_columns(qf):
    c = _case(np.random.default_rng(7), 20, 3, 8, 64, 40, np.full(20, 2))
    bf = lambda a: to_dev(a).view(torch.bfloat16)  # noqa: E731
    empty = qf.adapters(torch.empty(0, 8, 64, dtype=torch.bfloat16, device="cuda"), torch.empty(0, 40, 8, dtype=torch.bfloat16, device="cuda"),
                        torch.empty(0, device="cuda"))
    Y = torch.empty(20, 40, dtype=torch.bfloat16, device="cuda")
    qf.lora_rows(empty, to_dev(c["ids"]), bf(c["X"]), Y, qf.lora_rows_workspace(empty, 20), base=bf(c["base"]))
    assert torch.equal(Y, bf(c["base"]))
    none = qf.adapters(torch.empty(3, 8, 0, dtype=torch.bfloat16, device="cuda"), bf(c["B"]), to_dev(c["scale"]))
    qf.lora_rows(none, to_dev(c["ids"]), torch.empty(20, 0, dtype=torch.bfloat16, device="cuda"), Y, qf.lora_rows_workspace(none, 20))
    assert bool((Y == 0).all())


def test_graph_with_changing_ids(qf):
    """A captured call replayed with other adapters, rows and inputs, against eager calls."""
    rng = np.random.default_rng(8)
    M, n, r, K, N = 24, 6, 16, 512, 192
    c = _case(rng, M, n, r, K, N)
    bf = lambda a: to_dev(a).view(torch.bfloat16)  # noqa: E731
    a = qf.adapters(bf(c["A"]), bf(c["B"]), to_dev(c["scale"]))
    ids, X, base = to_dev(c["ids"]), bf(c["X"]), bf(c["base"])
    Y = [torch.empty(M, N, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    ws = [qf.lora_rows_workspace(a, M) for _ in range(2)]
    qf.lora_rows(a, ids, X, Y[0], ws[0], base=base)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        qf.lora_rows(a, ids, X, Y[0], ws[0], base=base)
    for i in range(5):
        ids.copy_(torch.from_numpy(rng.integers(-1, n, M).astype(np.int32)))
        X.normal_()
        base.normal_()
        graph.replay()
        qf.lora_rows(a, ids, X, Y[1], ws[1], base=base)
        torch.cuda.synchronize()
        assert torch.equal(Y[0], Y[1])


def test_python_refusals(qf):
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    scale = torch.ones(2, device="cuda")
    with pytest.raises(ValueError):
        qf.adapters(bf(2, 8, 64), bf(2, 32, 16), scale)
    with pytest.raises(TypeError):
        qf.adapters(torch.zeros(2, 8, 64, device="cuda"), bf(2, 32, 8), scale)
    with pytest.raises(TypeError):
        qf.adapters(bf(2, 8, 64), bf(2, 32, 8), scale.double())
    a = qf.adapters(bf(2, 8, 64), bf(2, 32, 8), scale)
    ids, ws = torch.zeros(4, dtype=torch.int32, device="cuda"), qf.lora_rows_workspace(a, 4)
    with pytest.raises(TypeError):
        qf.lora_rows(a, ids.long(), bf(4, 64), bf(4, 32), ws)
    with pytest.raises(ValueError):
        qf.lora_rows(a, ids[:3], bf(4, 64), bf(4, 32), ws)
    with pytest.raises(ValueError):
        qf.lora_rows(a, ids, bf(4, 64), bf(4, 32), ws, base=torch.zeros(4, 32, device="cuda"))
    with pytest.raises(ValueError):
        qf.lora_rows(a, ids, bf(4, 72), bf(4, 32), ws)
    with pytest.raises(qf.QFError):
        qf.lora_rows(a, ids, bf(4, 64), bf(4, 32), ws[:8])
