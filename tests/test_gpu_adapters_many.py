"""GPU: adapters of more than 64 rows, which are put in order first: NaN and infinities stay where they belong though rows
of other adapters ride along in the same products, and a captured call follows its ids.

Forms: groups of 16 rows with several adapters, groups of one adapter (64 rows an adapter and more: 32 at a time),
operands of ranks 17 to 32 through LDS with odd ends of K, and more adapters than are put in order."""
import numpy as np
import pytest

from tests.helpers import to_dev
from tests.test_gpu_adapters import _case, _check, _ref, _run

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

# rows, adapters, rank, K, N, rows of an adapter side by side
FORMS = [(100, 7, 16, 256, 72, False), (300, 40, 32, 328, 64, False), (200, 2, 32, 200, 136, True), (260, 3, 24, 1096, 40, False),
         (150, 1, 64, 264, 64, True), (90, 8300, 8, 64, 24, False)]


@pytest.fixture(scope="module")
def qf():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_39223_amd as qf
    qf.lib()
    return qf


def _ids(rng, M, n, runs):
    return np.arange(M) * n // M if runs else rng.choice(rng.permutation(n)[:12], M)


@pytest.mark.parametrize("M,n,r,K,N,runs", FORMS)
@pytest.mark.parametrize("f32", [False, True])
def test_non_finite_rows(qf, M, n, r, K, N, runs, f32):
    """A NaN or infinity in a row of X, or in base, stays in its row or its element."""
    rng = np.random.default_rng(M)
    c = _case(rng, M, n, r, K, N, _ids(rng, M, n, runs))
    clean = _run(qf, c, f32)
    _check(clean, *_ref(c), r, K, f32)
    c["X"][M // 3, K - 1], c["X"][M - 1, 0] = 0x7FC0, 0xFF80
    c["base"][5, 7] = 0x7FC0
    got = _run(qf, c, f32)
    assert np.isnan(got[M // 3]).all() and not np.isfinite(got[M - 1]).any() and np.isnan(got[5, 7])
    rest = np.ones((M, N), bool)
    rest[[M // 3, M - 1]], rest[5, 7] = False, False
    assert np.array_equal(got[rest], clean[rest])


@pytest.mark.parametrize("M,n,r,K,N,runs", FORMS)
@pytest.mark.parametrize("what", ["A", "B", "scale"])
def test_non_finite_adapters(qf, M, n, r, K, N, runs, what):
    """A NaN in an adapter reaches its own rows and no others, one in an adapter without rows nobody."""
    rng = np.random.default_rng(M + 1)
    ids = _ids(rng, M, n, runs)
    ids[::9] = -1
    c = _case(rng, M, n, r, K, N, ids)
    clean = _run(qf, c)
    own = int(ids[M // 2 + (M // 2 % 9 == 0)])
    spoiled = [own] + [a for a in range(n) if a not in ids][:1]
    for a in spoiled:
        if what == "scale":
            c["scale"][a] = np.nan
        else:
            c[what][a, -1, -1] = 0x7FC0
    got = _run(qf, c)
    bad = np.zeros((M, N), bool)
    bad[ids == own, -1 if what == "B" else slice(None)] = True
    assert bad.any() and np.array_equal(np.isnan(got), bad) and np.array_equal(got[~bad], clean[~bad])


@pytest.mark.parametrize("M,n,r,K,N,runs", FORMS)
def test_captured_with_changing_ids(qf, M, n, r, K, N, runs):
    rng = np.random.default_rng(M + 2)
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
        new = _ids(rng, M, n, runs) if i % 2 else rng.integers(-1, n + 1, M)
        ids.copy_(torch.from_numpy(np.asarray(new).astype(np.int32)))
        X.normal_()
        base.normal_()
        ws[0].fill_(0xFF)
        graph.replay()
        qf.lora_rows(a, ids, X, Y[1], ws[1], base=base)
        torch.cuda.synchronize()
        assert torch.equal(Y[0], Y[1])
