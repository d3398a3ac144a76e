"""The grouped layer, plain and with LoRA factors, on rows of which the last belong to no expert
(off[E] < T, what a sort with dropped slots leaves): NaN in those rows of X and dY reaches nothing, those
rows of Y and dX keep what they held, and everything else equals the call without them bit for bit."""
import numpy as np
import pytest

import workloads
from tests.helpers import from_dev, to_dev

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
HELD = 0x4123


@pytest.fixture(scope="module")
def qf():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_39223_amd as qf
    qf.lib()
    return qf


def _offsets(counts):
    off = np.zeros(len(counts) + 1, np.int64)
    off[1:] = np.cumsum(counts)
    return off


def _tailed(a, tail):
    return to_dev(np.concatenate([a, np.full((tail, a.shape[1]), 0x7FC0, np.uint16)]))


def _held(rows, cols):
    return torch.full((rows, cols), HELD, dtype=torch.int16, device="cuda")


def _same(got, want, live):
    """The rows of experts alike bit for bit, the others as they were."""
    assert np.array_equal(from_dev(got)[:live], from_dev(want)[:live])
    assert bool((got[live:] == HELD).all())


# (counts of rows, N, K, rows of no expert): more than 96 rows an expert with dY^T written by the dX
# launch (K >= 1793) and by the transposer; the last expert's rows ending inside and at a tile; few rows
# an expert (128-row tiles, experts decoded in the forward from 128 experts or tile columns on); none at all
SHAPES = [([300, 0, 513, 77], 264, 2048, 200), ([300, 0, 513, 77], 264, 512, 200), ([256, 512], 72, 2304, 1),
          ([700, 64, 0], 40, 256, 300), ([7, 0, 33, 64], 136, 512, 60), ([3, 1] * 64 + [20], 264, 256, 41),
          ([0, 0, 0], 64, 256, 50)]


@pytest.mark.parametrize("wfmt,afmt", [("nvfp4", "none"), ("mxfp4", "mxfp4"), ("q4k", "mxfp4"), ("none", "none")])
@pytest.mark.parametrize("counts,N,K,tail", SHAPES)
@pytest.mark.parametrize("way", ["again", "kept", "saved"])
def test_grouped_layer(qf, wfmt, afmt, counts, N, K, tail, way):
    rng = np.random.default_rng(N + K + tail)
    E, off = len(counts), _offsets(counts)
    live = int(off[-1])
    X, dY = workloads.normal_bf16(rng, (live, K)), workloads.normal_bf16(rng, (live, N))
    Wd, offd = to_dev(workloads.normal_bf16(rng, (E * N, K), 0.02)), to_dev(off)

    def run(extra):
        T = live + extra
        d = qf.grouped_desc(E, T, N, K, wfmt, afmt)
        ws = qf.grouped_workspace(d)
        ws.fill_(0xFF)                                             # NaN in every type that lies there
        sv = qf.grouped_saved_buffer(d) if way == "saved" else None
        x, dy = _tailed(X, extra), _tailed(dY, extra)
        Y, dX = _held(T, N), _held(T, K)
        dW = torch.full((E, N, K), 7.0, device="cuda")
        qf.qlinear_grouped_fwd(d, offd, x, Wd, Y, ws, saved=sv)
        if way == "kept":
            d = qf.grouped_desc(E, T, N, K, wfmt, afmt, flags=qf.FLAG_REUSE_WS)
        qf.qlinear_grouped_bwd_ste(d, offd, dy, x, Wd, dX, dW, ws, saved=sv)
        alone = torch.full((E, N, K), 7.0, device="cuda")
        qf.qlinear_grouped_bwd_ste(d, offd, dy, x, Wd, None, alone, ws, saved=sv)
        torch.cuda.synchronize()
        return Y, dX, dW, alone

    want, got = run(0), run(tail)
    _same(got[0], want[0], live)
    _same(got[1], want[1], live)
    for a in got[2:]:
        assert bool(torch.isfinite(a).all()) and torch.equal(a, want[2])


@pytest.mark.parametrize("wfmt,afmt,shared", [("nvfp4", "none", "A"), ("mxfp4", "mxfp4", ""), ("q4k", "none", "B")])
@pytest.mark.parametrize("counts,tail", [([37, 0, 300, 5, 1100, 64], 90), ([5, 0, 33], 240), ([0, 0], 20)])
def test_grouped_lora(qf, wfmt, afmt, shared, counts, tail):
    rng = np.random.default_rng(tail)
    E, off, N, K, r = len(counts), _offsets(counts), 264, 512, 20
    live = int(off[-1])
    X, dY = workloads.normal_bf16(rng, (live, K)), workloads.normal_bf16(rng, (live, N))
    Wd, offd = to_dev(workloads.normal_bf16(rng, (E * N, K), 0.02)), to_dev(off)
    A = torch.from_numpy(rng.standard_normal((r, K) if shared == "A" else (E, r, K)).astype(np.float32)).cuda()
    B = torch.from_numpy(rng.standard_normal((N, r) if shared == "B" else (E, N, r)).astype(np.float32)).cuda()
    lo = qf.lora(A * K ** -0.5, B * 0.01, 2.0, a_shared=shared == "A", b_shared=shared == "B")

    def run(extra):
        T = live + extra
        d = qf.grouped_desc(E, T, N, K, wfmt, afmt)
        ws = qf.grouped_lora_workspace(d, lo)
        ws.fill_(0xFF)
        x, dy = _tailed(X, extra), _tailed(dY, extra)
        Y, dX = _held(T, N), _held(T, K)
        dA, dB = torch.full_like(A, 7.0), torch.full_like(B, 7.0)
        qf.qlinear_grouped_lora_fwd(d, lo, offd, x, Wd, Y, ws)
        qf.qlinear_grouped_lora_bwd_ste(d, lo, offd, dy, x, Wd, dX, dA, dB, ws)
        torch.cuda.synchronize()
        return Y, dX, dA, dB

    want, got = run(0), run(tail)
    _same(got[0], want[0], live)
    _same(got[1], want[1], live)
    for a, b in zip(got[2:], want[2:]):
        assert bool(torch.isfinite(a).all()) and torch.equal(a, b)
