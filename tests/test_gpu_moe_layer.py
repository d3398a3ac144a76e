"""The router, sort, grouped experts, weighted sum and packed products together, as
examples/moe_layer.py runs them, against the whole layer in FP64 on the oracle's W_hat.

Between the inputs and any result lie at most eight roundings to bf16 (logits, gate/up, activation,
down, weighted sum, and as many on the way back) of 2^-8 relative each; every step is linear or has a
slope near one, so a result's relative error in norm stays below 8 * 2^-8 = 2^-5.  The router's choice
is the layer's own (a tie or near tie of bf16 logits decides it) and is taken from there; tokens are
masked, so some slots are dropped and the rows past the experts' last belong to nobody."""
import importlib.util
import os

import numpy as np
import pytest

import oracle
from oracle import experts as ox
from tests.helpers import bf16_to_f64, from_dev, to_dev

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("moe_layer", os.path.join(ROOT, "examples", "moe_layer.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _f64(t):
    return t.double().cpu().numpy()


def _off(got, ref):
    return float(np.linalg.norm(got - ref) / np.linalg.norm(ref))


@pytest.mark.parametrize("fmt", ["nvfp4", "mxfp4"])
@pytest.mark.parametrize("T,E,H,I,k,score", [(40, 8, 256, 128, 2, "softmax"), (300, 16, 512, 256, 4, "sigmoid")])
def test_training_step_and_serving(example, fmt, T, E, H, I, k, score):
    g = torch.Generator(device="cuda").manual_seed(T)

    def draw(*shape, std=1.0):
        return (torch.randn(shape, generator=g, device="cuda") * std).to(torch.bfloat16)

    Wr, Wgu, Wd = draw(E, H, std=0.05), draw(E, 2 * I, H, std=0.05), draw(E, H, I, std=0.05)
    X, dY = draw(T, H), draw(T, H)
    mask = (torch.rand(T, generator=g, device="cuda") < 0.9).to(torch.uint8)
    layer = example.MoELayer(Wr, Wgu, Wd, k, fmt, score)
    p = layer.plan(T)
    Y, kept = layer.forward(X, p, mask=mask)
    dX, dWr, dWgu, dWd = layer.backward(dY, kept, p)
    torch.cuda.synchronize()

    def hat(W):
        return np.stack([bf16_to_f64(oracle.fakequant(from_dev(w.view(torch.int16)), fmt)) for w in W])

    hgu, hd = hat(Wgu), hat(Wd)
    x, dy, z = _f64(X), _f64(dY), _f64(kept[1])
    ids = kept[2].cpu().numpy()
    assert (ids[mask.cpu().numpy() == 0] == -1).all()
    w = np.zeros((T, k))
    for t in range(T):
        c = [int(e) for e in ids[t] if e >= 0]
        w[t, :len(c)] = ox.scores([float(v) for v in z[t]], c, score, True)
    off, row_of, slot_of = ox.dispatch(ids, E)
    assert off[E] < T * k                                          # some slots were dropped
    assert np.array_equal(kept[5].cpu().numpy(), row_of)
    xg, n = ox.gather(slot_of, x, k), T * k
    G, A, yg = np.zeros((n, 2 * I)), np.zeros((n, I)), np.zeros((n, H))
    for e in range(E):
        s = slice(off[e], off[e + 1])
        G[s] = xg[s] @ hgu[e].T
        a, b = G[s, :I], G[s, I:]
        A[s] = a / (1 + np.exp(-a)) * b
        yg[s] = A[s] @ hd[e].T
    y = ox.combine(row_of, yg, w)
    assert _off(_f64(Y), y) < 2.0 ** -5
    dyg, dw = ox.combine_bwd(row_of, dy, yg, w)
    dz = ox.route_bwd(z, ids, dw, score, True)
    dxg, rgu, rd = np.zeros((n, H)), np.zeros(Wgu.shape), np.zeros(Wd.shape)
    for e in range(E):
        s = slice(off[e], off[e + 1])
        rd[e] = dyg[s].T @ A[s]
        da, a, b = dyg[s] @ hd[e], G[s, :I], G[s, I:]
        sg = 1 / (1 + np.exp(-a))
        dg = np.concatenate([da * b * (sg + a * sg * (1 - sg)), da * a * sg], axis=1)
        rgu[e] = dg.T @ xg[s]
        dxg[s] = dg @ hgu[e]
    dx = ox.combine(row_of, dxg) + dz @ _f64(Wr)
    for name, got, ref in (("dX", dX, dx), ("dWr", dWr, dz.T @ x), ("dWgu", dWgu, rgu), ("dWd", dWd, rd)):
        assert _off(_f64(got), ref) < 2.0 ** -5, name

    # served from the packed experts (weights not rounded to bf16: 2^-8 each), a few tokens and one
    gu, d = layer.packed(p["gu"], p["gu_saved"]), layer.packed(p["d"], p["d_saved"])
    live = np.nonzero(mask.cpu().numpy())[0]
    for rows in (live[:9], live[-1:]):
        few = X[to_dev(rows)].contiguous()
        out = layer.serve(few, gu, d, example.qf.moe_dispatch_workspace(len(rows), E, k))
        assert _off(_f64(out), y[rows]) < 2.0 ** -5
