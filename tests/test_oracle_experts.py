"""The FP64 reference of the router, the sort by expert, the weighted sum and the packed decode:
hand-worked rows, gradients against central differences, the decode against the format codecs, and
planted mistakes that the checks notice."""
import math

import numpy as np
import pytest

import oracle
from oracle import experts as ox
from tests.helpers import bf16_to_f64


def test_choice_order_ties_and_rows_without_experts():
    inf = math.inf
    assert ox.choose([1.0, 3.0, 3.0, -2.0], 3) == [1, 2, 0]
    assert ox.choose([-inf, 0.5, -inf, 0.5], 3) == [1, 3]
    assert ox.choose([-inf, -inf], 2) == []
    assert ox.choose([1.0, math.nan, inf], 2) == [1, 2]
    assert ox.choose([0.0, -0.0], 2) == [0, 1]


def test_hand_worked_weights():
    ids, w = ox.route(np.log(np.array([[1.0, 2.0, 5.0]])), 2, norm=False)
    assert ids.tolist() == [[2, 1]] and np.allclose(w, [[5 / 8, 2 / 8]])
    _, w = ox.route(np.log(np.array([[1.0, 2.0, 5.0]])), 2, scale=2.0)
    assert np.allclose(w, [[10 / 7, 4 / 7]])
    z = np.log(np.array([[1.0, 3.0, 1 / 3]]))                     # sigmoids 1/2, 3/4, 1/4
    assert np.allclose(ox.route(z, 2, "sigmoid", norm=False)[1], [[0.75, 0.5]])
    assert np.allclose(ox.route(z, 2, "sigmoid")[1], [[0.6, 0.4]])
    assert np.allclose(ox.route(np.array([[-900.0, -900.0]]), 2, "sigmoid")[1], [[0.5, 0.5]])


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("norm", [True, False])
def test_router_gradient_against_differences(score, norm):
    rng = np.random.default_rng(5)
    z, dw = rng.normal(size=(6, 7)), rng.normal(size=(6, 3))
    z[2, 1:] = -math.inf                                          # fewer experts than choices
    ids, _ = ox.route(z, 3, score, norm, 1.5, mask=[1, 1, 1, 1, 0, 1])
    dz = ox.route_bwd(z, ids, dw, score, norm, 1.5)
    h = 1e-6
    for t in range(6):
        for e in range(7):
            if z[t, e] == -math.inf:
                assert dz[t, e] == 0
                continue
            f = []
            for s in (h, -h):
                row = [float(v) for v in z[t]]
                row[e] += s
                c = [int(i) for i in ids[t] if i >= 0]            # the choice is held
                f.append(sum(1.5 * q * dw[t, j] for j, q in enumerate(ox.scores(row, c, score, norm))))
            assert abs((f[0] - f[1]) / (2 * h) - dz[t, e]) < 1e-8


def test_sort_is_stable_and_drops_to_the_end():
    off, row_of, slot_of = ox.dispatch(np.array([[2, 0], [-1, 2], [0, 9]], np.int32), 3)
    assert off.tolist() == [0, 2, 2, 4]
    assert row_of.tolist() == [[2, 0], [~4, 3], [1, ~5]]
    assert slot_of.tolist() == [1, 4, 0, 3, -1, -1]


def test_sum_and_gradients_against_differences():
    rng = np.random.default_rng(6)
    _, row_of, slot_of = ox.dispatch(np.array([[1, 0], [-1, 1], [-1, -1]], np.int32), 2)
    X = rng.normal(size=(3, 4))
    Xg = ox.gather(slot_of, X, 2)
    assert np.array_equal(Xg[row_of[0, 0]], X[0]) and np.array_equal(Xg[row_of[1, 1]], X[1])
    assert not Xg[3:].any()
    Yg, w, dY = rng.normal(size=(6, 4)), rng.normal(size=(3, 2)), rng.normal(size=(3, 4))
    loss = lambda yg, ww: float((ox.combine(row_of, yg, ww) * dY).sum())
    dYg, dw = ox.combine_bwd(row_of, dY, Yg, w)
    h = 1e-6
    for i in np.ndindex(Yg.shape):
        d = np.zeros_like(Yg)
        d[i] = h
        assert abs((loss(Yg + d, w) - loss(Yg - d, w)) / (2 * h) - dYg[i]) < 1e-8
    for i in np.ndindex(w.shape):
        d = np.zeros_like(w)
        d[i] = h
        assert abs((loss(Yg, w + d) - loss(Yg, w - d)) / (2 * h) - dw[i]) < 1e-8
    # the copy's gradient is the sum without weights
    dXg = rng.normal(size=(6, 4))
    dX = ox.combine(row_of, dXg)
    for i in np.ndindex(X.shape):
        d = np.zeros_like(X)
        d[i] = h
        f = [float((ox.gather(slot_of, X + s * d, 2) * dXg).sum()) for s in (1, -1)]
        assert abs((f[0] - f[1]) / (2 * h) - dX[i]) < 1e-8


@pytest.mark.parametrize("fmt", ["nvfp4", "mxfp4", "q4k"])
def test_decode_rounds_to_the_quantizers_x_hat(fmt):
    import workloads
    x = workloads.normal_bf16(np.random.default_rng(8), (5, 512), 0.02)
    if fmt == "q4k":
        r = oracle.q4k(x)
        W = ox.decode(fmt, r["packed"].reshape(5, 2, 144))
    else:
        r = getattr(oracle, fmt)(x)
        W = ox.decode(fmt, r["codes"], r["scales"], r.get("S"))
    hat = bf16_to_f64(r["xhat"])
    # x_hat is this value after at most three binary32 roundings and one to bf16 (8 significant bits)
    assert np.all(np.abs(W - hat) <= 2.0 ** -8 * np.abs(W) * 1.001 + (2.0 ** -22 * 0.02 * 16 if fmt == "q4k" else 0))


def test_planted_mistakes_are_noticed():
    rng = np.random.default_rng(9)
    z = np.round(rng.normal(size=(20, 9)))                        # many ties
    ids, w = ox.route(z, 4)
    wrong = np.argsort(-z[:, ::-1], axis=1, kind="stable")[:, :4]
    assert not np.array_equal(ids, 8 - wrong)                     # ties to the highest expert
    _, w_all = ox.route(z, 4, norm=False)
    assert np.abs(w - w_all).max() > 0.05
    off, row_of, _ = ox.dispatch(ids, 9)
    assert not np.array_equal(np.argsort(ids.reshape(-1), kind="stable").reshape(ids.shape), row_of)
    d = rng.integers(0, 256, size=(3, 1, 144)).astype(np.uint8)
    d[..., 1] = d[..., 3] = 0x2C                                  # finite FP16 scales
    swapped = d.copy()
    swapped[..., 4:8], swapped[..., 8:12] = d[..., 8:12], d[..., 4:8]
    assert not np.array_equal(ox.decode("q4k", d), ox.decode("q4k", swapped))
