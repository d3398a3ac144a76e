"""The decode step's FP64 reference against closed forms and against plain loops that share nothing with it."""
import math

import numpy as np

import oracle
from oracle import serving as sv


def test_places():
    table = np.array([[3, 1], [2, 9]], np.int32)
    got = sv.places(np.array([0, 3, 4]), [5, 1], table, 4, 4, 6)
    assert got == [(3, 2), (3, 3), (1, 0), (2, 0), "nobody", "nobody"]
    assert sv.places(np.array([0, 3, 4]), [2, 6], table, 4, 4, 4) == [None, (3, 0), (3, 1), None]   # page 9 is none
    assert sv.places(None, [8, 9], table, 4, 4, 2) == [(1, 3), None]                               # past the table


def test_quantized_heads_are_the_quantizers():
    rng = np.random.default_rng(0)
    x = ((rng.standard_normal((3, 128)) * 2).astype(np.float32).view(np.uint32) >> 16).astype(np.uint16)
    codes, scales, S, hat = sv.quantize_heads(x, 2, "nvfp4", [4.0, 6.0])
    one = oracle.nvfp4(x[:, 64:], 6.0)
    assert np.array_equal(codes[:, 1], one["codes"]) and np.array_equal(scales[:, 1], one["scales"]) and S[1] == np.float32(one["S"])
    assert np.array_equal(hat[:, 1], one["xhat"])
    # what is written is what the pool's values decode to
    pool = np.zeros((2, 2, 16, 32), np.uint8), np.zeros((2, 2, 16, 4), np.uint8)
    c, s = sv.write(*pool, [(1, 5), None, (0, 0)], codes, scales)
    v = sv.values(c, s, S, "nvfp4")
    assert np.all(np.abs(v[1, 1, 5] - oracle.bf16_array_to_f64(hat[0, 1])) <= 2.0 ** -8 * np.abs(v[1, 1, 5]))
    assert np.all(v[1, :, 6] == 0) and np.array_equal(c[0, :, 0], codes[2])


def test_attention_closed_forms():
    D, page = 4, 2
    K, V = np.zeros((2, 1, page, D)), np.zeros((2, 1, page, D))
    V[0, 0, 0], V[0, 0, 1], V[1, 0, 0] = 1, 2, 6
    table = np.array([[0, 1]], np.int32)
    q = np.ones((1, 2, D))
    O, lse, *_ = sv.attention(q, K, V, None, [3], table, 0.5)       # equal scores: the mean
    assert np.allclose(O, 3) and np.allclose(lse, math.log(3))
    K[1, 0, 0] = math.log(5) / 2                                    # a score of log 5 for the last token
    O, lse, *_ = sv.attention(q, K, V, None, [3], table, 0.5)
    assert np.allclose(O, (1 + 2 + 5 * 6) / 7) and np.allclose(lse, math.log(7))
    O, lse, *_ = sv.attention(q, K, V, None, [3], table, 0.5, window=1)
    assert np.allclose(O, 6) and np.allclose(lse, math.log(5))
    O, lse, *_ = sv.attention(np.ones((3, 2, D)), K, V, np.array([0, 3]), [3], table, 0.5)   # causal rows
    assert np.allclose(O[:, 0, 0], [1, 1.5, 33 / 7])
    O, lse, *_ = sv.attention(np.ones((2, 2, D)), K, V, np.array([0, 2]), [1], table, 0.5)   # a row below zero
    assert np.all(O[0] == 0) and np.all(lse[0] == -math.inf) and np.allclose(O[1], 1)
    table[0, 0] = 7                                                 # a page that is none
    O, _, *_ = sv.attention(q, K, V, None, [3], table, 0.5)
    assert np.allclose(O, 6)


def test_attention_by_loops():
    rng = np.random.default_rng(1)
    H, G, D, page, lens, new = 2, 3, 8, 4, [9, 6], [4, 1]
    K, V = rng.standard_normal((2, 6, H, page, D))
    table = rng.permutation(6).reshape(2, 3).astype(np.int32)
    q = rng.standard_normal((5, H * G, D))
    O, lse, *_ = sv.attention(q, K, V, np.array([0, 4, 5]), lens, table, 0.3, window=3)
    t = 0
    for b in range(2):
        for i in range(new[b]):
            own = lens[b] - new[b] + i
            for h in range(H * G):
                num, den = np.zeros(D), 0.0
                for p in range(max(0, own - 2), own + 1):
                    w = math.exp(0.3 * float(np.dot(q[t, h], K[table[b, p // page], h // G, p % page])))
                    num, den = num + w * V[table[b, p // page], h // G, p % page], den + w
                assert np.allclose(O[t, h], num / den) and math.isclose(lse[t, h], math.log(den))
            t += 1


def test_adapters():
    A, B = np.arange(12.0).reshape(2, 2, 3), np.array([[[1.0, 0], [0, 1]], [[2, 1], [1, 0]]])
    x = np.array([[1.0, 0, 0], [0, 1, 0], [1, 1, 1]])
    Y, mag = sv.lora_rows([1, 2, 0], x, A, B, [1.0, 0.5], base=np.ones((3, 2)))
    # row 0: A_1 x = (6, 9), B_1 z = (21, 6), halved; row 1 has no adapter; row 2: A_0 x = (3, 12)
    assert np.array_equal(Y, [[11.5, 4], [1, 1], [4, 13]]) and np.array_equal(mag[1], [0, 0])
    Y, _ = sv.lora_rows([1, 2, 0], x, A, B, [1.0, 0.5], ranks=[1, 0])
    assert np.array_equal(Y, [[0, 0], [0, 0], [3, 0]])
