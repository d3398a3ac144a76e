"""GPU: the attention over the 4-bit cache at the ends of FP32's range: large scores, scales of queries and heads
that only together are ordinary, heads of tiny values."""
import numpy as np
import pytest

import workloads
from oracle import serving as sv
from tests import kv_cases as kc
from tests.helpers import bf16_to_f64, to_dev
from tests.test_gpu_kv import U, _attend, _cache, _check, _seqs

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def qf():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_39223_amd as qf
    qf.lib()
    return qf


# tokens, new tokens, heads of queries to one of keys: one piece and several, 16 and 32 rows a wave, 128 a workgroup
CALLS = [([200, 70], None, 4), ([700, 60], None, 4), ([700, 60], [9, 7], 4), ([700, 300], [60, 50], 3)]


@pytest.mark.parametrize("fmt", ["nvfp4", "mxfp4"])
@pytest.mark.parametrize("lens,new,G", CALLS)
@pytest.mark.parametrize("size", [20, 22, 23, 24, 25, 26, 28, 30, 40, 100])
@pytest.mark.parametrize("one", [None, 0, 63, 256, 690])
def test_scores_of_any_size(qf, fmt, lens, new, G, size, one):
    """Scores about 2^size: all keys the same, but one twice as large.  A row whose scores are positive gets that
    token's value if it sees it, every other row the mean of the other values it sees.

    Equal keys have equal scores bit for bit, so probabilities are equal and add nothing but their own rounding:
    (2^-11 + (n / 2 + 192) u) of the mean of |v|, and 2^-8 of the output.  Scores apart by more than 2^6 leave nothing
    of the smaller.  The log-sum-exp has the score's error, (D + 16) u of sum |q||k| |scale|."""
    D, H, page = 64, 2, 16
    rng = np.random.default_rng(size + sum(lens))
    B, cols, T = len(lens), -(-max(lens) // page), len(lens) if new is None else sum(new)
    table, offsets = kc.table(rng, B, cols, B * cols), None if new is None else kc.offsets_of(new)
    k, v = kc.pool(rng, fmt, B * cols, H, page, D), kc.pool(rng, fmt, B * cols, H, page, D)
    k[0][:], k[1][:] = k[0][:1, :, :1], 0x40 if fmt == "nvfp4" else 124
    for b in range(B):
        if one is not None and one < lens[b]:
            k[1][table[b, one // page], :, one % page] += 8 if fmt == "nvfp4" else 1
    qh = workloads.normal_bf16(rng, (T, H * G * D))
    q = bf16_to_f64(qh).reshape(T, H, G, D)
    key = sv.values(k[0][:1, :, :1], np.full_like(k[1][:1, :, :1], 0x40 if fmt == "nvfp4" else 124), k[2], fmt)[0, :, 0]   # [H, D]
    z = np.einsum("thgd,hd->thg", q, key)
    scale = float(np.float32(2.0 ** size / np.abs(z).mean()))
    z = z * scale
    assert np.abs(z).min() > 2.0 ** 6
    big = scale * np.einsum("thgd,hd->thg", np.abs(q), np.abs(key))
    V = sv.values(*v, fmt)
    o, l = _attend(qf, _cache(qf, fmt, k, v), _seqs(qf, lens, table, offsets), to_dev(qh), H, D, H * G, scale)
    o, l = o.reshape(T, H, G, D), l.reshape(T, H, G)
    for b in range(B):
        rows = [b] if new is None else range(offsets[b], offsets[b + 1])
        for i, t in enumerate(rows):
            own = lens[b] - len(rows) + i
            pos = np.arange(own + 1)
            vals = V[table[b, pos // page], :, pos % page]                              # [n, H, D]
            rest = pos[pos != one] if one is not None else pos
            for h in range(H):
                for g in range(G):
                    twice = one is not None and one <= own and (z[t, h, g] > 0 or len(rest) == 0)
                    those = [one] if twice else rest
                    want, mag = vals[those, h].mean(0), np.abs(vals[those, h]).mean(0)
                    n = len(those)
                    bound = (2.0 ** -11 + (n / 2 + 192) * U) * mag + 2.0 ** -8 * np.abs(want)
                    assert np.all(np.abs(o[t, h, g] - want) <= bound), (t, h, g, o[t, h, g], want)
                    top = z[t, h, g] * (2 if twice else 1)
                    lbound = (D + 16) * U * big[t, h, g] * 2 + (n / 4 + 80) * U + 4 * U * abs(top)
                    assert abs(l[t, h, g] - (top + np.log(n))) <= lbound, (t, h, g)


@pytest.mark.parametrize("lens,new,G", CALLS)
@pytest.mark.parametrize("scale,S,query", [(1.3 * 2.0 ** -100, 2.0 ** -46, 2.0 ** 127), (-(2.0 ** -110), 2.0 ** -43, 2.0 ** 127),
                                           (2.0 ** -149, 2.0 ** 20, 2.0 ** 119), (2.0 ** 90, 2.0 ** 39, 2.0 ** -126),
                                           (-(2.0 ** 90), 2.0 ** 39, 2.0 ** -126)])
def test_scales_that_meet_in_the_middle(qf, lens, new, G, scale, S, query):
    """A scale times a head's tensor scale outside FP32's range, or where it has few bits left, times queries that bring
    the scores back to ordinary size."""
    D, H, page = 256, 2, 16
    rng = np.random.default_rng(3)
    B, cols, T = len(lens), -(-max(lens) // page), len(lens) if new is None else sum(new)
    table, offsets = kc.table(rng, B, cols, B * cols), None if new is None else kc.offsets_of(new)
    k, v = kc.pool(rng, "nvfp4", B * cols, H, page, D), kc.pool(rng, "nvfp4", B * cols, H, page, D)
    k[0][:] &= 0x77                                                # (all positive, so that 256 of them add up)
    k[1][:] = rng.integers(0x08, 0x10, k[1].shape) if query < 1 else rng.integers(0x70, 0x7E, k[1].shape)
    k = k[0], k[1], np.full(H, S, np.float32)
    qh = np.full((T, H * G * D), int(np.float32(query).view(np.uint32)) >> 16, np.uint16)
    qh[:, ::5] -= 0x20                                             # (some a little smaller)
    ref = sv.attention(bf16_to_f64(qh).reshape(T, H * G, D), sv.values(*k, "nvfp4"), sv.values(*v, "nvfp4"), offsets, lens, table,
                       scale)
    assert 2.0 ** -10 < np.abs(ref[2]).max() < 2.0 ** 10
    o, l = _attend(qf, _cache(qf, "nvfp4", k, v), _seqs(qf, lens, table, offsets), to_dev(qh), H, D, H * G, scale)
    _check(o, l, ref, max(lens), D)


@pytest.mark.parametrize("D", [64, 256])
@pytest.mark.parametrize("lens,new,G", CALLS)
@pytest.mark.parametrize("S", [2.0 ** -100, 2.0 ** -118, 2.0 ** -124])
def test_heads_of_tiny_values(qf, D, lens, new, G, S):
    """Values near the least normal number come out as precise as any."""
    H, page = 2, 16
    rng = np.random.default_rng(4)
    B, cols, T = len(lens), -(-max(lens) // page), len(lens) if new is None else sum(new)
    table, offsets = kc.table(rng, B, cols, B * cols), None if new is None else kc.offsets_of(new)
    k, v = kc.pool(rng, "nvfp4", B * cols, H, page, D), kc.pool(rng, "nvfp4", B * cols, H, page, D)
    v = v[0], v[1], np.full(H, S, np.float32)
    qh = workloads.normal_bf16(rng, (T, H * G * D))
    ref = sv.attention(bf16_to_f64(qh).reshape(T, H * G, D), sv.values(*k, "nvfp4"), sv.values(*v, "nvfp4"), offsets, lens, table,
                       D ** -0.5)
    o, l = _attend(qf, _cache(qf, "nvfp4", k, v), _seqs(qf, lens, table, offsets), to_dev(qh), H, D, H * G)
    _check(o, l, ref, max(lens), D)
