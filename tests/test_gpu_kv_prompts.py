"""GPU: the 4-bit cache written and read back bit for bit in the forms that prompts take, two and eight tokens a lane
(from 2 and 10 units of 512 lanes a compute unit on), with tails in every group of tokens.

With several tokens a lane the two lanes of an NVFP4 block share its scales' divisions, one taking the even tokens, the
other the odd ones: blocks with a NaN, an infinity, zeros or one element alone lie in tokens of either kind and in either
half of a block, beside ordinary ones.  Rows without a place and rows of nobody are among them."""
import numpy as np
import pytest

import workloads
from oracle import serving as sv
from tests import kv_cases as kc
from tests.helpers import bf16_to_f64, from_dev, to_dev
from tests.test_gpu_kv import _cache, _seqs

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def qf():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_39223_amd as qf
    qf.lib()
    return qf


# heads, their size, tokens (just past a threshold at 256 compute units, and odd), page
TWO = [(128, 128, 67, 16), (3, 256, 1369, 64), (2, 128, 4101, 32), (1, 64, 16391, 128)]
EIGHT = [(128, 128, 323, 16), (3, 256, 6831, 64), (2, 128, 20487, 32), (1, 64, 81927, 128)]


def _rows(rng, T, C):
    """bf16 [T, C]: ordinary values and, in some tokens, blocks that are not."""
    x = workloads.normal_bf16(rng, (T, C))
    for value in (0x7FC0, 0x7F80, 0xFF80, 0x0000, 0x8000, 0x0001, 0x7F00):
        for t in rng.integers(0, T, 12):
            c = int(rng.integers(0, C))
            if value in (0x0000, 0x8000):
                x[t, c // 32 * 32:c // 32 * 32 + 32] = value       # (whole blocks of zeros)
            elif value == 0x0001:
                x[t, c // 32 * 32:c // 32 * 32 + 32] = 0           # the least subnormal alone among zeros
                x[t, c] = value
            else:
                x[t, c] = value
    return x


def _with_nans(qf, ref, x, H, amax):
    """The oracle leaves open what a block with a NaN under a given tensor scale becomes: its codes are those of the library's
    quantizer, its scale is NaN, and it is read back as NaN."""
    rows = np.nonzero(((x & 0x7FFF) > 0x7F80).any(1))[0]
    D = x.shape[1] // H
    xs = x[rows].reshape(len(rows), H, D)
    for h in range(H):
        out = [torch.zeros(len(rows), n, dtype=t, device="cuda") for n, t in ((D // 2, torch.uint8), (D // 16, torch.uint8), (D, torch.int16))]
        qf.fakequant_nvfp4(to_dev(np.ascontiguousarray(xs[:, h])), to_dev(amax[h:h + 1].copy()), qf.AMAX_GIVEN, None, *out)
        for r, o in zip((ref[0], ref[1], ref[3]), out):
            r[rows, h] = from_dev(o)
    bad = ((xs & 0x7FFF) > 0x7F80).reshape(len(rows), H, D // 16, 16).any(-1)
    assert np.all(ref[1][rows][bad] == 0x7F)
    hat = ref[3][rows].reshape(*bad.shape, 16)
    hat[bad] = 0x7FC0
    ref[3][rows] = hat.reshape(len(rows), H, D)


@pytest.mark.parametrize("fmt", ["nvfp4", "mxfp4"])
@pytest.mark.parametrize("H,D,T,page", TWO + EIGHT)
@pytest.mark.parametrize("ragged", [False, True])
def test_written_and_read(qf, fmt, H, D, T, page, ragged):
    rng = np.random.default_rng(T + D)
    if ragged:
        cuts = np.sort(rng.integers(0, T - 5, 3))
        new = [int(v) for v in np.diff(np.concatenate([[0], cuts, [T - 5]]))] + [0]     # (the last 5 rows are nobody's)
        lens = [n + int(rng.integers(0, 50)) for n in new]
        lens[1] = max(new[1] - 3, 0)                               # its first rows are below zero
    else:
        new, lens = None, None
    if new is None:                                                # a token a sequence
        B = T
        lens = [int(v) for v in rng.integers(0, 3 * page, B)]
    else:
        B = len(new)
    cols = -(-max(lens) // page)
    table = kc.table(rng, B, cols, B * cols + 1)
    table[rng.integers(0, B, 2), rng.integers(0, cols, 2)] = [-1, B * cols + 1]
    if ragged:
        lens[0] = cols * page + 2                                  # its last two rows are past the table
    offsets = None if new is None else kc.offsets_of(new)
    # pages of a token a sequence are many; of wide heads a few shared ones (rows still have a place each)
    if new is None:
        table[:, :] = -1
        order, p = rng.permutation(T), max(1, -(-T // page))
        for b in range(B):
            lens[b] = int(order[b] % page) + 1
            table[b, 0] = order[b] // page
        table[::17, 0] = -7
        pages = p
    else:
        pages = B * cols + 1
    x = [_rows(rng, T, H * D) for _ in range(2)]
    finite = [np.where((a & 0x7F80) == 0x7F80, 0, a) for a in x]
    amax = [(np.abs(bf16_to_f64(np.where((a & 0x7FFF) > 0x4200, 0, a))).max() * (0.3 + rng.random(H))).astype(np.float32) for a in finite]
    ref = [sv.quantize_heads(a, H, fmt, g) for a, g in zip(x, amax)]
    if fmt == "nvfp4":
        for r, a, m in zip(ref, x, amax):
            _with_nans(qf, r, a, H, m)
    where = sv.places(offsets, lens, table, page, pages, T)
    assert None in where and (new is None or "nobody" in where)
    block = kc.BLOCK[fmt]
    old = [(np.full((pages, H, page, D // 2), 0x5A, np.uint8), np.full((pages, H, page, D // block), 0x31, np.uint8), r[2]) for r in ref]
    cache, seqs = _cache(qf, fmt, *old), _seqs(qf, lens, table, offsets)
    qf.kv_write(cache, seqs, to_dev(x[0]), to_dev(x[1]))
    got = [from_dev(t) for t in cache._tensors[:4]]
    for i in range(2):
        codes, scales = sv.write(old[i][0], old[i][1], where, ref[i][0], ref[i][1])
        assert np.array_equal(got[2 * i + 1], scales) and np.array_equal(got[2 * i], codes)
    out = [torch.full((T, H * D), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    qf.kv_read(cache, seqs, *out)
    kinds = np.array([2 if w == "nobody" else 1 if w is None else 0 for w in where])
    for i in range(2):
        want = np.where((kinds == 2)[:, None], np.uint16(0x40E0), np.where((kinds == 1)[:, None], np.uint16(0), ref[i][3].reshape(T, -1)))
        assert np.array_equal(from_dev(out[i].view(torch.int16)), want)
