"""GPU: NaN and infinities in the attention over the 4-bit cache where a row's tokens are taken in several pieces,
and in rows that see nothing.

What a row that sees something owes to them: a NaN or infinity in its query makes all of it NaN, so does a
NaN scale among the keys that it sees, whichever piece they are in.  A row that sees nothing gets zeros and
-inf whatever its query holds, and whatever other rows see.  Rows that are not NaN keep the bounds of
tests/test_gpu_kv.py."""
import numpy as np
import pytest

import workloads
from oracle import serving as sv
from tests import kv_cases as kc
from tests.helpers import bf16_to_f64, to_dev
from tests.test_gpu_kv import _attend, _cache, _check, _seqs

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

# tokens, new tokens (None: one each), heads of queries to one of keys; in calls of so many pieces of 256 tokens:
# 16 rows a wave, 32, and 128 a workgroup, which heads of 256 do not take; few pieces and many (two merges)
CALLS = [([700, 60], None, 4, 3), ([2700, 300], None, 4, 11), ([700, 60], [9, 7], 4, 3), ([2700, 300], [9, 7], 4, 11),
         ([700, 300], [60, 50], 3, 3), ([2700, 300], [60, 50], 3, 11)]


@pytest.fixture(scope="module")
def qf():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_39223_amd as qf
    qf.lib()
    return qf


class Call:
    """Pools of arbitrary codes and the sequences of a call."""

    def __init__(self, qf, fmt, lens, new, G, D, pieces=None, H=2, page=16, window=0, max_len=None, seed=0):
        rng = np.random.default_rng(seed + D + len(lens))
        self.qf, self.fmt, self.lens, self.H, self.Hq, self.D, self.page = qf, fmt, lens, H, H * G, D, page
        self.window, self.max_len = window, max_len
        B, cols = len(lens), max(1, -(-max(lens) // page))
        self.table = kc.table(rng, B, cols, B * cols + 1)
        self.offsets = None if new is None else kc.offsets_of(new)
        self.T = B if new is None else sum(new)
        self.k, self.v = (kc.pool(rng, fmt, B * cols + 1, H, page, D) for _ in range(2))
        self.q = workloads.normal_bf16(rng, (self.T, self.Hq * D))
        if pieces is not None:
            ws = qf.kv_attention_workspace(_cache(qf, fmt, self.k, self.v), self._sequences(), self.T, self.Hq, window=window)
            assert ws.numel() // (self.T * self.Hq * (D + 2) * 4) == pieces

    def _sequences(self):
        return _seqs(self.qf, self.lens, self.table, self.offsets, self.max_len)

    def at(self, b, pos):
        """Page and place of a token."""
        return self.table[b, pos // self.page], pos % self.page

    def run(self, scale=None):
        return _attend(self.qf, _cache(self.qf, self.fmt, self.k, self.v), self._sequences(), to_dev(self.q), self.H, self.D, self.Hq,
                       scale, self.window)

    def ref(self, scale=None):
        return sv.attention(bf16_to_f64(self.q).reshape(self.T, self.Hq, self.D), sv.values(*self.k, self.fmt),
                            sv.values(*self.v, self.fmt), self.offsets, self.lens, self.table,
                            self.D ** -0.5 if scale is None else scale, self.window, self.max_len)

    def check(self, o, l, ref):
        """NaN where the reference is, whole rows, and in bounds elsewhere."""
        bad = np.isnan(ref[1])
        assert np.array_equal(np.isnan(l), bad) and np.array_equal(np.isnan(o), np.broadcast_to(bad[..., None], o.shape))
        o[bad], l[bad] = 7, 7                                      # (as _check wants what is NaN in the reference)
        _check(o, l, ref, max(self.lens), self.D)


@pytest.mark.parametrize("fmt", ["nvfp4", "mxfp4"])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("lens,new,G,pieces", CALLS)
def test_queries_in_several_pieces(qf, fmt, D, lens, new, G, pieces):
    """A NaN, an infinity of either sign in a query: its row is NaN, and all others keep their bits."""
    c = Call(qf, fmt, lens, new, G, D, pieces)
    clean, clean_l = c.run()
    spoiled = [(0, 0, 0x7FC0), (c.T // 2, c.Hq - 1, 0x7F80), (c.T - 1, c.Hq // 2, 0xFF80)]
    for t, h, bits in spoiled:
        c.q[t, h * D + 5 + 7 * h] = bits
    o, l = c.run()
    for t, h, _ in spoiled:
        assert np.isnan(o[t, h]).all() and np.isnan(l[t, h]), (t, h)
        o[t, h], l[t, h] = clean[t, h], clean_l[t, h]
    assert np.array_equal(o, clean) and np.array_equal(l, clean_l)


@pytest.mark.parametrize("fmt", ["nvfp4", "mxfp4"])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("lens,new,G,pieces", [([513, 60], None, 4, 3), ([2561, 300], None, 4, 11), ([513, 60], [9, 7], 4, 3),
                                               ([2561, 300], [9, 7], 4, 11), ([513, 300], [60, 50], 3, 3), ([2561, 300], [60, 50], 3, 11)])
@pytest.mark.parametrize("which", ["a piece", "the last token"])
def test_keys_of_a_whole_piece(qf, fmt, D, lens, new, G, pieces, which):
    """Keys with NaN scales that are all that a row sees in one piece: the second one, or the newest token, which
    is alone in the last."""
    c = Call(qf, fmt, lens, new, G, D, pieces)
    for pos in range(256, 512) if which == "a piece" else [lens[0] - 1]:
        p, i = c.at(0, pos)
        c.k[1][p, 1, i] = 0x7F if fmt == "nvfp4" else 0xFF
    ref = c.ref()
    assert np.isnan(ref[1]).any() and np.isfinite(ref[1]).any()
    c.check(*c.run(), ref)


@pytest.mark.parametrize("fmt", ["nvfp4", "mxfp4"])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("lens,new,G", [([3, 40], [10, 12], 4), ([30, 300], [60, 200], 3), ([0, 700], [9, 9], 4), ([9, 2700], [60, 50], 3)])
@pytest.mark.parametrize("spoil", ["query", "scale nan", "scale inf"])
def test_rows_that_see_nothing(qf, fmt, D, lens, new, G, spoil):
    """Rows below position zero, among rows that see something: zeros, whatever their queries and the scale are."""
    c = Call(qf, fmt, lens, new, G, D)
    empty = new[0] - lens[0]
    if spoil == "query":
        c.q[:empty] = np.random.default_rng(0).choice([0x7FC0, 0x7F80, 0xFF80, 0x3F80], c.q[:empty].shape)
    scale = {"query": None, "scale nan": float("nan"), "scale inf": float("inf")}[spoil]
    o, l = c.run(scale)
    assert np.all(o[:empty] == 0) and np.all(l[:empty] == -np.inf)
    if spoil == "query":
        c.check(o, l, c.ref())
    else:
        assert np.isnan(o[empty:]).all() and np.isnan(l[empty:]).all()


@pytest.mark.parametrize("fmt", ["nvfp4", "mxfp4"])
@pytest.mark.parametrize("lens,new,G", [([150, 90], None, 4), ([150, 90], [12, 30], 4), ([150, 140], [70, 90], 3)])
def test_tokens_that_are_not_seen(qf, fmt, lens, new, G):
    """Pages that are none, and a window that lies behind max_len: zeros for queries of NaN too."""
    c = Call(qf, fmt, lens, new, G, 64)
    c.table[0] = -5
    own = c.T // 2 if new is None else new[0]                      # rows of the first sequence
    c.q[:own] = 0x7FC0
    o, l = c.run()
    assert np.all(o[:own] == 0) and np.all(l[:own] == -np.inf)
    c.check(o, l, c.ref())
    c = Call(qf, fmt, lens, new, G, 64, window=20, max_len=100)
    ref = c.ref()
    blind = ref[1][:, 0] == -np.inf
    assert blind.any() and not blind.all()
    c.q[blind] = 0x7F80
    o, l = c.run()
    assert np.all(o[blind] == 0) and np.all(l[blind] == -np.inf)
    c.check(o, l, c.ref())
