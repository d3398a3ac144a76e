"""The packed products, adapters, 4-bit cache and attention over it together, as examples/decode_step.py runs
them: prompts in one ragged call, then single tokens, eager and captured.

The codes in the cache jump where a rounding falls the other way, so each part is compared with FP64 on the
layer's own input to it.  A projection rounds its weights (the GEMM's to bf16), its output and the sum with
the adapter's product, 2^-8 relative each: 3 * 2^-8 < 2^-6 in norm (nothing cancels between random terms).
The written codes are the oracle's bit for bit.  Attention rounds its output once, 2^-8, and probabilities by
2^-11: together below 2^-7 in norm."""
import importlib.util
import os

import numpy as np
import pytest

import oracle
from oracle import serving as sv
from tests.helpers import bf16_to_f64, from_dev, to_dev

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("decode_step", os.path.join(ROOT, "examples", "decode_step.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _f64(t):
    return t.double().cpu().numpy()


def _bits(t):
    return from_dev(t.contiguous().view(torch.int16))


def _off(got, ref):
    return float(np.linalg.norm(got - ref) / np.linalg.norm(ref))


class Setup:
    def __init__(self, example, fmt, kv_fmt, hidden=256, Hq=6, H=2, D=64, page=16, B=3, cols=12, n=4, r=8):
        self.qf, self.kv_fmt, self.shape = example.qf, kv_fmt, (Hq, H, D, page)
        g = torch.Generator(device="cuda").manual_seed(hidden + D)
        self.draw = lambda *s, std=1.0: (torch.randn(s, generator=g, device="cuda") * std).to(torch.bfloat16)
        W = self.draw((Hq + 2 * H) * D, hidden, std=0.06), self.draw(hidden, Hq * D, std=0.06)
        self.A = [(self.draw(n, r, w.shape[1], std=0.06), self.draw(n, w.shape[0], r, std=0.1)) for w in W]
        self.scale = torch.tensor([0.5, -0.25, 1.0, 2.0], device="cuda")
        self.hat = [bf16_to_f64(oracle.fakequant(_bits(w), fmt)) for w in W]
        self.adapters = [self.qf.adapters(a, b, self.scale) for a, b in self.A]
        self.amax = np.full(H, 6.0, np.float32) if kv_fmt == "nvfp4" else None
        S = None if kv_fmt == "mxfp4" else to_dev(self.amax / np.float32(2688))
        self.layers = [example.Attention(*W, Hq, H, D, B * cols, page, fmt, kv_fmt, S, S) for _ in range(2)]
        for layer in self.layers:
            for t in layer.cache._tensors[:4]:
                t.fill_(0xFF)                                       # (what nobody has written: NaN scales)
        self.table = torch.randperm(B * cols, generator=g, device="cuda").to(torch.int32).view(B, cols)

    def check(self, layer, X, ids, Y, qkv, O, offsets, lens):
        """One step's parts against FP64 on their own inputs; the cache holds it already."""
        Hq, H, D, page = self.shape
        for i, (x, y) in enumerate(((X, qkv), (O, Y))):
            a, b = (_f64(t) for t in self.A[i])
            want, _ = sv.lora_rows(ids.cpu().numpy(), _f64(x), a, b, _f64(self.scale), _f64(x) @ self.hat[i].T)
            assert _off(_f64(y), want) < 2.0 ** -6, i
        table, cache, n, m = self.table.cpu().numpy(), [from_dev(t) for t in layer.cache._tensors[:4]], Hq * D, H * D
        where = sv.places(offsets, lens, table, page, cache[0].shape[0], X.shape[0])
        vals = []
        for i, x in enumerate((qkv[:, n:n + m], qkv[:, n + m:])):
            codes, scales, S, _ = sv.quantize_heads(_bits(x), H, self.kv_fmt, self.amax)
            for t, w in enumerate(where):
                assert np.array_equal(cache[2 * i][w[0], :, w[1]], codes[t]) and np.array_equal(cache[2 * i + 1][w[0], :, w[1]], scales[t])
            with np.errstate(all="ignore"):
                vals.append(sv.values(cache[2 * i], cache[2 * i + 1], S, self.kv_fmt))
        want = sv.attention(_f64(qkv[:, :n]).reshape(-1, Hq, D), *vals, offsets, lens, table, D ** -0.5)[0]
        assert _off(_f64(O), want.reshape(-1, n)) < 2.0 ** -7


@pytest.mark.parametrize("fmt,kv_fmt", [("nvfp4", "nvfp4"), ("mxfp4", "mxfp4"), ("mxfp4", "nvfp4")])
@pytest.mark.parametrize("lengths", [[20, 1, 33], [90, 64, 130]])
def test_prompts_then_tokens(example, fmt, kv_fmt, lengths):
    s = Setup(example, fmt, kv_fmt)
    qf, layer = s.qf, s.layers[0]
    lens = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    ids = torch.tensor([2, -1, 0], dtype=torch.int32, device="cuda")
    offsets = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int64)
    seqs, T = qf.kv_sequences(lens, s.table, to_dev(offsets)), sum(lengths)
    X, each = s.draw(T, 256), torch.repeat_interleave(ids, lens.long())
    out = layer.step(X, each, seqs, s.adapters, layer.plan(T, seqs, s.adapters))
    s.check(layer, X, each, *out, offsets, lengths)
    seqs = qf.kv_sequences(lens, s.table)
    ws = layer.plan(3, seqs, s.adapters)
    for i in range(1, 4):                                           # a token each; the second request's page ends
        lens.add_(1)
        X = s.draw(3, 256)
        out = layer.step(X, ids, seqs, s.adapters, ws)
        s.check(layer, X, ids, *out, None, [v + i for v in lengths])


def test_two_graphs_with_shared_workspaces(example):
    """Two captured steps of different sizes that share their workspaces, replayed in turn while lengths, adapters
    and inputs change, against eager steps on a second cache; eager work of the same calls lies between."""
    s = Setup(example, "nvfp4", "nvfp4", cols=80)
    qf = s.qf
    lens = torch.ones(3, dtype=torch.int32, device="cuda")
    ids = torch.zeros(3, dtype=torch.int32, device="cuda")
    X = s.draw(3, 256)
    draft_off = torch.tensor([0, 2, 3, 6], dtype=torch.int64, device="cuda")
    Xd, idd = s.draw(6, 256), torch.zeros(6, dtype=torch.int32, device="cuda")
    calls = [(X, ids, qf.kv_sequences(lens, s.table)), (Xd, idd, qf.kv_sequences(lens, s.table, draft_off))]
    plans = [s.layers[0].plan(x.shape[0], q, s.adapters) for x, _, q in calls]
    shared = [max(a, b, key=lambda t: t.numel()) for a, b in zip(*plans)]
    own = [s.layers[1].plan(x.shape[0], q, s.adapters) for x, _, q in calls]
    for x, i, q in calls:                                           # (loads what is loaded lazily)
        s.layers[0].step(x, i, q, s.adapters, shared)
        s.layers[1].step(x, i, q, s.adapters, own[0] if x is X else own[1])
    torch.cuda.synchronize()
    graphs, outs = [], []
    for x, i, q in calls:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append(s.layers[0].step(x, i, q, s.adapters, shared))
    for n in (9, 17, 1250, 40, 700):
        lens.copy_(torch.tensor([n, max(3, n // 2), n + 5], dtype=torch.int32))
        for t in (X, Xd):
            t.normal_()
        ids.random_(-1, 5)
        idd.random_(-1, 5)
        want = []
        for which in (0, 1, 0):
            graphs[which].replay()
            x, i, q = calls[which]
            want = s.layers[1].step(x, i, q, s.adapters, own[which])
            torch.cuda.synchronize()
            for a, b in zip(outs[which], want):
                assert torch.equal(a.view(torch.int16), b.view(torch.int16))
    for a, b in zip(s.layers[0].cache._tensors[:4], s.layers[1].cache._tensors[:4]):
        assert torch.equal(a, b)


def test_example_runs(example, capsys, monkeypatch):
    monkeypatch.setattr(example.sys, "argv", ["decode_step.py", "3"])
    example.main()
    assert "3 steps" in capsys.readouterr().out
