"""A mixture-of-experts MLP on the library's calls: one quantization-aware training step of every
part (router, sort by expert, the experts' two grouped layers, weighted sum, and all gradients), then
the same layer served from the packed experts that the training step left behind.

    python examples/moe_layer.py [tokens]

The experts are gated: Y = W_d (silu(gate) * up) with [gate; up] = W_gu x.  The router stays in bf16
and unquantized; torch does the router's product and the activation.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2609_39223_amd as qf  # noqa: E402

BLOCK = {"nvfp4": 16, "mxfp4": 32}


def _up(v):
    return (v + 255) // 256 * 256


def _empty(*shape, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device="cuda")


def activate(g):
    """silu(gate) * up of [rows, 2 I] in 32 bits, rounded once."""
    a, b = g.float().chunk(2, dim=1)
    return (torch.nn.functional.silu(a) * b).to(torch.bfloat16)


def activate_bwd(g, dh):
    a, b = g.float().chunk(2, dim=1)
    s, d = torch.sigmoid(a), dh.float()
    return torch.cat([d * b * (s + a * s * (1 - s)), d * a * s], dim=1).to(torch.bfloat16)


class MoELayer:
    """E experts of width I on a hidden size of H, k of them a token; weights Wr [E, H] (router),
    Wgu [E, 2 I, H] and Wd [E, H, I] in bf16, quantized to `fmt` (nvfp4 or mxfp4) on every forward."""

    def __init__(self, Wr, Wgu, Wd, k, fmt="nvfp4", score="softmax"):
        self.Wr, self.Wgu, self.Wd, self.k, self.fmt, self.score = Wr, Wgu, Wd, k, fmt, score
        self.E, self.H, self.I = Wgu.shape[0], Wgu.shape[2], Wd.shape[2]

    # ---------------------------------------------------------------- training
    def plan(self, T):
        """Descriptors, workspaces and saved buffers for T tokens; a training loop keeps them."""
        E, H, I, n = self.E, self.H, self.I, T * self.k
        p = {"gu": qf.grouped_desc(E, n, 2 * I, H, self.fmt), "d": qf.grouped_desc(E, n, H, I, self.fmt),
             "sort": qf.moe_dispatch_workspace(T, E, self.k)}
        for name in ("gu", "d"):
            p[name + "_ws"], p[name + "_saved"] = qf.grouped_workspace(p[name]), qf.grouped_saved_buffer(p[name])
        return p

    def route(self, X, mask=None):
        z = X @ self.Wr.t()
        T = X.shape[0]
        ids, w = _empty(T, self.k, dtype=torch.int32), _empty(T, self.k, dtype=torch.float32)
        qf.moe_route(z, ids, w, score=self.score, mask=mask)
        return z, ids, w

    def sort(self, ids, ws, X=None):
        T, n = ids.shape[0], ids.numel()
        off, row_of = _empty(self.E + 1, dtype=torch.int64), _empty(T, self.k, dtype=torch.int32)
        slot_of = _empty(n, dtype=torch.int32)
        Xg = None if X is None else _empty(n, self.H)
        qf.moe_dispatch(ids, off, row_of, slot_of, ws, X=X, Xg=Xg)
        return off, row_of, slot_of, Xg

    def forward(self, X, p, mask=None):
        n = X.shape[0] * self.k
        z, ids, w = self.route(X, mask)
        off, row_of, _, Xg = self.sort(ids, p["sort"], X)
        G, Yg, Y = _empty(n, 2 * self.I), _empty(n, self.H), _empty(X.shape[0], self.H)
        qf.qlinear_grouped_fwd(p["gu"], off, Xg, self.Wgu, G, p["gu_ws"], saved=p["gu_saved"])
        A = activate(G)
        qf.qlinear_grouped_fwd(p["d"], off, A, self.Wd, Yg, p["d_ws"], saved=p["d_saved"])
        qf.moe_combine(row_of, Yg, Y, w=w)
        return Y, (X, z, ids, w, off, row_of, Xg, G, A, Yg)

    def backward(self, dY, kept, p):
        """dX and the gradients of Wr (bf16 product), Wgu and Wd (FP32)."""
        X, z, ids, w, off, row_of, Xg, G, A, Yg = kept
        n = Xg.shape[0]
        dYg, dw = _empty(n, self.H), torch.empty_like(w)
        qf.moe_combine_bwd(row_of, dY, dYg, Yg=Yg, w=w, dw=dw)
        dA, dWd = _empty(n, self.I), _empty(*self.Wd.shape, dtype=torch.float32)
        qf.qlinear_grouped_bwd_ste(p["d"], off, dYg, A, self.Wd, dA, dWd, p["d_ws"], saved=p["d_saved"])
        dG = activate_bwd(G, dA)
        dXg, dWgu = _empty(n, self.H), _empty(*self.Wgu.shape, dtype=torch.float32)
        qf.qlinear_grouped_bwd_ste(p["gu"], off, dG, Xg, self.Wgu, dXg, dWgu, p["gu_ws"], saved=p["gu_saved"])
        dX, dz = torch.empty_like(X), torch.empty_like(z)
        qf.moe_dispatch_bwd(row_of, dXg, dX)
        qf.moe_route_bwd(z, ids, dw, dz, score=self.score)
        dX = (dX.float() + (dz @ self.Wr).float()).to(torch.bfloat16)
        return dX, dz.t() @ X, dWgu, dWd

    # ----------------------------------------------------------------- serving
    def packed(self, desc, saved):
        """The experts' packed weight as the forward left it in its saved buffer."""
        rows, K = desc.E * desc.N, desc.K
        at = _up(4 * desc.E) if self.fmt == "nvfp4" else 0
        codes = saved[at:at + rows * K // 2]
        at += _up(rows * K // 2)
        scales = saved[at:at + rows * K // BLOCK[self.fmt]]
        S = saved[:4 * desc.E].view(torch.float32) if self.fmt == "nvfp4" else None
        return qf.packed_weight(self.fmt, desc.N, K, codes, scales, S, E=desc.E)

    def serve(self, X, gu, d, ws):
        """A decode step: gate/up reads the tokens' rows through the sort, so none is copied."""
        n = X.shape[0] * self.k
        _, ids, w = self.route(X)
        off, row_of, slot_of, _ = self.sort(ids, ws)
        G, Yg, Y = _empty(n, 2 * self.I), _empty(n, self.H), torch.empty_like(X)
        qf.packed_matvec_grouped(gu, off, X, G, rows=slot_of, rows_div=self.k)
        qf.packed_matvec_grouped(d, off, activate(G), Yg)
        return qf.moe_combine(row_of, Yg, Y, w=w)


def main():
    T = int(sys.argv[1]) if len(sys.argv) > 1 else 4096
    E, H, I, k = 32, 2048, 1024, 4
    g = torch.Generator(device="cuda").manual_seed(0)

    def draw(*shape, std=1.0):
        return (torch.randn(shape, generator=g, device="cuda") * std).to(torch.bfloat16)

    layer = MoELayer(draw(E, H, std=0.02), draw(E, 2 * I, H, std=0.02), draw(E, H, I, std=0.02), k)
    X, dY, p = draw(T, H), draw(T, H), layer.plan(T)
    Y, kept = layer.forward(X, p)
    dX, dWr, dWgu, dWd = layer.backward(dY, kept, p)
    print(f"trained on {T} tokens: |Y| {Y.float().norm():.4g}  |dX| {dX.float().norm():.4g}  |dWr| {dWr.float().norm():.4g}"
          f"  |dWgu| {dWgu.norm():.4g}  |dWd| {dWd.norm():.4g}")
    gu, d = layer.packed(p["gu"], p["gu_saved"]), layer.packed(p["d"], p["d_saved"])
    few = X[:16].contiguous()
    served = layer.serve(few, gu, d, qf.moe_dispatch_workspace(16, E, k))
    off = (served.float() - Y[:16].float()).norm() / Y[:16].float().norm()
    print(f"served 16 of them from the packed experts: relative difference {off:.2e}")


if __name__ == "__main__":
    main()
