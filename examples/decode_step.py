"""The attention half of a transformer layer served on the library's calls: projections with packed weights and
every request's own low-rank adapter, new keys and values into the 4-bit paged cache, attention over it, and the
output projection.  Prompts of several requests go through in one ragged call; after them one captured graph
is replayed for every token.

    python examples/decode_step.py [steps]

Position encoding, norms and the MLP are left out (examples/moe_layer.py has an MLP); torch does the residual.
"""
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2609_39223_amd as qf  # noqa: E402

BLOCK = {"nvfp4": 16, "mxfp4": 32}


def _empty(*shape, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device="cuda")


def pack(W, fmt):
    """A weight's descriptor, codes, block scales and tensor scale."""
    N, K = W.shape
    codes, scales, S = _empty(N, K // 2, dtype=torch.uint8), _empty(N, K // BLOCK[fmt], dtype=torch.uint8), None
    if fmt == "nvfp4":
        S, amax = _empty(1, dtype=torch.float32), torch.zeros(1, device="cuda")
        qf.fakequant_nvfp4(W, amax, s_out=S, codes=codes, scales=scales)
    else:
        qf.fakequant_mxfp4(W, codes=codes, scales=scales)
    return qf.packed_weight(fmt, N, K, codes, scales, S), codes, scales, S


class Attention:
    """Hq heads of queries over H of keys and values, D wide; Wqkv [(Hq + 2 H) D, hidden] and Wo [hidden, Hq D] in
    bf16, packed to `fmt`; the cache in `kv_fmt`, its heads' tensor scales (nvfp4) given as k_S, v_S."""

    def __init__(self, Wqkv, Wo, Hq, H, D, pages, page, fmt="nvfp4", kv_fmt="nvfp4", k_S=None, v_S=None):
        self.Hq, self.H, self.D, self.fmt = Hq, H, D, fmt
        self.weights = pack(Wqkv, fmt), pack(Wo, fmt)
        parts = [_empty(pages, H, page, D // d, dtype=torch.uint8) for d in (2, BLOCK[kv_fmt], 2, BLOCK[kv_fmt])]
        self.cache = qf.kv_cache(kv_fmt, *parts, k_S, v_S)

    def plan(self, T, seqs, adapters):
        """Workspaces for T rows of these sequences; a server keeps them."""
        return (qf.kv_attention_workspace(self.cache, seqs, T, self.Hq), *[qf.lora_rows_workspace(a, T) for a in adapters])

    def project(self, weight, X, a, ids, ws):
        """X W^T of the packed weight and on top of it each row's adapter."""
        w, *parts = weight
        M, Y = X.shape[0], _empty(X.shape[0], w.N)
        if M <= 64:
            qf.packed_matvec(w, X, Y)
        else:
            qf.gemm_packed_b(M, w.N, w.K, X, X.stride(0), self.fmt, *parts, Y, Y.stride(0))
        return qf.lora_rows(a, ids, X, Y, ws, base=Y)

    def step(self, X, ids, seqs, adapters, ws):
        """The new tokens' rows X [T, hidden], request adapters ids [T]: a prompt's, or one a sequence.  Returns
        the output rows and what they were made from."""
        n, m = self.Hq * self.D, self.H * self.D
        qkv = self.project(self.weights[0], X, adapters[0], ids, ws[1])
        qf.kv_write(self.cache, seqs, qkv[:, n:n + m], qkv[:, n + m:])
        O = qf.kv_attention(self.cache, seqs, qkv[:, :n], _empty(X.shape[0], n), ws[0])
        return self.project(self.weights[1], O, adapters[1], ids, ws[2]), qkv, O


def main():
    steps = int(sys.argv[1]) if len(sys.argv) > 1 else 64
    hidden, Hq, H, D, page, B, n, r = 2048, 16, 4, 128, 32, 16, 3, 16
    g = torch.Generator(device="cuda").manual_seed(0)

    def draw(*shape, std=1.0):
        return (torch.randn(shape, generator=g, device="cuda") * std).to(torch.bfloat16)

    Wqkv, Wo = draw((Hq + 2 * H) * D, hidden, std=0.02), draw(hidden, Hq * D, std=0.02)
    adapters = [qf.adapters(draw(n, r, K, std=0.02), draw(n, N, r, std=0.02), torch.full((n,), 0.5, device="cuda"))
                for N, K in (Wqkv.shape, Wo.shape)]
    # tensor scales of the cache's heads from a calibration batch
    kv = (draw(256, hidden).float() @ Wqkv[Hq * D:].float().t()).view(256, 2, H, D).abs().amax((0, 3)) / 2688
    lengths = [57 * (i + 1) for i in range(B)]
    cols = (max(lengths) + steps) // page + 1
    layer = Attention(Wqkv, Wo, Hq, H, D, B * cols, page, k_S=kv[0].contiguous(), v_S=kv[1].contiguous())
    table = torch.randperm(B * cols, device="cuda").to(torch.int32).view(B, cols)
    lens = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    ids = torch.arange(B, dtype=torch.int32, device="cuda") % (n + 1)          # (every fourth request has none)

    # the prompts, rows of all requests back to back
    T = sum(lengths)
    offsets = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), lens.long().cumsum(0)])
    prompts = qf.kv_sequences(lens, table, offsets, max_len=max(lengths))
    X = draw(T, hidden)
    Y, _, _ = layer.step(X, torch.repeat_interleave(ids, lens), prompts, adapters, layer.plan(T, prompts, adapters))
    print(f"{B} prompts, {T} tokens: |Y| {Y.float().norm():.4g}")

    # a token a request and step, captured once
    seqs = qf.kv_sequences(lens, table, max_len=max(lengths) + steps)
    ws = layer.plan(B, seqs, adapters)
    x = Y[offsets[1:] - 1].contiguous()

    def one():
        lens.add_(1)
        y, _, _ = layer.step(x, ids, seqs, adapters, ws)
        z = x.float() + y.float()
        x.copy_(z * torch.rsqrt((z * z).mean(1, keepdim=True)))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        one()                                                       # (counts as a step)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one()
    torch.cuda.synchronize()
    t = time.perf_counter()
    for _ in range(steps - 1):
        graph.replay()
    torch.cuda.synchronize()
    us = (time.perf_counter() - t) / max(steps - 1, 1) * 1e6
    print(f"{steps} steps to {int(lens.max())} tokens: |x| {x.float().norm():.4g}, {us:.0f} us each")


if __name__ == "__main__":
    main()
