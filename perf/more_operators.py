"""Performance cases of the operators that a decode step has around its packed products: the 4-bit
cache of keys and values, the attention that reads it, and the low-rank adapters of many requests.

Kinds of case (a case is a dict of plain values with a "kind"):

  store     quantizing the new tokens' keys and values into their sequences' pages, and reading the
            same tokens back (their values as the cache holds them).
  read      reading whole sequences back out of the cache.
  attend    attention of the new tokens' queries over the cache (causal, grouped heads, paged): the
            output and its log-sum-exp.
  adapters  rows of many requests, each with its own adapter: base + scale (x A^T) B^T.

Where `own` is false the operators run in their plain form, elementary torch operations in 32 bits.
Inputs follow the layers they stand for: values and queries N(0, 1), keys with some large channels,
projections' outputs N(0, 1), factors N(0, 1 / sqrt K) and N(0, 0.02).
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda"
BLOCK = {"nvfp4": 16, "mxfp4": 32}


def _kv(name, kind, fmt, B, new, L, H, G, D, page, ragged, window=0):
    """B sequences of at most L tokens in the cache, at most `new` of them new; H heads of keys and
    values, G queries' heads to each."""
    c = dict(kind=kind, fmt=fmt, B=B, new=new, L=L, H=H, G=G, D=D, page=page, ragged=ragged, window=window)
    return dict(c, name=name) if name else c


def _lora(name, M, n, r, K, N, runs, none):
    """M rows that n adapters of rank r share; runs: an adapter's rows lie together (prompts), else
    they are mixed (a decode step); one row in `none` has no adapter (0: every row has one)."""
    c = dict(kind="adapters", M=M, n=n, r=r, K=K, N=N, runs=runs, none=none)
    return dict(c, name=name) if name else c


def listed():
    return [
        # The new token of 64 sequences of a decode step: latency counts.
        _kv("store_decode_64", "store", "mxfp4", 64, 1, 4096, 8, 4, 128, 16, True),
        # Prompts of three requests going into the cache.
        _kv("store_prompts_16k", "store", "nvfp4", 3, 8192, 8192, 8, 4, 128, 64, True),
        # Sequences of odd lengths read back, wide heads.
        _kv("read_ragged_d256", "read", "nvfp4", 5, 0, 3001, 4, 4, 256, 32, True),
        # A long prompt's cache read back, as a copy into another layer's layout does.
        _kv("read_32k", "read", "mxfp4", 1, 0, 32768, 8, 4, 128, 64, False),
        # A handful of short conversations: latency counts.
        _kv("attend_decode_short", "attend", "mxfp4", 4, 1, 517, 8, 4, 128, 16, True),
        # One long document, one token at a time: little but the cache to read.
        _kv("attend_decode_128k", "attend", "nvfp4", 1, 1, 131072, 8, 4, 128, 64, False),
        # A full batch at 8K tokens each, the attention of the 9B-class layer.
        _kv("attend_decode_64x8k", "attend", "nvfp4", 64, 1, 8192, 8, 4, 128, 64, False),
        # Drafted tokens checked five at a time under a sliding window, lengths as they come.
        _kv("attend_draft_16x5", "attend", "mxfp4", 16, 5, 4099, 4, 8, 64, 32, True, 2048),
        # A piece of a prompt against what was cached before it.
        _kv("attend_chunk_2k", "attend", "nvfp4", 1, 2048, 10240, 8, 4, 128, 64, False),
        # The QKV projection of 16 sequences, an adapter each.
        _lora("adapters_decode_16", 16, 16, 16, 4096, 6144, False, 0),
        # A mixed batch on fewer adapters of a higher rank, some requests without.
        _lora("adapters_mixed_61", 61, 24, 64, 4096, 4096, False, 7),
        # Prompts of six requests through the gate/up projection's adapters.
        _lora("adapters_prompts_4k", 4099, 6, 32, 4096, 24576, True, 0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = {c["kind"]: [max(work(x)[u] for x in listed() if x["kind"] == c["kind"]) for u in ("bytes", "flops")]
            for c in listed()}
    while True:
        kind = rng.choice(["store", "read", "attend", "attend", "attend", "adapters", "adapters"])
        if kind == "adapters":
            M = _log(rng, 1, 4096)
            c = _lora(None, M, min(M, _log(rng, 1, 64)), rng.choice([8, 16, 24, 32, 64, 128]),
                      _log(rng, 256, 14336) // 8 * 8, _log(rng, 256, 24576) // 8 * 8, rng.random() < 0.4,
                      rng.choice([0, 0, 5]))
            if c["n"] * c["r"] > 1536:                     # (the plain form multiplies all of them)
                continue
        else:
            L = _log(rng, 1, 131072)
            c = _kv(None, kind, rng.choice(["nvfp4", "mxfp4"]), _log(rng, 1, 96), 0, L, rng.choice([1, 2, 4, 8]),
                    rng.choice([1, 2, 4, 5, 8, 16]), rng.choice([64, 128, 128, 256]), rng.choice([16, 32, 64, 128]),
                    rng.random() < 0.7, rng.choice([0, 0, 0, 1024]) if kind == "attend" else 0)
            if kind != "read":
                c["new"] = min(L, rng.choice([1, 1, _log(rng, 2, 8), _log(rng, 9, 2048)]))
            if kind == "store" and rng.random() < 0.5:
                c["new"] = L
            if c["B"] * L > 64 * 8192 or c["B"] * c["new"] > 16384:
                continue
            if kind == "attend" and c["B"] * c["new"] * c["G"] * c["H"] * L > 2048 * 32 * 10240:
                continue
        w = work(c)
        if all(w[u] <= m for u, m in zip(("bytes", "flops"), most[kind])):
            return c


# ---------------------------------------------------------------------------------- inputs
def _lengths(case):
    """The sequences' lengths and numbers of new tokens; the first has the most of both."""
    B, L, new = case["B"], case["L"], case["new"]
    if not case["ragged"]:
        return [L] * B, [new] * B
    rng = random.Random(B * 1000003 + L * 101 + new)
    lens = [L] + [rng.randint(max(1, L // 4), L) for _ in range(B - 1)]
    return lens, [min(n, rng.randint((new + 1) // 2, new) if i else new) for i, n in enumerate(lens)]


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) % (1 << 62))
    return g


def _randn(g, *shape, std=1.0):
    return torch.randn(shape, generator=g, device=DEV) * std


def _like_keys(g, x):
    """x [..., D] with one channel in sixteen five times as large."""
    big = torch.randperm(x.shape[-1], generator=g, device=DEV)[:x.shape[-1] // 16]
    x[..., big] *= 5.0
    return x


def _encode(x, S, fmt):
    """codes (two a byte) and scale bytes of fp32 x [..., H, D], S [H]: the formats' steps in 32 bits."""
    b = x.unflatten(-1, (-1, BLOCK[fmt]))
    a = b.abs().amax(-1)
    if fmt == "nvfp4":
        S = S[:, None]
        s = (a / (6.0 * S)).clamp(max=448.0).to(torch.float8_e4m3fn)
        d = S * s.float()
        y = b.abs() * torch.where(d == 0, torch.zeros_like(d), 1.0 / d)[..., None]
        s = s.view(torch.uint8)
    else:
        p = torch.where(a == 0, -127, (torch.frexp(a).exponent - 3).clamp(-127, 127))
        y = torch.ldexp(b.abs(), -p[..., None])
        s = (p + 127).to(torch.uint8)
    # nearest of 0, .5, 1, 1.5, 2, 3, 4, 6; halfway to the even code
    c = sum((y > e).to(torch.uint8) for e in (0.25, 1.25, 2.5, 5.0)) + sum((y >= e).to(torch.uint8) for e in (0.75, 1.75, 3.5))
    c = (c | (torch.signbit(b).to(torch.uint8) << 3)).flatten(-2)
    return c[..., 0::2] | (c[..., 1::2] << 4), s


def _sequences(case, g):
    """lens, offsets of the new tokens (None: one each) and the table of pages, which lie anywhere."""
    lens, new = _lengths(case)
    page, B = case["page"], case["B"]
    width = max(-(-n // page) for n in lens)
    pages = B * width + 3
    table = torch.randperm(pages, generator=g, device=DEV)[:B * width].view(B, width).to(torch.int32)
    counts = lens if case["kind"] == "read" else new
    offsets = None
    if any(n != 1 for n in counts):
        offsets = torch.tensor([0] + counts, device=DEV).cumsum(0)
    return pages, {"lens": torch.tensor(lens, dtype=torch.int32, device=DEV), "offsets": offsets, "table": table.contiguous(),
                   "T": sum(counts)}


def _inputs(case, seed):
    g = _gen(seed)
    if case["kind"] == "adapters":
        M, n, r, K, N = (case[x] for x in ("M", "n", "r", "K", "N"))
        order = torch.randperm(n, generator=g, device=DEV)
        row = torch.arange(M, device=DEV)
        ids = order[row * n // M] if case["runs"] else order[row % n][torch.randperm(M, generator=g, device=DEV)]
        if case["none"]:
            ids = torch.where(row % case["none"] == case["none"] - 1, -1, ids)
        bf = torch.bfloat16
        return {"ids": ids.to(torch.int32), "X": _randn(g, M, K).to(bf), "base": _randn(g, M, N).to(bf),
                "A": _randn(g, n, r, K, std=K ** -0.5).to(bf), "B": _randn(g, n, N, r, std=0.02).to(bf),
                "scale": torch.full((n,), 2.0, device=DEV) * torch.rand(n, generator=g, device=DEV).add_(0.5)}
    H, D, page, fmt = case["H"], case["D"], case["page"], case["fmt"]
    pages, s = _sequences(case, g)
    shape = (pages, H, page, D)
    for x in "kv":
        # the tensor scale of a head as calibration leaves it: about the largest value seen / 2688
        S = (25.0 if x == "k" else 5.0) / 2688 * (0.8 + 0.4 * torch.rand(H, generator=g, device=DEV))
        s[x + "_S"] = S if fmt == "nvfp4" else None
        if case["kind"] == "store":
            s[x + "_codes"] = torch.zeros(*shape[:3], D // 2, dtype=torch.uint8, device=DEV)
            s[x + "_scales"] = torch.zeros(*shape[:3], D // BLOCK[fmt], dtype=torch.uint8, device=DEV)
            new = _randn(g, s["T"], H, D)
            s[x.upper()] = (_like_keys(g, new) if x == "k" else new).to(torch.bfloat16).flatten(1)
        else:
            data = _randn(g, pages, page, H, D)
            data = _like_keys(g, data) if x == "k" else data
            c, b = _encode(data, S, fmt)
            s[x + "_codes"], s[x + "_scales"] = c.transpose(1, 2).contiguous(), b.transpose(1, 2).contiguous()
    if case["kind"] == "attend":
        s["Q"] = _randn(g, s["T"], H * case["G"] * D).to(torch.bfloat16)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if case["kind"] == "adapters":
        s["Y"] = torch.empty_like(s["base"])
        if own:
            import paper_2609_39223_amd as qf
            s["adapters"] = qf.adapters(s["A"], s["B"], s["scale"])
            s["ws"] = qf.lora_rows_workspace(s["adapters"], case["M"])
        return s
    T, width = s["T"], case["H"] * case["D"]
    if case["kind"] == "attend":
        s["O"] = torch.empty_like(s["Q"])
        s["lse"] = torch.empty(T, case["H"] * case["G"], device=DEV)
    else:
        s["K_out"], s["V_out"] = (torch.empty(T, width, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    if own:
        import paper_2609_39223_amd as qf
        s["cache"] = qf.kv_cache(case["fmt"], s["k_codes"], s["k_scales"], s["v_codes"], s["v_scales"], s["k_S"], s["v_S"])
        s["seqs"] = qf.kv_sequences(s["lens"], s["table"], offsets=s["offsets"], max_len=case["L"])
        if case["kind"] == "attend":
            s["ws"] = qf.kv_attention_workspace(s["cache"], s["seqs"], T, case["H"] * case["G"], window=case["window"])
    return s


# ------------------------------------------------------------------------ the plain forms
def _token_places(s):
    """Sequence and position of each of the T tokens: the last ones of their sequences."""
    t = torch.arange(s["T"], device=DEV)
    if s["offsets"] is None:
        return t, s["lens"].long() - 1
    b = torch.searchsorted(s["offsets"], t, right=True) - 1
    return b, s["lens"].long()[b] - s["offsets"][b + 1] + t


def _decoded(codes, scales, S, fmt):
    """Values [..., D] of codes [..., D/2], the scales' steps included, S [..., 1] or None."""
    v = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
    m = (v & 7).float()
    m = torch.where(m < 4, 0.5 * m, torch.where(m < 6, m - 2.0, 2.0 * m - 8.0))
    m = torch.where(v > 7, -m, m)
    if fmt == "nvfp4":
        d = scales.view(torch.float8_e4m3fn).float() * S
    else:
        d = torch.ldexp(torch.ones_like(scales, dtype=torch.float32), scales.int() - 127)
    return (m.unflatten(-1, (-1, BLOCK[fmt])) * d[..., None]).flatten(-2)


def _plain_read(s, x, b, pos):
    """Keys or values of sequence b at position pos (of one shape), [..., H, D]."""
    page = s["case"]["page"]
    pg = s["table"][b, pos // page].long()
    S = s[x + "_S"]
    return _decoded(s[x + "_codes"][pg, :, pos % page], s[x + "_scales"][pg, :, pos % page],
                    None if S is None else S[:, None], s["case"]["fmt"])


def _plain_store(s):
    case = s["case"]
    b, pos = _token_places(s)
    pg = s["table"][b, pos // case["page"]].long()
    for x in "kv":
        c, d = _encode(s[x.upper()].float().unflatten(1, (case["H"], case["D"])), s[x + "_S"], case["fmt"])
        s[x + "_codes"][pg, :, pos % case["page"]] = c
        s[x + "_scales"][pg, :, pos % case["page"]] = d


def _plain_attend(s):
    case = s["case"]
    B, H, G, D, new = (case[x] for x in ("B", "H", "G", "D", "new"))
    lens = s["lens"].long()
    off = torch.arange(B + 1, device=DEV) if s["offsets"] is None else s["offsets"]
    n = off[1:] - off[:-1]
    i = torch.arange(new, device=DEV)
    tok = (off[:-1, None] + i).clamp(max=s["T"] - 1)
    q = s["Q"].float().view(s["T"], H, G, D)[tok]                     # [B, new, H, G, D]
    q = q.permute(0, 2, 1, 3, 4).reshape(B, H, new * G, D)
    pos = torch.arange(case["L"], device=DEV)
    at = torch.minimum(pos, lens[:, None] - 1)                        # (past the end: masked below)
    seq = torch.arange(B, device=DEV)[:, None].expand_as(at)
    k = _plain_read(s, "k", seq, at).permute(0, 2, 3, 1)              # [B, H, D, L]
    z = (q @ k) * D ** -0.5
    last = (lens - n)[:, None] + i                                    # [B, new]
    see = pos <= last[..., None]
    if case["window"]:
        see = see & (pos > last[..., None] - case["window"])
    see = see[:, None, :, None, :].expand(B, 1, new, G, case["L"]).reshape(B, 1, new * G, case["L"])
    z = z.masked_fill(~see, -math.inf)
    top = z.amax(-1, keepdim=True)
    top = torch.where(top > -math.inf, top, torch.zeros_like(top))
    z = torch.exp(z - top)
    total = z.sum(-1, keepdim=True)
    o = (z @ _plain_read(s, "v", seq, at).transpose(1, 2)) / torch.where(total > 0, total, torch.ones_like(total))
    lse = (top + torch.log(total)).view(B, H, new, G).transpose(1, 2).reshape(B, new, H * G)
    o = o.view(B, H, new, G, D).permute(0, 2, 1, 3, 4).reshape(B, new, H * G * D)
    t = torch.arange(s["T"], device=DEV)
    b = torch.searchsorted(off, t, right=True) - 1
    return {"O": o[b, t - off[b]].to(torch.bfloat16), "lse": lse[b, t - off[b]]}


def _plain_adapters(s):
    case = s["case"]
    n, r = case["n"], case["r"]
    z = s["X"].float() @ s["A"].float().view(n * r, -1).t()
    mine = s["ids"][:, None] == torch.arange(n, device=DEV)
    z = (z.view(-1, n, r) * (mine * s["scale"])[..., None]).view(-1, n * r)
    y = z @ s["B"].float().transpose(1, 2).reshape(n * r, -1)
    return {"Y": (s["base"].float() + y).to(torch.bfloat16)}


def _run_plain(s):
    kind = s["case"]["kind"]
    if kind == "adapters":
        return _plain_adapters(s)
    if kind == "attend":
        return _plain_attend(s)
    if kind == "store":
        _plain_store(s)
    b, pos = _token_places(s)
    return {x.upper(): _plain_read(s, x, b, pos).to(torch.bfloat16).flatten(1) for x in "kv"}


def _run_own(s):
    import paper_2609_39223_amd as qf
    case = s["case"]
    kind = case["kind"]
    if kind == "adapters":
        return {"Y": qf.lora_rows(s["adapters"], s["ids"], s["X"], s["Y"], s["ws"], base=s["base"])}
    if kind == "attend":
        qf.kv_attention(s["cache"], s["seqs"], s["Q"], s["O"], s["ws"], window=case["window"], lse=s["lse"])
        return {"O": s["O"], "lse": s["lse"]}
    if kind == "store":
        qf.kv_write(s["cache"], s["seqs"], s["K"], s["V"])
    qf.kv_read(s["cache"], s["seqs"], s["K_out"], s["V_out"])
    return {"K": s["K_out"], "V": s["V_out"]}


def run(s):
    return _run_own(s) if own else _run_plain(s)


def work(case):
    if case["kind"] == "adapters":
        M, n, r, K, N = (case[x] for x in ("M", "n", "r", "K", "N"))
        return {"bytes": 2 * n * r * (K + N) + 2 * M * (K + 2 * N), "flops": 2.0 * M * r * (K + N)}
    H, G, D = case["H"], case["G"], case["D"]
    token = int(H * D * (1 + 2 / BLOCK[case["fmt"]]))                 # keys and values, codes and scales
    lens, new = _lengths(case)
    if case["kind"] == "store":
        return {"bytes": sum(new) * 2 * (token + 4 * H * D), "flops": 8.0 * sum(new) * H * D}
    if case["kind"] == "read":
        return {"bytes": sum(lens) * (token + 4 * H * D), "flops": 4.0 * sum(lens) * H * D}
    W = case["window"] or max(lens)
    pairs = sum(min(p + 1, W) for n, m in zip(lens, new) for p in range(n - m, n))
    seen = sum(min(n, m + W - 1) for n, m in zip(lens, new))
    rows = sum(new) * H * G
    return {"bytes": seen * token + rows * (4 * D + 4), "flops": 4.0 * D * H * G * pairs}


# ---------------------------------------------------------- the same results in 64 bits
def _e2m1_nearest(y):
    """|y| to the nearest of the eight magnitudes by distance, halfway to the one of even index."""
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=DEV)
    best, value = torch.full_like(y, math.inf), torch.zeros_like(y)
    for i in (0, 2, 4, 6, 1, 3, 5, 7):
        d = (y.abs() - grid[i]).abs()
        value = torch.where(d < best, grid[i], value)
        best = torch.minimum(best, d)
    return torch.where(y < 0, -value, value)


def _exact_held(x, S, fmt):
    """The values that stand for x [T, H, D] (64 bits), from the formats' definitions: the scale
    steps are defined in 32 bits, so each is rounded there."""
    f32 = lambda t: t.float().double()  # noqa: E731
    b = x.view(*x.shape[:2], -1, BLOCK[fmt])
    a = b.abs().amax(-1)
    if fmt == "mxfp4":
        d = torch.exp2((torch.floor(torch.log2(a.clamp(min=2.0 ** -120))) - 2).clamp(-127, 127))
        return (_e2m1_nearest(b / d[..., None]) * d[..., None]).view_as(x)
    S = S.double()[None, :, None]
    t = f32(a / f32(6 * S)).clamp(max=448.0)
    step = torch.exp2(torch.floor(torch.log2(t.clamp(min=2.0 ** -6))) - 3)
    d = f32(S * (torch.round(t / step) * step))
    inv = torch.where(d > 0, f32(1 / d.clamp(min=1e-300)), 0.0)
    return (_e2m1_nearest(f32(b * inv[..., None])) * d[..., None]).view_as(x)


def _exact_values(s, x, b, pos):
    """[n, H, D] of sequence b's positions, element by element from the codes."""
    case = s["case"]
    pg = s["table"][b].long()[pos // case["page"]]
    code, scale = (s[x + n][pg, :, pos % case["page"]].long() for n in ("_codes", "_scales"))
    code = torch.stack([code % 16, code // 16], -1).flatten(-2)
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=DEV)
    v = torch.where(code >= 8, -1.0, 1.0) * grid[code % 8]
    if case["fmt"] == "mxfp4":
        d = torch.exp2(scale.double() - 127)
    else:
        e, f = scale // 8, (scale % 8).double()
        d = torch.where(e == 0, f / 512, torch.exp2(e.double() - 7) * (1 + f / 8)) * s[x + "_S"].double()[:, None]
    return v * d.repeat_interleave(BLOCK[case["fmt"]], -1)


def _exact_attend(s):
    case = s["case"]
    H, G, D = case["H"], case["G"], case["D"]
    lens, new = _lengths(case)
    outs, sums = [], []
    at = 0
    for b, (n, m) in enumerate(zip(lens, new)):
        pos = torch.arange(n, device=DEV)
        K, V = _exact_values(s, "k", b, pos), _exact_values(s, "v", b, pos)
        Q = s["Q"][at:at + m].double().view(m, H, G, D)
        at += m
        o = torch.empty(m, H, G, D, dtype=torch.float64, device=DEV)
        l = torch.empty(m, H, G, dtype=torch.float64, device=DEV)
        i = torch.arange(n - m, n, device=DEV)[:, None]
        hidden = (pos > i) | (pos <= i - (case["window"] or n + 1))
        for h in range(H):
            z = torch.einsum("mgd,nd->gmn", Q[:, h], K[:, h]) / math.sqrt(D)
            z = z.masked_fill(hidden, -math.inf)
            e = torch.logsumexp(z, -1, keepdim=True)
            o[:, h] = (torch.exp(z - e) @ V[:, h]).transpose(0, 1)
            l[:, h] = e[..., 0].t()
        outs.append(o.reshape(m, -1))
        sums.append(l.reshape(m, -1))
    return {"O": torch.cat(outs), "lse": torch.cat(sums)}


def exact(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if case["kind"] == "adapters":
        Y = s["base"].double()
        for a in range(case["n"]):
            rows = torch.nonzero(s["ids"] == a).reshape(-1)
            z = s["X"][rows].double() @ s["A"][a].double().t()
            Y[rows] += s["scale"][a].double() * (z @ s["B"][a].double().t())
        return {"Y": Y}
    if case["kind"] == "attend":
        return _exact_attend(s)
    if case["kind"] == "store":
        return {x.upper(): _exact_held(s[x.upper()].double().view(s["T"], case["H"], case["D"]), s[x + "_S"],
                                       case["fmt"]).flatten(1) for x in "kv"}
    lens, _ = _lengths(case)
    return {x.upper(): torch.cat([_exact_values(s, x, b, torch.arange(n, device=DEV)) for b, n in enumerate(lens)]).flatten(1)
            for x in "kv"}
