"""The calls of a decoder's serving step that this library is timed on: new
tokens' K and V into a paged cache, attention of one new token over that cache,
and the matrix product with bias, activation and residual, each beside its plain
form in elementary torch operations and its arithmetic in 64 bits.

Inputs are drawn on the GPU from the seed alone: unit normals in bf16 for
activations, queries, keys and values (Q and K that give scores of unit variance),
weight matrices scaled by 1/sqrt(K).  q, k and v are slices of one fused
projection, pages are handed out in random order.
"""
from __future__ import annotations

import math

import torch

own = False

E4M3_MAX = 448.0


# ---------------------------------------------------------------------------
# The cases

def _append(T, B, Hkv, D, page, cached, fp8):
    """T new tokens spread over B sequences that hold up to `cached` tokens."""
    return dict(op="append", T=T, B=B, Hkv=Hkv, D=D, page=page, cached=cached, fp8=fp8)


def _attn(B, Hq, Hkv, D, page, max_len, ragged, fp8, out):
    return dict(op="attn", B=B, Hq=Hq, Hkv=Hkv, D=D, page=page, max_len=max_len, ragged=ragged,
                fp8=fp8, out=out)


def _gemm(M, N, K, act, bias, residual, out):
    return dict(op="gemm", M=M, N=N, K=K, act=act, bias=bias, residual=residual, out=out)


def listed():
    cases = {
        # the new token of each of 32 sequences, one decode step: all launch
        "append_decode_b32": _append(32, 32, 8, 128, 64, 4000, False),
        # a chunk of two prompts of odd length into an 8-bit cache
        "append_chunk_fp8_t2047": _append(2047, 2, 8, 128, 64, 600, True),
        # a batch of whole prompts
        "append_prefill_t16k": _append(16384, 4, 8, 128, 64, 0, False),
        # one short conversation, few heads: latency
        "attn_b1_s37_d64": _attn(1, 8, 2, 64, 16, 37, False, False, "bf16"),
        # one long document, one sequence: the cache's length has to fill the GPU
        "attn_b1_s100k_fp8": _attn(1, 32, 8, 128, 64, 100001, False, True, "bf16"),
        # a decode step of eight sequences of a grouped-query decoder against an 8k cache
        "attn_b8_s8191": _attn(8, 32, 8, 128, 64, 8191, False, False, "bf16"),
        # a serving batch of mixed lengths (an idle slot among them) in small pages
        "attn_b64_ragged_s16k": _attn(64, 32, 8, 128, 16, 16384, True, False, "bf16"),
        # every head with a cache of its own, fp32 result
        "attn_mha_b16_s2001_d64": _attn(16, 32, 32, 64, 32, 2001, False, False, "fp32"),
        # one token's output projection onto the residual stream
        "gemm_m1_n4096_k4096": _gemm(1, 4096, 4096, "none", False, True, "bf16"),
        # the MLP's first product of a decode step of 24 sequences
        "gemm_m24_n14336_k4096": _gemm(24, 14336, 4096, "gelu_tanh", True, False, "bf16"),
        # a chunk of tokens of odd length, odd widths, fp32 residual stream
        "gemm_m389_n4232_k8264": _gemm(389, 4232, 8264, "none", True, True, "fp32"),
        # the MLP's first product over a 4096 token prefill
        "gemm_m4096_n8192_k8192": _gemm(4096, 8192, 8192, "silu", True, False, "bf16"),
    }
    return [dict(name=n, **c) for n, c in cases.items()]


def _log(rng, lo, hi):
    """An integer in [lo, hi], even over the logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_any(rng):
    op = rng.choice(["append", "attn", "attn", "gemm", "gemm"])
    if op == "gemm":
        M = rng.choice([_log(rng, 1, 64), _log(rng, 1, 4096)])
        return _gemm(M, 8 * _log(rng, 8, 2048), 8 * _log(rng, 8, 2048),
                     rng.choice(["none", "none", "relu", "gelu", "gelu_tanh", "silu"]),
                     rng.random() < 0.5, rng.random() < 0.5, rng.choice(["bf16", "bf16", "fp32"]))
    Hkv, D = rng.choice([1, 2, 4, 8, 16, 32]), rng.choice([64, 128])
    page, fp8 = rng.choice([16, 32, 64, 128, 256]), rng.random() < 0.4
    B = _log(rng, 1, 128)
    if op == "append":
        T = B if rng.random() < 0.5 else max(B, _log(rng, 2, 16384))
        return _append(T, B, Hkv, D, page, _log(rng, 1, 4096), fp8)
    Hq = Hkv * rng.choice([g for g in (1, 2, 3, 4, 8, 16, 32) if Hkv * g <= 64])
    return _attn(B, Hq, Hkv, D, page, _log(rng, 1, 100001), rng.random() < 0.6, fp8,
                 rng.choice(["bf16", "fp32"]))


def draw(rng):
    top = [(c["op"], work(c), _held(c)) for c in listed()]
    while True:
        c = _draw_any(rng)
        w, held = work(c), _held(c)
        same = [t for t in top if t[0] == c["op"]]
        if (w["flops"] <= max(t[1]["flops"] for t in same)
                and w["bytes"] <= max(t[1]["bytes"] for t in same)
                and held <= max(t[2] for t in same)):
            return c


def _lengths(c):
    """The cached lengths of the sequences: all of them max_len, or from one to
    max_len, even over the logarithm, with an idle slot in a batch of eight or more."""
    B, top = c["B"], c["max_len"]
    if not c["ragged"]:
        return [top] * B
    lens = [round(top ** (i / max(1, B - 1))) for i in range(B)]
    if B >= 8:
        lens[0] = 0
    lens[-1] = top
    return lens


def _shares(c):
    """The new tokens of each sequence."""
    B, T = c["B"], c["T"]
    return [T // B + (b < T % B) for b in range(B)]


def _held(c):
    """Elements of the cache pages that a case holds (of B, for a product)."""
    if c["op"] == "gemm":
        return c["N"] * c["K"]
    most = c["max_len"] if c["op"] == "attn" else c["cached"] + max(_shares(c))
    return 2 * c["B"] * -(-most // c["page"]) * c["page"] * c["Hkv"] * c["D"]


# ---------------------------------------------------------------------------
# Inputs

def _normal(g, shape, std=1.0, dtype=torch.bfloat16):
    # drawn in slices of 2^27 elements, so that no fp32 copy of a large tensor is made
    t = torch.empty(shape, dtype=dtype, device=g.device)
    flat = t.view(-1)
    for i in range(0, flat.numel(), 1 << 27):
        s = flat[i:i + (1 << 27)]
        s.copy_(torch.randn(s.numel(), generator=g, device=g.device).mul_(std))
    return t


def _pages(g, c, most):
    """A page table [B, pages of `most` tokens] over a shuffled pool, the pool's two
    caches and their scales (None for bf16)."""
    B, Hkv, D, page = c["B"], c["Hkv"], c["D"], c["page"]
    per = -(-most // page)
    table = torch.randperm(B * per, generator=g, device=g.device).to(torch.int32).view(B, per)
    shape = (B * per, Hkv, page, D)
    if not c["fp8"]:
        return table, _normal(g, shape), _normal(g, shape), None, None
    # e4m3 with a scale per head that puts unit normals at 4.5 sigma of its range
    top = torch.rand(2, Hkv, generator=g, device=g.device).mul_(0.2).add_(0.9)
    ks, vs = (top * (4.5 / E4M3_MAX)).unbind(0)
    std = E4M3_MAX / 4.5
    return (table, _normal(g, shape, std, torch.bfloat16).clamp_(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn),
            _normal(g, shape, std, torch.bfloat16).clamp_(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn),
            ks.contiguous(), vs.contiguous())


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    c = case
    if c["op"] == "gemm":
        M, N, K = c["M"], c["N"], c["K"]
        out = torch.bfloat16 if c["out"] == "bf16" else torch.float32
        return dict(case=c, a=_normal(g, (M, K)), b=_normal(g, (K, N), std=K ** -0.5),
                    bias=_normal(g, (N,)) if c["bias"] else None,
                    residual=_normal(g, (M, N), dtype=out) if c["residual"] else None, out=out)
    Hkv, D, B = c["Hkv"], c["D"], c["B"]
    if c["op"] == "append":
        shares, T = _shares(c), c["T"]
        table, kc, vc, ks, vs = _pages(g, c, c["cached"] + max(shares))
        qkv = _normal(g, (T, 6 * Hkv, D))
        held = torch.randint(0, c["cached"] + 1, (B,), generator=g, device=g.device)
        seq = torch.repeat_interleave(torch.arange(B, device=g.device),
                                      torch.tensor(shares, device=g.device), output_size=T)
        first = torch.tensor([sum(shares[:b]) for b in range(B)], device=g.device)
        pos = held[seq] + torch.arange(T, device=g.device) - first[seq]
        return dict(case=c, k=qkv[:, 4 * Hkv:5 * Hkv], v=qkv[:, 5 * Hkv:], kc=kc, vc=vc, ks=ks, vs=vs,
                    table=table, pos=pos.to(torch.int32), seq=seq.to(torch.int32))
    Hq = c["Hq"]
    table, kc, vc, ks, vs = _pages(g, c, c["max_len"])
    qkv = _normal(g, (B, Hq + 2 * Hkv, D))
    lens = torch.tensor(_lengths(c), device=g.device)
    lens = lens[torch.randperm(B, generator=g, device=g.device)]
    return dict(case=c, q=qkv[:, :Hq], kc=kc, vc=vc, ks=ks, vs=vs, table=table,
                lens=lens.to(torch.int32),
                out=torch.bfloat16 if c["out"] == "bf16" else torch.float32)


# ---------------------------------------------------------------------------
# One pass

def _values(cache, scale):
    """What a cache holds: itself, or the values that its 8-bit numbers stand for."""
    return cache if scale is None else cache.float() * scale[:, None, None]


def run(state):
    if own:
        return _run_own(state)
    return _PLAIN[state["case"]["op"]](state)


def _run_own(s):
    from paper_2504_17577_amd import tileattn

    c = s["case"]
    if c["op"] == "append":
        kc, vc = tileattn.kv_cache_append(s["k"], s["v"], s["kc"], s["vc"], s["table"], s["pos"],
                                          seq=s["seq"], k_scale=s["ks"], v_scale=s["vs"])
        return _values(kc, s["ks"]), _values(vc, s["vs"])
    if c["op"] == "attn":
        return tileattn.attn_decode_paged(s["q"], s["kc"], s["vc"], s["table"], s["lens"],
                                          k_scale=s["ks"], v_scale=s["vs"], out_dtype=s["out"])
    return tileattn.gemm_bf16_epilogue(s["a"], s["b"], bias=s["bias"], activation=c["act"],
                                       residual=s["residual"], out_dtype=s["out"])


def _store(cache, scale, page, offset, x):
    if scale is None:
        cache[page, :, offset] = x
    else:
        x = (x.float() / scale[:, None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
        cache.view(torch.uint8)[page, :, offset] = x.view(torch.uint8)
    return _values(cache, scale)


def _plain_append(s):
    pos, P = s["pos"].long(), s["case"]["page"]
    page, offset = s["table"][s["seq"].long(), pos // P].long(), pos % P
    return _store(s["kc"], s["ks"], page, offset, s["k"]), _store(s["vc"], s["vs"], page, offset, s["v"])


def _gathered(cache, scale, table):
    """[B, Hkv, positions, D] in 32 bits."""
    x = cache.view(torch.uint8)[table].view(cache.dtype) if scale is not None else cache[table]
    B, per, Hkv, P, D = x.shape
    x = x.transpose(1, 2).float().reshape(B, Hkv, per * P, D)
    return x if scale is None else x * scale[:, None, None]


def _plain_attn(s):
    q = s["q"].float()
    B, Hq, D = q.shape
    k, v = _gathered(s["kc"], s["ks"], s["table"].long()), _gathered(s["vc"], s["vs"], s["table"].long())
    Hkv = k.shape[1]
    sc = (q.view(B, Hkv, Hq // Hkv, D) @ k.transpose(2, 3)) * (1.0 / math.sqrt(D))
    hide = torch.arange(k.shape[2], device=q.device) >= s["lens"][:, None]
    sc = sc.masked_fill_(hide[:, None, None], -math.inf)
    m = sc.amax(3, keepdim=True).clamp_(min=-3e38)
    p = (sc - m).exp_()
    total = p.sum(3, keepdim=True)
    o = (p @ v) / total.clamp(min=1e-30)
    return o.view(B, Hq, D).to(s["out"]), (m + total.log()).view(B, Hq)


def _activated(x, act):
    if act == "relu":
        return x.clamp(min=0.0)
    if act == "gelu":
        return 0.5 * x * (1.0 + torch.erf(x * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * x * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (x + 0.044715 * x * x * x)))
    return x / (1.0 + torch.exp(-x)) if act == "silu" else x


def _plain_gemm(s):
    x = s["a"].float() @ s["b"].float()
    if s["bias"] is not None:
        x = x + s["bias"].float()
    x = _activated(x, s["case"]["act"])
    if s["residual"] is not None:
        x = x + s["residual"].float()
    return x.to(s["out"])


_PLAIN = {"append": _plain_append, "attn": _plain_attn, "gemm": _plain_gemm}


# ---------------------------------------------------------------------------
# What a pass cannot do without

def work(case):
    c = case
    if c["op"] == "gemm":
        M, N, K = c["M"], c["N"], c["K"]
        size = 2 if c["out"] == "bf16" else 4
        return {"bytes": 2 * (M * K + K * N) + size * M * N * (1 + c["residual"]) + 2 * N * c["bias"],
                "flops": 2 * M * N * K}
    size = 1 if c["fp8"] else 2
    if c["op"] == "append":
        n = 2 * c["T"] * c["Hkv"] * c["D"]
        return {"bytes": n * (2 + size) + 8 * c["T"], "flops": n}
    keys = sum(_lengths(c))
    rows = c["B"] * c["Hq"]
    return {"bytes": 2 * keys * c["Hkv"] * c["D"] * size + rows * (c["D"] * (4 if c["out"] == "bf16" else 6) + 4),
            "flops": 4 * keys * c["Hq"] * c["D"]}


# ---------------------------------------------------------------------------
# The same results in 64 bits

def _exact_append(s):
    def stored(cache, scale, x):
        held = cache.double() if scale is None else cache.double() * scale.double()[None, :, None, None]
        x = x.double()
        if scale is not None:   # the nearest e4m3 numbers of x / scale, as 64-bit values
            u = (x / scale.double()[None, :, None]).clamp(-E4M3_MAX, E4M3_MAX)
            step = torch.exp2(torch.floor(torch.log2(u.abs().clamp(min=2.0 ** -6))) - 3)
            x = torch.round(u / step) * step * scale.double()[None, :, None]
        flat = held.transpose(1, 2).reshape(-1, *held.shape[1:2], held.shape[3])
        P = s["case"]["page"]
        pos = s["pos"].long()
        at = s["table"].long()[s["seq"].long(), pos.div(P, rounding_mode="floor")] * P + pos.remainder(P)
        flat[at] = x
        return flat.view(held.shape[0], P, held.shape[1], held.shape[3]).transpose(1, 2).contiguous()

    return stored(s["kc"], s["ks"], s["k"]), stored(s["vc"], s["vs"], s["v"])


def _exact_attn(s):
    q = s["q"].double()
    B, Hq, D = q.shape
    Hkv, P = s["kc"].shape[1], s["kc"].shape[2]
    o = torch.zeros(B, Hq, D, dtype=torch.float64, device=q.device)
    lse = torch.full((B, Hq), -math.inf, dtype=torch.float64, device=q.device)
    for b, n in enumerate(s["lens"].tolist()):
        if n == 0:
            continue
        pages = s["table"][b, :-(-n // P)].tolist()
        k = torch.cat([s["kc"][p].double() for p in pages], 1)[:, :n]
        v = torch.cat([s["vc"][p].double() for p in pages], 1)[:, :n]
        if s["ks"] is not None:
            k = k * s["ks"].double()[:, None, None]
            v = v * s["vs"].double()[:, None, None]
        for h in range(Hkv):
            rows = slice(h * (Hq // Hkv), (h + 1) * (Hq // Hkv))
            sc = (k[h] @ q[b, rows].t().contiguous()).t() / math.sqrt(D)
            lse[b, rows] = torch.logsumexp(sc, 1)
            o[b, rows] = torch.exp(sc - lse[b, rows][:, None]) @ v[h]
    return o, lse


def _exact_gemm(s):
    x = s["a"].double() @ s["b"].double()
    if s["bias"] is not None:
        x += s["bias"].double()
    act = s["case"]["act"]
    if act == "relu":
        x = torch.where(x > 0, x, torch.zeros_like(x))
    elif act == "gelu":
        x = 0.5 * x * torch.erfc(-x / math.sqrt(2.0))
    elif act == "gelu_tanh":
        x = x * torch.sigmoid(2 * math.sqrt(2.0 / math.pi) * (x + 0.044715 * x ** 3))
    elif act == "silu":
        x = x * torch.sigmoid(x)
    if s["residual"] is not None:
        x += s["residual"].double()
    return x


def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "attn": _exact_attn, "gemm": _exact_gemm}[case["op"]](s)
