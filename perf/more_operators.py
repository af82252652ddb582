"""More calls of a decoder's serving step that this library is timed on: the norm and
position rotation of queries and keys on their way into the paged cache, attention of
one new token over a cache held in 4 bits, the matrix product with 4-bit weights, and
the choice of the next token from the logits, each beside its plain form in elementary
torch operations and its arithmetic in 64 bits.

4-bit numbers are MXFP4: e2m1 elements, two to a byte (the first in the low half), with
a power of two (e8m0, one byte) for every 32 of a row.

Inputs are drawn on the GPU from the seed alone: unit normals in bf16 for activations,
queries, keys and values, weights scaled by 1/sqrt(K), pages in random order, logits
whose spread differs from row to row.
"""
from __future__ import annotations

import math

import torch

own = False

E4M3_MAX = 448.0
GROUP = 32
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# ---------------------------------------------------------------------------
# The cases

def _append(T, B, Hq, Hkv, D, page, cached, cache, norm, rot, inter):
    """T new tokens spread over B sequences that hold up to `cached` tokens, the first
    `rot` dims of a head rotated, in pairs of neighbours (inter) or of halves."""
    return dict(op="append", T=T, B=B, Hq=Hq, Hkv=Hkv, D=D, page=page, cached=cached, cache=cache,
                norm=norm, rot=rot, inter=inter)


def _attn(B, Hq, Hkv, D, page, max_len, ragged, out):
    return dict(op="attn", B=B, Hq=Hq, Hkv=Hkv, D=D, page=page, max_len=max_len, ragged=ragged, out=out)


def _gemm(M, N, K, act, bias, residual, out):
    return dict(op="gemm", M=M, N=N, K=K, act=act, bias=bias, residual=residual, out=out)


def _sample(B, V, dtype, top_k, top_p, min_p):
    """One token of each of B rows of V logits; top_k 0 and top_p, min_p false: without."""
    return dict(op="sample", B=B, V=V, dtype=dtype, top_k=top_k, top_p=top_p, min_p=min_p)


def listed():
    cases = {
        # the new token of each of 32 sequences, one decode step: all launch
        "rope_decode_b32": _append(32, 32, 32, 8, 128, 64, 4000, "bf16", False, 128, False),
        # a chunk of two prompts of odd length into a 4-bit cache, queries and keys normed
        "rope_chunk_fp4_t2047": _append(2047, 2, 32, 8, 128, 64, 10, "mxfp4", True, 128, False),
        # a batch of whole prompts, queries and keys normed
        "rope_prefill_t16k": _append(16384, 4, 32, 8, 128, 64, 0, "bf16", True, 128, False),
        # one short conversation, few heads: latency
        "attn4_b1_s37_d64": _attn(1, 8, 2, 64, 16, 37, False, "bf16"),
        # a serving batch of mixed lengths (an idle slot among them) in small pages
        "attn4_b64_ragged_s16k": _attn(64, 32, 8, 128, 16, 16384, True, "bf16"),
        # one long document, one sequence: the cache's length has to fill the GPU
        "attn4_b1_s100k": _attn(1, 32, 8, 128, 64, 100001, False, "fp32"),
        # one token's output projection onto the residual stream
        "gemm4_m1_n4096_k4096": _gemm(1, 4096, 4096, "none", False, True, "bf16"),
        # the MLP's first product of a decode step of 24 sequences
        "gemm4_m24_n14336_k4096": _gemm(24, 14336, 4096, "gelu_tanh", True, False, "bf16"),
        # a chunk of tokens of odd length, odd widths, fp32 residual stream
        "gemm4_m1021_n4232_k8224": _gemm(1021, 4232, 8224, "none", True, True, "fp32"),
        # one conversation's next token from a vocabulary of 32000
        "sample_b1_v32000": _sample(1, 32000, "bf16", 50, True, False),
        # a batch without top-k: the nucleus may hold thousands of tokens
        "sample_b64_v128001_topp": _sample(64, 128001, "fp32", 0, True, False),
        # a large batch with every filter
        "sample_b256_v131072_all": _sample(256, 131072, "bf16", 64, True, True),
    }
    return [dict(name=n, **c) for n, c in cases.items()]


def _log(rng, lo, hi):
    """An integer in [lo, hi], even over the logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_any(rng):
    op = rng.choice(["append", "attn", "gemm", "gemm", "sample"])
    if op == "gemm":
        M = rng.choice([_log(rng, 1, 64), _log(rng, 1, 1021)])
        return _gemm(M, 8 * _log(rng, 8, 2048), 32 * _log(rng, 2, 512),
                     rng.choice(["none", "none", "relu", "gelu", "gelu_tanh", "silu"]),
                     rng.random() < 0.5, rng.random() < 0.5, rng.choice(["bf16", "bf16", "fp32"]))
    if op == "sample":
        return _sample(_log(rng, 1, 256), _log(rng, 100, 200000), rng.choice(["bf16", "fp32"]),
                       rng.choice([0, _log(rng, 1, 1000)]), rng.random() < 0.6, rng.random() < 0.3)
    Hkv, D = rng.choice([1, 2, 4, 8, 16, 32]), rng.choice([64, 128])
    page = rng.choice([16, 32, 64, 128, 256])
    B = _log(rng, 1, 128)
    Hq = Hkv * rng.choice([g for g in (1, 2, 3, 4, 8, 16, 32) if Hkv * g <= 64])
    if op == "append":
        T = B if rng.random() < 0.5 else max(B, _log(rng, 2, 16384))
        rot = rng.choice([D, D, D // 2, 16 * rng.randint(1, D // 16)])
        return _append(T, B, Hq, Hkv, D, page, _log(rng, 1, 4096), rng.choice(["bf16", "e4m3", "mxfp4"]),
                       rng.random() < 0.5, rot, rng.random() < 0.4)
    return _attn(B, Hq, Hkv, D, page, _log(rng, 1, 100001), rng.random() < 0.6, rng.choice(["bf16", "fp32"]))


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
    """Elements of the cache pages that a case holds (of the weights, for a product,
    of the logits)."""
    if c["op"] == "gemm":
        return c["N"] * c["K"]
    if c["op"] == "sample":
        return c["B"] * c["V"]
    most = c["max_len"] if c["op"] == "attn" else c["cached"] + max(_shares(c))
    return 2 * c["B"] * -(-most // c["page"]) * c["page"] * c["Hkv"] * c["D"]


# ---------------------------------------------------------------------------
# 4-bit numbers

def _mx_scale_bytes(groups):
    """The scale's byte of each group of 32 along the last dimension: the power of two
    that puts the group's largest number between 3.5 and 7 (at most 6 after rounding;
    an infinity counts as the largest number)."""
    top = groups.abs().amax(-1).clamp(max=torch.finfo(torch.float32).max)
    return (((top.float().view(torch.int32) + 0x200000) >> 23) - 2).clamp(1, 252)


def _mx_codes(x):
    """(bytes of two elements each, scale bytes) of x's rows of whole groups."""
    groups = x.float().unflatten(-1, (-1, GROUP))
    e = _mx_scale_bytes(groups)
    y = groups * torch.exp2(127.0 - e.float())[..., None]
    a = y.abs()
    code = ((a > 0.25).byte() + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0))
    code = (code + 8 * torch.signbit(y)).byte().flatten(-2)
    return code[..., 0::2] | (code[..., 1::2] << 4), e.byte()


def _mx_pairs(device, dtype):
    """The two numbers of every byte."""
    one = torch.tensor(LEVELS, device=device)
    one = torch.cat([one, -one])
    return torch.stack([one.repeat(16), one.repeat_interleave(16)], 1).to(dtype)


def _mx_values(codes, scales, dtype=torch.float32, pairs=None):
    """What codes [.., n / 2] with scales [.., n / 32] stand for."""
    pairs = _mx_pairs(codes.device, dtype) if pairs is None else pairs
    x = pairs[codes.int()].flatten(-2).unflatten(-1, (-1, GROUP))
    return (x * scales.view(torch.float8_e8m0fnu).to(dtype)[..., None]).flatten(-2)


def _normal(g, shape, std=1.0, dtype=torch.bfloat16):
    # drawn in slices of 2^27 elements, so that no fp32 copy of a large tensor is made
    t = torch.empty(shape, dtype=dtype, device=g.device)
    flat = t.view(-1)
    for i in range(0, flat.numel(), 1 << 27):
        s = flat[i:i + (1 << 27)]
        s.copy_(torch.randn(s.numel(), generator=g, device=g.device).mul_(std))
    return t


def _mx_normal(g, rows, n, std=1.0):
    """Codes [rows, n / 2] and scales [rows, n / 32] of normals, in slices of 2^25."""
    codes = torch.empty(rows, n // 2, dtype=torch.uint8, device=g.device)
    scales = torch.empty(rows, n // GROUP, dtype=torch.uint8, device=g.device)
    step = max(1, (1 << 25) // n)
    for i in range(0, rows, step):
        m = min(step, rows - i)
        codes[i:i + m], scales[i:i + m] = _mx_codes(
            torch.randn(m, n, generator=g, device=g.device).mul_(std))
    return codes, scales


# ---------------------------------------------------------------------------
# Inputs

def _table(g, c, most):
    """A page table [B, pages of `most` tokens] over a shuffled pool, and its size."""
    B, per = c["B"], -(-most // c["page"])
    table = torch.randperm(B * per, generator=g, device=g.device).to(torch.int32).view(B, per)
    return table, B * per


def _mx_cache(g, c, pages):
    Hkv, D, page = c["Hkv"], c["D"], c["page"]
    codes, scales = _mx_normal(g, pages * Hkv * page, D)
    return codes.view(pages, Hkv, page, D // 2), scales.view(pages, Hkv, page, D // GROUP)


def _prepare_append(c, g):
    Hq, Hkv, D, B, T, rot = c["Hq"], c["Hkv"], c["D"], c["B"], c["T"], c["rot"]
    shares = _shares(c)
    most = c["cached"] + max(shares)
    table, pages = _table(g, c, most)
    ks = vs = None
    if c["cache"] == "mxfp4":
        kc, ks = _mx_cache(g, c, pages)
        vc, vs = _mx_cache(g, c, pages)
    else:
        kc, vc = (_normal(g, (pages, Hkv, c["page"], D)) for _ in range(2))
        if c["cache"] == "e4m3":
            # a scale per head that puts unit normals at 4.5 sigma of its range
            top = torch.rand(2, Hkv, generator=g, device=g.device).mul_(0.2).add_(0.9)
            ks, vs = (s.contiguous() for s in (top * (4.5 / E4M3_MAX)).unbind(0))
            std = E4M3_MAX / 4.5
            kc, vc = ((x * std).clamp_(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn) for x in (kc, vc))
    qkv = _normal(g, (T, Hq + 2 * Hkv, D))
    held = torch.randint(0, c["cached"] + 1, (B,), generator=g, device=g.device)
    seq = torch.repeat_interleave(torch.arange(B, device=g.device),
                                  torch.tensor(shares, device=g.device), output_size=T)
    first = torch.tensor([sum(shares[:b]) for b in range(B)], device=g.device)
    pos = held[seq] + torch.arange(T, device=g.device) - first[seq]
    angle = (torch.arange(most, device=g.device, dtype=torch.float64)[:, None]
             * 10000.0 ** (-torch.arange(0, rot, 2, device=g.device, dtype=torch.float64) / rot))
    w = [(_normal(g, (D,), 0.2) + 1.0) if c["norm"] else None for _ in range(2)]
    pairs = _mx_pairs(g.device, torch.bfloat16)
    return dict(case=c, pairs=pairs, q=qkv[:, :Hq], k=qkv[:, Hq:Hq + Hkv], v=qkv[:, Hq + Hkv:], qw=w[0], kw=w[1],
                cos_sin=torch.cat([angle.cos(), angle.sin()], 1).float(), kc=kc, vc=vc, ks=ks, vs=vs,
                table=table, pos=pos.to(torch.int32), seq=seq.to(torch.int32))


def _prepare_attn(c, g):
    Hq, Hkv, D, B = c["Hq"], c["Hkv"], c["D"], c["B"]
    table, pages = _table(g, c, c["max_len"])
    kc, ks = _mx_cache(g, c, pages)
    vc, vs = _mx_cache(g, c, pages)
    qkv = _normal(g, (B, Hq + 2 * Hkv, D))
    lens = torch.tensor(_lengths(c), device=g.device)
    lens = lens[torch.randperm(B, generator=g, device=g.device)]
    return dict(case=c, q=qkv[:, :Hq], kc=kc, vc=vc, ks=ks, vs=vs, table=table, lens=lens.to(torch.int32),
                out=torch.bfloat16 if c["out"] == "bf16" else torch.float32)


def _prepare_gemm(c, g):
    M, N, K = c["M"], c["N"], c["K"]
    out = torch.bfloat16 if c["out"] == "bf16" else torch.float32
    w, ws = _mx_normal(g, N, K, K ** -0.5)
    return dict(case=c, a=_normal(g, (M, K)), w=w, ws=ws, bias=_normal(g, (N,)) if c["bias"] else None,
                residual=_normal(g, (M, N), dtype=out) if c["residual"] else None, out=out)


def _prepare_sample(c, g):
    B, V = c["B"], c["V"]
    rand = lambda lo, hi: torch.rand(B, generator=g, device=g.device).mul_(hi - lo).add_(lo)  # noqa: E731
    logits = torch.randn(B, V, generator=g, device=g.device)
    logits *= torch.exp(rand(math.log(1.0), math.log(4.0)))[:, None]      # from unsure to sure
    some = torch.randint(0, V, (B, 8), generator=g, device=g.device)      # a few that the context favours
    logits.scatter_add_(1, some, torch.rand(B, 8, generator=g, device=g.device).mul_(6.0))
    temperature = rand(0.6, 1.2)
    if B >= 8:
        temperature[torch.randint(0, B, (1,), generator=g, device=g.device)] = 0.0   # a greedy request
    top_k = torch.full((B,), c["top_k"], dtype=torch.int32, device=g.device) if c["top_k"] else None
    return dict(case=c, logits=logits.to(torch.bfloat16 if c["dtype"] == "bf16" else torch.float32),
                u=torch.rand(B, generator=g, device=g.device), temperature=temperature, top_k=top_k,
                top_p=rand(0.8, 0.98) if c["top_p"] else None, min_p=rand(0.01, 0.1) if c["min_p"] else None)


_PREPARE = {"append": _prepare_append, "attn": _prepare_attn, "gemm": _prepare_gemm, "sample": _prepare_sample}


def prepare(case, seed):
    return _PREPARE[case["op"]](case, torch.Generator(device="cuda").manual_seed(seed))


# ---------------------------------------------------------------------------
# One pass

def run(state):
    if own:
        return _run_own(state)
    return _PLAIN[state["case"]["op"]](state)


def _held_values(cache, scale, kind, pairs):
    """What a cache holds, 8 and 4 bits as the values that they stand for."""
    if kind == "mxfp4":
        return _mx_values(cache, scale, torch.bfloat16, pairs)
    return (cache.float() * scale[:, None, None]).to(torch.bfloat16) if kind == "e4m3" else cache


def _run_own(s):
    from paper_2504_17577_amd import tileattn

    c = s["case"]
    if c["op"] == "append":
        q, kc, vc = tileattn.qk_norm_rope_append(
            s["q"], s["k"], s["v"], s["kc"], s["vc"], s["table"], s["pos"], cos_sin=s["cos_sin"],
            q_weight=s["qw"], k_weight=s["kw"], interleaved=c["inter"], seq=s["seq"],
            k_scale=s["ks"], v_scale=s["vs"])
        return (q, _held_values(kc, s["ks"], c["cache"], s["pairs"]),
                _held_values(vc, s["vs"], c["cache"], s["pairs"]))
    if c["op"] == "attn":
        return tileattn.attn_decode_paged(s["q"], s["kc"], s["vc"], s["table"], s["lens"],
                                          k_scale=s["ks"], v_scale=s["vs"], out_dtype=s["out"])
    if c["op"] == "gemm":
        return tileattn.gemm_mxfp4_epilogue(s["a"], s["w"], s["ws"], bias=s["bias"], activation=c["act"],
                                            residual=s["residual"], out_dtype=s["out"])
    return tileattn.sample_logits(s["logits"], s["u"], temperature=s["temperature"], top_k=s["top_k"],
                                  top_p=s["top_p"], min_p=s["min_p"])


def _rotated(x, weight, s):
    """x's heads normed (where there is a weight) and rotated, in x's type."""
    c = s["case"]
    if weight is not None:
        x = x / ((x * x).mean(-1, keepdim=True) + 1e-6).sqrt() * weight.to(x.dtype)
    half = c["rot"] // 2
    turn = s["cos_sin"][s["pos"].long()].to(x.dtype)[:, None]
    cos, sin = turn[..., :half], turn[..., half:]
    a, b = (x[..., 0:c["rot"]:2], x[..., 1:c["rot"]:2]) if c["inter"] else (x[..., :half], x[..., half:2 * half])
    a, b = a * cos - b * sin, b * cos + a * sin
    y = torch.stack([a, b], -1).flatten(-2) if c["inter"] else torch.cat([a, b], -1)
    return torch.cat([y, x[..., c["rot"]:]], -1)


def _store(cache, scale, kind, pairs, page, offset, x):
    """x [T, Hkv, D], in 32 or 64 bits, into its places; what the cache then holds."""
    if kind == "mxfp4":
        cache[page, :, offset], scale[page, :, offset] = _mx_codes(x)
    elif kind == "e4m3":
        x = (x.double() / scale.double()[:, None]).clamp(-E4M3_MAX, E4M3_MAX).float().to(torch.float8_e4m3fn)
        cache.view(torch.uint8)[page, :, offset] = x.view(torch.uint8)
    else:
        cache[page, :, offset] = x.to(cache.dtype)
    return _held_values(cache, scale, kind, pairs)


def _plain_append(s):
    pos, P, kind = s["pos"].long(), s["case"]["page"], s["case"]["cache"]
    page, offset = s["table"][s["seq"].long(), pos // P].long(), pos % P
    q = _rotated(s["q"].float(), s["qw"], s).to(torch.bfloat16)
    # keys in 64 bits: one that lies next to the border of two of the cache's numbers
    k = _rotated(s["k"].double(), s["kw"], s)
    return (q, _store(s["kc"], s["ks"], kind, s["pairs"], page, offset, k),
            _store(s["vc"], s["vs"], kind, s["pairs"], page, offset, s["v"].float()))


def _gathered(cache, scale, table):
    """[B, Hkv, positions, D] in 32 bits."""
    x = _mx_values(cache[table].transpose(1, 2), scale[table].transpose(1, 2))
    return x.flatten(2, 3)


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
    x = s["a"].float() @ _mx_values(s["w"], s["ws"]).t()
    if s["bias"] is not None:
        x = x + s["bias"].float()
    x = _activated(x, s["case"]["act"])
    if s["residual"] is not None:
        x = x + s["residual"].float()
    return x.to(s["out"])


def _plain_sample(s):
    """Weights and their sums in 64 bits: they decide at borders."""
    x = s["logits"].float()
    B, V = x.shape
    best = x.amax(1, keepdim=True)
    greedy = s["temperature"] == 0
    T = torch.where(greedy, 1.0, s["temperature"]).double()[:, None]
    w = ((x.double() - best) / T).exp()
    _, order = torch.sort(x, dim=1, descending=True, stable=True)    # ties: lower index first
    ws = w.gather(1, order)
    keep = torch.ones_like(ws, dtype=torch.bool)
    if s["top_k"] is not None:
        keep &= torch.arange(V, device=x.device) < s["top_k"][:, None]
    if s["top_p"] is not None:
        held = ws * keep
        before = held.cumsum(1) - held
        keep &= before < s["top_p"].double()[:, None] * held.sum(1, keepdim=True)
    if s["min_p"] is not None:
        keep &= ws >= s["min_p"].double()[:, None]
    keep[:, 0] = True
    kept = w * torch.zeros_like(keep).scatter_(1, order, keep)
    upto = kept.cumsum(1)
    token = (upto <= s["u"].double()[:, None] * upto[:, -1:]).sum(1).clamp_(max=V - 1)
    first = torch.where(x == best, torch.arange(V, device=x.device), V).amin(1)
    token = torch.where(greedy, first, token)
    logp = (x.double().gather(1, token[:, None]) - best) / T - w.sum(1, keepdim=True).log()
    return token.to(torch.int32), logp[:, 0].float()


_PLAIN = {"append": _plain_append, "attn": _plain_attn, "gemm": _plain_gemm, "sample": _plain_sample}


# ---------------------------------------------------------------------------
# What a pass cannot do without

def work(case):
    c = case
    if c["op"] == "gemm":
        M, N, K = c["M"], c["N"], c["K"]
        size = 2 if c["out"] == "bf16" else 4
        return {"bytes": 2 * M * K + N * K * 17 // 32 + size * M * N * (1 + c["residual"]) + 2 * N * c["bias"],
                "flops": 2 * M * N * K}
    if c["op"] == "sample":
        n = c["B"] * c["V"]
        return {"bytes": n * (2 if c["dtype"] == "bf16" else 4) + c["B"] * 28, "flops": 4 * n}
    if c["op"] == "append":
        q, kv = c["T"] * c["Hq"] * c["D"], 2 * c["T"] * c["Hkv"] * c["D"]
        size = {"bf16": 64, "e4m3": 32, "mxfp4": 17}[c["cache"]]
        return {"bytes": 4 * q + 2 * kv + kv * size // 32 + c["T"] * (8 + 4 * c["rot"]),
                "flops": 6 * q + 3 * kv}
    keys, rows = sum(_lengths(c)), c["B"] * c["Hq"]
    return {"bytes": 2 * keys * c["Hkv"] * c["D"] * 17 // 32 + rows * (c["D"] * (4 if c["out"] == "bf16" else 6) + 4),
            "flops": 4 * keys * c["Hq"] * c["D"]}


# ---------------------------------------------------------------------------
# The same results in 64 bits

def _numbers(codes, scales):
    """The 64-bit values of 4-bit numbers, from their fields."""
    nib = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).long()
    exp, man = (nib >> 1) & 3, (nib & 1).double()
    x = torch.where(exp > 0, (1.0 + man / 2) * 2.0 ** (exp - 1).double(), man / 2)
    x = torch.where(nib >= 8, -x, x)
    return x * (2.0 ** (scales.double() - 127.0)).repeat_interleave(GROUP, -1)


def _exact_append(s):
    c = s["case"]

    def turned(x, weight):
        x = x.double()
        if weight is not None:
            x = x * torch.rsqrt(x.pow(2).sum(-1, keepdim=True) / c["D"] + 1e-6) * weight.double()
        n = c["rot"] // 2
        z = torch.complex(*(t.contiguous() for t in s["cos_sin"][s["pos"].long()].double().split(n, 1)))[:, None]
        part = x[..., :c["rot"]]
        pair = part.unflatten(-1, (n, 2)) if c["inter"] else part.unflatten(-1, (2, n)).transpose(-1, -2)
        y = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * z)
        y = y.flatten(-2) if c["inter"] else y.transpose(-1, -2).flatten(-2)
        return torch.cat([y, x[..., c["rot"]:]], -1)

    def rounded(x, scale):
        if c["cache"] == "e4m3":      # the nearest e4m3 numbers of x / scale
            u = (x / scale.double()[None, :, None]).clamp(-E4M3_MAX, E4M3_MAX)
            step = torch.exp2(torch.floor(torch.log2(u.abs().clamp(min=2.0 ** -6))) - 3)
            return torch.round(u / step) * step * scale.double()[None, :, None]
        if c["cache"] == "mxfp4":     # the nearest e2m1 numbers of x / 2^e
            g = x.unflatten(-1, (-1, GROUP))
            top = g.abs().amax(-1, keepdim=True).clamp(min=2.0 ** -120)
            low = torch.floor(torch.log2(top))
            e = torch.exp2(low - 2 + (top >= 1.75 * torch.exp2(low)))
            u = (g / e).clamp(-6.0, 6.0)
            step = torch.exp2(torch.floor(torch.log2(u.abs().clamp(min=1.0))) - 1)
            return (torch.round(u / step) * step * e).flatten(-2)
        return x

    def stored(cache, scale, x):
        if c["cache"] == "mxfp4":
            held = _numbers(cache, scale)
        else:
            held = cache.double() if scale is None else cache.double() * scale.double()[None, :, None, None]
        flat = held.transpose(1, 2).reshape(-1, held.shape[1], held.shape[3])
        P, pos = c["page"], s["pos"].long()
        at = s["table"].long()[s["seq"].long(), pos.div(P, rounding_mode="floor")] * P + pos.remainder(P)
        flat[at] = rounded(x, scale)
        return flat.view(held.shape[0], P, held.shape[1], held.shape[3]).transpose(1, 2).contiguous()

    return (turned(s["q"], s["qw"]), stored(s["kc"], s["ks"], turned(s["k"], s["kw"])),
            stored(s["vc"], s["vs"], s["v"].double()))


def _exact_attn(s):
    q = s["q"].double()
    B, Hq, D = q.shape
    Hkv, P = s["kc"].shape[1], s["kc"].shape[2]
    o = torch.zeros(B, Hq, D, dtype=torch.float64, device=q.device)
    lse = torch.full((B, Hq), -math.inf, dtype=torch.float64, device=q.device)
    for b, n in enumerate(s["lens"].tolist()):
        if n == 0:
            continue
        pages = s["table"][b, :-(-n // P)].long()
        k, v = (_numbers(c[pages], e[pages]).transpose(0, 1).flatten(1, 2)[:, :n]
                for c, e in ((s["kc"], s["ks"]), (s["vc"], s["vs"])))
        for h in range(Hkv):
            rows = slice(h * (Hq // Hkv), (h + 1) * (Hq // Hkv))
            sc = (k[h] @ q[b, rows].t().contiguous()).t() / math.sqrt(D)
            lse[b, rows] = torch.logsumexp(sc, 1)
            o[b, rows] = torch.exp(sc - lse[b, rows][:, None]) @ v[h]
    return o, lse


def _exact_gemm(s):
    x = s["a"].double() @ _numbers(s["w"], s["ws"]).t().contiguous()
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


def _exact_sample(s):
    """Row by row: the kept tokens' list, then the walk along it in order of index."""
    c = s["case"]
    V = c["V"]
    tokens, logps = [], []
    for b in range(c["B"]):
        x, T = s["logits"][b].double(), float(s["temperature"][b])
        z = x if T == 0 else x / T
        logp = z - torch.logsumexp(z, 0)
        if T == 0:
            token = int((x == x.max()).nonzero()[0])
        else:
            order = torch.sort(-x, stable=True).indices
            n = min(V, int(s["top_k"][b])) if s["top_k"] is not None else V
            p = logp[order[:n]].exp()
            if s["top_p"] is not None:
                reach = p.cumsum(0) >= float(s["top_p"][b]) * p.sum()
                n = min(n, int(reach.nonzero()[0]) + 1)
            if s["min_p"] is not None:
                n = max(1, min(n, int((p >= float(s["min_p"][b]) * p[0]).sum())))
            chosen = order[:n].sort().values
            upto = logp[chosen].exp().cumsum(0)
            token = int(chosen[(upto > float(s["u"][b]) * upto[-1]).nonzero()[0]])
        tokens.append(token)
        logps.append(logp[token])
    return torch.tensor(tokens, dtype=torch.int32, device=x.device), torch.stack(logps)


def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "attn": _exact_attn, "gemm": _exact_gemm, "sample": _exact_sample}[case["op"]](s)
