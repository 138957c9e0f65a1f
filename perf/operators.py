"""Operators of a transformer's decoding step on 4-bit operands, as timed cases.

The kinds, each one call of a user's program:

  quantize    activations to MXFP4 and back (mxfp4_quantize, mxfp4_dequantize): the values that
              the 4-bit codes and their block scales stand for
  linear      mxfp4_linear on bf16 activations and a weight that is stored in MXFP4
  rotary      rotary positions on the heads of a tensor
  append      keys (rotated) and values of new tokens into a paged cache
  attention   one new token a sequence over its pages of the cache

``run`` computes them in plain torch operations, or, with ``own`` set, by the package's calls.
"""
import math

import torch

own = False

BLOCK = 32
BASE = 10000.0
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
MOST_MACS = 4608 * 8192 * 8192
MOST_QUANTIZED = 18432 * 4608
MOST_ROTATED = 4608 * 32 * 128
MOST_CACHED = 262144 * 8 * 128


# ------------------------------------------------------------------- the cases

def listed():
    def linear(name, M, K, N, gelu=False, bias=True):
        return {"name": name, "kind": "linear", "M": M, "K": K, "N": N, "gelu": gelu, "bias": bias}

    def rotary(name, tokens, heads, d, rot, layout, head_major, last):
        return {"name": name, "kind": "rotary", "tokens": tokens, "heads": heads, "d": d, "rot": rot,
                "layout": layout, "head_major": head_major, "last": last}

    def append(name, seqs, new, kv, d, page, layout, last, fp8):
        return {"name": name, "kind": "append", "seqs": seqs, "new": new, "kv": kv, "d": d,
                "page": page, "layout": layout, "last": last, "fp8": fp8}

    def attention(name, seqs, kv, group, d, page, shortest, longest, fp8, window=0):
        return {"name": name, "kind": "attention", "seqs": seqs, "kv": kv, "group": group, "d": d,
                "page": page, "shortest": shortest, "longest": longest, "fp8": fp8,
                "window": window}

    return [
        # a few tokens of a 1152-wide model: launches and latency
        {"name": "quantize_33", "kind": "quantize", "M": 33, "K": 1152},
        # the batched input of an MLP's second layer: memory traffic
        {"name": "quantize_18432", "kind": "quantize", "M": 18432, "K": 4608},
        # one token through a 4096-wide layer: the weight is read once, latency
        linear("linear_token", 1, 4096, 4096),
        # a ragged layer with GELU (333 tokens, N no multiple of a tile)
        linear("linear_ragged", 333, 2048, 1000, gelu=True),
        # a whole sequence through an 8192-wide layer: the matrix product itself
        linear("linear_large", 4608, 8192, 8192, bias=False),
        # the queries and keys of one decoding step, far along, half of each head rotated
        rotary("rotary_step", 32, 40, 128, 64, "half", False, 1 << 20),
        # a whole sequence's queries, head by head as the attention takes them
        rotary("rotary_sequence", 4608, 32, 128, 128, "interleaved", True, 4608),
        # one new token of each of 64 sequences into a bf16 cache
        append("append_step", 64, 1, 8, 128, 16, "half", 4096, False),
        # prompts of 1153 tokens into an e4m3 cache
        append("append_prompts", 4, 1153, 8, 128, 64, "interleaved", 1153, True),
        # four short sequences, one of them still empty: latency
        attention("attention_short", 4, 8, 4, 128, 16, 0, 333, False),
        # a ragged batch over an e4m3 cache, as a server holds it
        attention("attention_batch", 64, 8, 5, 128, 64, 129, 4096, True),
        # one very long context: the cache is read once
        attention("attention_long", 1, 8, 8, 128, 64, 262143, 262143, False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["quantize", "quantize", "linear", "linear", "linear", "rotary", "rotary",
                       "append", "append", "attention", "attention", "attention"])
    if kind == "quantize":
        while True:
            M, K = _log(rng, 1, 18432), 64 * _log(rng, 1, 192)
            if M * K <= MOST_QUANTIZED:
                return {"kind": kind, "M": M, "K": K}
    if kind == "linear":
        while True:
            M, K, N = _log(rng, 1, 4608), 64 * _log(rng, 8, 192), _log(rng, 64, 12288)
            if M * K * N <= MOST_MACS:
                return {"kind": kind, "M": M, "K": K, "N": N, "gelu": rng.random() < 0.3,
                        "bias": rng.random() < 0.7}
    d = rng.choice([64, 128, 128, 256])
    layout = rng.choice(["half", "interleaved"])
    if kind == "rotary":
        while True:
            tokens, heads = _log(rng, 1, 18432), _log(rng, 1, 64)
            if tokens * heads * d <= MOST_ROTATED:
                return {"kind": kind, "tokens": tokens, "heads": heads, "d": d,
                        "rot": rng.choice([d, d, d // 2, d // 4, 20]), "layout": layout,
                        "head_major": rng.random() < 0.4, "last": _log(rng, tokens + 1, 1 << 21)}
    kv, page, fp8 = rng.choice([1, 2, 4, 8, 8, 16, 32]), rng.choice([8, 16, 16, 32, 64, 128]), rng.random() < 0.5
    if kind == "append":
        while True:
            seqs, new = _log(rng, 1, 256), rng.choice([1, _log(rng, 2, 4608)])
            last = _log(rng, new, max(new, 8192))
            if max(seqs * new * 64, seqs * (last + page)) * kv * d <= MOST_CACHED:
                return {"kind": kind, "seqs": seqs, "new": new, "kv": kv, "d": d, "page": page,
                        "layout": layout, "last": last, "fp8": fp8}
    while True:
        seqs, longest = _log(rng, 1, 256), _log(rng, 1, 262144)
        if seqs * (longest + page) * kv * d <= MOST_CACHED:
            return {"kind": kind, "seqs": seqs, "kv": kv, "group": rng.choice([1, 2, 4, 5, 8, 16]),
                    "d": d, "page": page, "shortest": rng.randint(0, longest), "longest": longest,
                    "fp8": fp8, "window": rng.choice([0, 0, 0, _log(rng, 1, longest)])}


# ------------------------------------------------------------------- inputs

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 6007 + 101)


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _randint(g, lo, hi, shape):
    return torch.randint(lo, hi, shape, generator=g, device="cuda", dtype=torch.int32)


def _tokens(g, M, K):
    """Transformer activations: heavy tails and a few outlier channels."""
    x = _randn(g, M, K) * torch.exp(0.5 * _randn(g, M, K))
    x[:, torch.randperm(K, generator=g, device="cuda")[:max(1, K // 500)]] *= 60.0
    return x.mul_(0.3).bfloat16()


def _frequencies(rot):
    """Turns a position of each pair, as 64-bit fixed-point fractions of a turn (int64 tensor)."""
    turns = [int(BASE ** (-2.0 * i / rot) / (2.0 * math.pi) * 2.0 ** 64) for i in range(rot // 2)]
    return torch.tensor([t - (1 << 64) if t >= 1 << 63 else t for t in turns], dtype=torch.int64,
                        device="cuda")


def _lengths(case):
    """The batch's lengths, evenly from the shortest to the longest."""
    n, lo, hi = case["seqs"], case["shortest"], case["longest"]
    return [hi if n == 1 else lo + (hi - lo) * i // (n - 1) for i in range(n)]


def _pages(g, lengths, page):
    """Page table of sequences of these lengths over shuffled pages (unused entries -1), and the
    number of pages."""
    need = [-(-n // page) for n in lengths]
    order = torch.randperm(sum(need) + 1, generator=g, device="cuda").to(torch.int32)
    have = torch.tensor(need, device="cuda")
    first = torch.cumsum(have, 0) - have
    col = torch.arange(max(max(need), 1), device="cuda")
    at = (first[:, None] + col[None]).clamp(max=sum(need))
    return torch.where(col[None] < have[:, None], order[at], -1).to(torch.int32), sum(need) + 1


def _cache(g, pages, case):
    """Keys and values of a layer: [pages, kv heads, page, d], bf16 or e4m3."""
    shape = (pages, case["kv"], case["page"], case["d"])
    dtype = torch.float8_e4m3fn if case["fp8"] else torch.bfloat16
    k, v = (torch.empty(shape, dtype=dtype, device="cuda") for _ in range(2))
    for t in (k, v):
        for part in t.split(max(1, (1 << 26) // (case["kv"] * case["page"] * case["d"]))):
            part.copy_(_randn(g, *part.shape))
    return k, v


def _tensors(case, seed):
    """The tensors of a case, from the seed alone."""
    g, kind = _gen(seed), case["kind"]
    if kind == "quantize":
        return {"x": _tokens(g, case["M"], case["K"])}
    if kind == "linear":
        K, N = case["K"], case["N"]
        # a stored MXFP4 weight: codes [K/32, N, 16] (element 2i in the low half of byte i), block
        # scales [K/128 rounded up, N, 4]
        return {"x": _tokens(g, case["M"], K),
                "codes": torch.randint(0, 256, (K // BLOCK, N, BLOCK // 2), generator=g, device="cuda",
                                       dtype=torch.uint8),
                "scales": torch.randint(118, 122, (-(-K // 128), N, 4), generator=g, device="cuda",
                                        dtype=torch.uint8),
                "bias": _randn(g, N).bfloat16() if case["bias"] else None}
    if kind == "rotary":
        tokens, heads, d = case["tokens"], case["heads"], case["d"]
        x = _randn(g, *((heads, tokens, d) if case["head_major"] else (tokens, heads, d))).bfloat16()
        positions = torch.sort(_randint(g, 0, case["last"], (tokens,)))[0].to(torch.int32)
        return {"x": x.transpose(0, 1) if case["head_major"] else x, "positions": positions,
                "freqs": _frequencies(case["rot"])}
    if kind == "append":
        seqs, new, kv, d = case["seqs"], case["new"], case["kv"], case["d"]
        table, pages = _pages(g, [case["last"]] * seqs, case["page"])
        k, v = _cache(g, pages, case)
        first = _randint(g, 0, case["last"] - new + 1, (seqs, 1))
        positions = first + torch.arange(new, device="cuda", dtype=torch.int32)[None]
        kv_new = _randn(g, seqs * new, 2, kv, d).bfloat16()
        return {"k_cache": k, "v_cache": v, "table": table, "k": kv_new[:, 0], "v": kv_new[:, 1],
                "positions": positions.reshape(-1).to(torch.int32), "freqs": _frequencies(d),
                "sequences": torch.arange(seqs, device="cuda", dtype=torch.int32).repeat_interleave(new)}
    lengths = _lengths(case)
    order = torch.randperm(len(lengths), generator=g, device="cuda").tolist()
    lengths = [lengths[i] for i in order]
    table, pages = _pages(g, lengths, case["page"])
    k, v = _cache(g, pages, case)
    return {"k_cache": k, "v_cache": v, "table": table,
            "q": 2.0 * _randn(g, case["seqs"], case["kv"] * case["group"], case["d"]),
            "lengths": torch.tensor(lengths, device="cuda", dtype=torch.int32)}


# scales of an e4m3 cache: a stored value stands for itself times the scale
K_SCALE, V_SCALE = 0.75, 1.25


def prepare(case, seed):
    t = _tensors(case, seed)
    if case["kind"] == "attention":
        t["q"] = t["q"].bfloat16()
    if case["kind"] in ("append", "attention"):
        t["k_scale"], t["v_scale"] = (K_SCALE, V_SCALE) if case["fp8"] else (1.0, 1.0)
    return {"case": case, **t}


# ------------------------------------------------------------------- one pass

def run(s):
    kind = s["case"]["kind"]
    if own:
        return _run_own(s, s["case"], kind)
    return {"quantize": _plain_quantize, "linear": _plain_linear, "rotary": _plain_rotary,
            "append": _plain_append, "attention": _plain_attention}[kind](s, s["case"])


def _run_own(s, c, kind):
    import paper_2509_26436_amd as q4
    if kind == "quantize":
        return {"values": q4.mxfp4_dequantize(q4.mxfp4_quantize(s["x"]))}
    if kind == "linear":
        w = q4.MxTensor(s["codes"], s["scales"], c["N"], c["K"])
        return {"y": q4.mxfp4_linear(s["x"], w, s["bias"], q4.EPI_GELU_TANH if c["gelu"] else q4.EPI_NONE)}
    if kind == "rotary":
        return {"y": q4.rotary(s["x"], s["positions"], s["freqs"], c["layout"])}
    cache = q4.PagedCache(s["k_cache"], s["v_cache"], s["table"], s["k_scale"], s["v_scale"])
    if kind == "append":
        q4.paged_append(cache, s["k"], s["v"], s["positions"], s["sequences"], s["freqs"], c["layout"])
        return {"k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    return {"o": q4.paged_attention(s["q"], cache, s["lengths"], window=c["window"])}


def _round_e2m1(v):
    """fp32 to the nearest e2m1 value, ties to the even code, saturating at 6."""
    a = v.abs()
    r = torch.where(a < 2, torch.round(a * 2) / 2,
                    torch.where(a < 4, torch.round(a), (torch.round(a / 2) * 2).clamp(max=6)))
    return torch.copysign(r, v)


def _mx_values(x):
    """The values that MXFP4 holds of x [M, K], in fp32."""
    b = x.float().reshape(x.shape[0], -1, BLOCK)
    top = b.abs().amax(-1, keepdim=True)
    e = torch.where(top > 0, torch.frexp(top)[1] - 3, -127).clamp(min=-127)
    return torch.ldexp(_round_e2m1(torch.ldexp(b, -e)), e).reshape(x.shape)


def _stored_values(codes, scales, N, K):
    """The values of a stored MXFP4 tensor as [N, K], in fp32."""
    table = torch.tensor([*E2M1, *(-v for v in E2M1)], device=codes.device)
    pairs = torch.stack([codes & 15, codes >> 4], -1).reshape(K // BLOCK, N, BLOCK)
    e = scales.permute(0, 2, 1).reshape(-1, N)[:K // BLOCK].int() - 127
    v = torch.ldexp(table[pairs.int()], e[..., None])
    return v.permute(1, 0, 2).reshape(N, K)


def _plain_quantize(s, c):
    return {"values": _mx_values(s["x"]).bfloat16()}


def _plain_linear(s, c):
    w = _stored_values(s["codes"], s["scales"], c["N"], c["K"])
    y = _mx_values(s["x"]) @ w.t()
    if s["bias"] is not None:
        y = y + s["bias"].float()
    if c["gelu"]:
        y = 0.5 * y * (1 + torch.tanh(math.sqrt(2 / math.pi) * (y + 0.044715 * y * y * y)))
    return {"y": y.bfloat16()}


def _rotate(x, positions, freqs, layout):
    """fp32 [tokens, heads, d] with its first 2 len(freqs) channels rotated; angles in 64 bits."""
    half = freqs.numel()
    turns = positions.double()[:, None] * (freqs.double() / 2.0 ** 64)[None]
    angle = 2 * math.pi * (turns - torch.floor(turns))
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    x = x.float()
    pair = x[..., :2 * half]
    if layout == "half":
        a, b = pair[..., :half], pair[..., half:]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = pair[..., 0::2], pair[..., 1::2]
        y = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([y, x[..., 2 * half:]], -1)


def _plain_rotary(s, c):
    return {"y": _rotate(s["x"], s["positions"], s["freqs"], c["layout"]).bfloat16()}


def _plain_append(s, c):
    k = _rotate(s["k"], s["positions"], s["freqs"], c["layout"]) / s["k_scale"]
    v = s["v"].float() / s["v_scale"]
    at, page = s["positions"].long(), c["page"]
    where = s["table"][s["sequences"].long(), at // page].long(), slice(None), at % page
    for cache, new in ((s["k_cache"], k), (s["v_cache"], v)):
        new = new.clamp(-448, 448).to(cache.dtype) if c["fp8"] else new.to(cache.dtype)
        raw = torch.uint8 if c["fp8"] else torch.bfloat16
        cache.view(raw)[where] = new.view(raw)
    return {"k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _plain_attention(s, c):
    seqs, kv, group, d = c["seqs"], c["kv"], c["group"], c["d"]
    table = s["table"].long().clamp(min=0)

    def gathered(cache, scale):
        t = cache.view(torch.uint8 if c["fp8"] else torch.bfloat16)[table].view(cache.dtype).float()
        return t.transpose(1, 2).reshape(seqs, kv, -1, d) * scale
    q = s["q"].float().reshape(seqs, kv, group, d)
    scores = torch.matmul(q, gathered(s["k_cache"], s["k_scale"]).transpose(2, 3)) / math.sqrt(d)
    at, n = torch.arange(scores.shape[-1], device=scores.device), s["lengths"][:, None]
    seen = (at < n) & (at >= n - c["window"]) if c["window"] else at < n
    scores = torch.where(seen[:, None, None], scores, -math.inf)
    p = torch.exp(scores - scores.amax(-1, keepdim=True).clamp(min=-3e38))
    o = torch.matmul(p, gathered(s["v_cache"], s["v_scale"])) / p.sum(-1, keepdim=True).clamp(min=1e-30)
    return {"o": o.reshape(seqs, kv * group, d).bfloat16()}


# ------------------------------------------------------------------- what a pass needs

def work(case):
    kind = case["kind"]
    if kind == "quantize":
        n = case["M"] * case["K"]
        return {"bytes": 4.0 * n, "flops": 4.0 * n}
    if kind == "linear":
        M, K, N = case["M"], case["K"], case["N"]
        return {"bytes": 2.0 * M * K + 0.53125 * N * K + 2.0 * N * case["bias"] + 2.0 * M * N,
                "flops": 2.0 * M * N * K}
    if kind == "rotary":
        n = case["tokens"] * case["heads"] * case["d"]
        return {"bytes": 4.0 * n + 4.0 * case["tokens"], "flops": 3.0 * n}
    if kind == "append":
        n = case["seqs"] * case["new"] * case["kv"] * case["d"]
        return {"bytes": 2.0 * n * (2 + (1 if case["fp8"] else 2)), "flops": 5.0 * n}
    keys = sum(min(n, case["window"] or n) for n in _lengths(case))
    heads, d = case["kv"] * case["group"], case["d"]
    return {"bytes": 2.0 * keys * case["kv"] * d * (1 if case["fp8"] else 2) + 4.0 * case["seqs"] * heads * d,
            "flops": 4.0 * keys * heads * d}


# ------------------------------------------------------------------- the same in 64 bits

def _exact_mx(x):
    """Nearest of the sixteen e2m1 values, by distance, in 64 bits (ties to the even code)."""
    levels = torch.tensor(E2M1, dtype=torch.float64, device=x.device)
    out = torch.empty(x.shape, dtype=torch.float64, device=x.device)
    for part, to in zip(x.split(1024), out.split(1024)):
        b = part.double().reshape(part.shape[0], -1, BLOCK)
        top = b.abs().amax(-1, keepdim=True)
        scale = torch.exp2(torch.floor(torch.log2(top)) - 2)
        scale = torch.where(top > 0, scale, torch.ones_like(scale)).clamp(min=2.0 ** -127)
        a = b.abs() / scale
        best, code = torch.full_like(a, math.inf), torch.zeros_like(a)
        for i, level in enumerate(E2M1):
            far = (a - level).abs()
            nearer = (far < best) | ((far == best) & (i % 2 == 0))
            best, code = torch.where(nearer, far, best), torch.where(nearer, float(i), code)
        to.copy_((levels[code.long()] * torch.sign(b) * scale).reshape(part.shape))
    return out


def _exact_rotation(x, positions, rot, layout):
    x = x.double().clone()
    for i in range(rot // 2):
        angle = torch.remainder(positions.double() * BASE ** (-2.0 * i / rot), 2 * math.pi)[:, None]
        j, k = (i, i + rot // 2) if layout == "half" else (2 * i, 2 * i + 1)
        a, b = x[..., j].clone(), x[..., k].clone()
        x[..., j] = a * torch.cos(angle) - b * torch.sin(angle)
        x[..., k] = a * torch.sin(angle) + b * torch.cos(angle)
    return x


def _exact_append(t, case):
    page, sequences, positions = case["page"], t["sequences"].tolist(), t["positions"].tolist()
    if len(positions) > 20000:
        return None
    scales = (K_SCALE, V_SCALE) if case["fp8"] else (1.0, 1.0)
    table = t["table"].tolist()
    at = torch.tensor([table[b][p // page] * page + p % page for b, p in zip(sequences, positions)],
                      device="cuda")
    out = {}
    for name, new, scale in (("k", _exact_rotation(t["k"], t["positions"], case["d"], case["layout"]), scales[0]),
                             ("v", t["v"].double(), scales[1])):
        cache = t[name + "_cache"].double().transpose(1, 2).reshape(-1, case["kv"], case["d"])
        cache[at] = new / scale
        out[name + "_cache"] = cache.reshape(-1, page, case["kv"], case["d"]).transpose(1, 2)
    return out


def _exact_attention(t, case):
    q, page, d = t["q"].bfloat16().double(), case["page"], case["d"]
    scales = (K_SCALE, V_SCALE) if case["fp8"] else (1.0, 1.0)
    out = torch.zeros_like(q)
    for b, n in enumerate(t["lengths"].tolist()):
        first = max(0, n - case["window"]) if case["window"] else 0
        if n == 0:
            continue
        at = t["table"][b, :-(-n // page)].long()
        for h in range(case["kv"]):
            k, v = (t[c][:, h].view(torch.uint8 if case["fp8"] else torch.bfloat16)[at].view(t[c].dtype)
                    .double().reshape(-1, d)[first:n] * s for c, s in zip(("k_cache", "v_cache"), scales))
            heads = slice(h * case["group"], (h + 1) * case["group"])
            out[b, heads] = torch.softmax(q[b, heads] @ k.t() / math.sqrt(d), -1) @ v
    return out


def exact(case, seed):
    t, kind = _tensors(case, seed), case["kind"]
    if kind == "quantize":
        return {"values": _exact_mx(t["x"])}
    if kind == "rotary":
        return {"y": _exact_rotation(t["x"], t["positions"], case["rot"], case["layout"])}
    if kind == "append":
        return _exact_append(t, case)
    if kind == "attention":
        return None if case["seqs"] * case["kv"] > 4096 else {"o": _exact_attention(t, case)}
    N, K = case["N"], case["K"]
    levels = torch.tensor([*E2M1, *(-v for v in E2M1)], dtype=torch.float64, device="cuda")
    w = torch.empty(N, K, dtype=torch.float64, device="cuda")
    for block in range(K // BLOCK):
        scale = torch.exp2(t["scales"][block // 4, :, block % 4].double() - 127)[:, None]
        c = t["codes"][block].long()
        w[:, block * BLOCK:(block + 1) * BLOCK:2] = levels[c % 16] * scale
        w[:, block * BLOCK + 1:(block + 1) * BLOCK:2] = levels[c // 16] * scale
    y = _exact_mx(t["x"]) @ w.t()
    if t["bias"] is not None:
        y += t["bias"].double()
    if case["gelu"]:
        y = y * 0.5 * (1 + torch.tanh(math.sqrt(2 / math.pi) * (y + 0.044715 * y ** 3)))
    return {"y": y}
