"""The operators around a verification call, as cases that can be timed and compared.

A verification call runs the model on a block of drafted tokens behind each sequence's context.  Four operators of the
package serve it besides the drafting, the head and the acceptance:

  attention  ``tree_attention``: a block of drafted nodes attends to the cached context and to its own ancestors
  cache      ``cache_write`` / ``cache_read``: the paged cache, bfloat16 or E4M3 with a power-of-two scale per vector
  rope       ``rope_rows``: rotary positions of the block's queries and keys
  score      ``score_tokens``: log probabilities of given tokens, entropy and the likeliest alternatives

``run`` computes them in plain torch operations, or with the package's kernels where ``own`` is set.
"""
import math

import torch

own = False

E8_BIAS = 127      # bias of a scale byte: scale = 2 ** (byte - 127)
E8_TOP = 7         # largest scale exponent, so that 448 * 2 ** 7 bounds what the cache holds
E4M3_MAX = 448.0


# ------------------------------------------------------------------------------------------------ the cases
def _attention(name, S, N, width, Hq, Hkv, D, L, spread, page, kv):
    """S sequences, N drafted nodes each (width 0: a random tree, else rows of `width` columns), contexts of
    L - spread .. L tokens, a cache of kv type in pages of `page` tokens."""
    return {"name": name, "op": "attention", "S": S, "N": N, "width": width, "Hq": Hq, "Hkv": Hkv, "D": D, "L": L, "spread": spread, "page": page, "kv": kv}


def listed():
    return [
        # plain decoding of one sequence: one token, the latency of a call
        _attention("attention-token", 1, 1, 1, 32, 8, 128, 4095, 0, 64, "bf16"),
        # a decode step of a 7B-shaped model (one key head for each query head): 8 draft rows of 1 + 5 columns
        _attention("attention-step", 1, 48, 6, 32, 32, 128, 4096, 0, 64, "bf16"),
        # small heads shared by an odd number of queries, a ragged batch of short contexts, a tree of 23 nodes
        _attention("attention-odd", 8, 23, 0, 14, 2, 64, 777, 700, 32, "bf16"),
        # a serving batch: 64 sequences, 16 rows of 1 + 8 columns, contexts around 2048 tokens, the smallest pages
        _attention("attention-batch", 64, 144, 9, 32, 8, 128, 2048, 512, 16, "e4m3"),
        # long contexts and a small tree: the time to read the cache once
        _attention("attention-long", 4, 37, 0, 32, 8, 128, 131072, 1000, 128, "e4m3"),
        # the widest draft block (64 rows of 1 + 10 columns) over long contexts: bound by the matrix products
        _attention("attention-block", 4, 704, 11, 32, 8, 128, 16384, 300, 64, "bf16"),
        # what a step commits: at most 9 accepted nodes of 144 for each of 64 sequences, quantised, and read back
        {"name": "cache-commit", "op": "cache", "S": 64, "N": 144, "take": 9, "Hkv": 8, "D": 128, "L": 2048, "page": 16, "kv": "e4m3", "rot": 0},
        # prompts written at once with their keys rotated on the way, and read back
        {"name": "cache-prompt", "op": "cache", "S": 8, "N": 4001, "take": 0, "Hkv": 8, "D": 128, "L": 100, "page": 64, "kv": "e4m3", "rot": 128},
        # a decode step's block: 48 tokens, 32 + 32 heads
        {"name": "rope-step", "op": "rope", "T": 48, "Hq": 32, "Hkv": 32, "D": 128, "rot": 128, "interleaved": False, "factor": 1.0, "top": 4096},
        # prompts in a long context: neighbouring pairs, half of each head, positions stretched by 8
        {"name": "rope-prompt", "op": "rope", "T": 32001, "Hq": 32, "Hkv": 8, "D": 128, "rot": 64, "interleaved": True, "factor": 8.0, "top": 131072},
        # a decode step's rows over a vocabulary of 32000: the time to read the head once
        {"name": "score-step", "op": "score", "M": 48, "V": 32000, "d": 4096, "alt": 5},
        # the widest step over a vocabulary of 128256: bound by the matrix product
        {"name": "score-block", "op": "score", "M": 2816, "V": 128256, "d": 4096, "alt": 8},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attention", "attention", "attention", "cache", "rope", "score"])
    if op == "attention":
        while True:
            group, Hkv = rng.choice([1, 2, 4, 7, 8]), rng.choice([1, 2, 4, 8, 32])
            width = rng.choice([0, 0, 1, 4, 6, 9, 11])
            N = _log(rng, 1, 700)
            N = max(1, N // width) * width if width else N
            c = _attention("", _log(rng, 1, 64), N, width, group * Hkv, Hkv, rng.choice([64, 128]), _log(rng, 1, 131072), 0,
                           rng.choice([16, 32, 64, 128]), rng.choice(["bf16", "e4m3"]))
            c["spread"] = rng.randrange(0, c["L"] + 1)
            rows, keys = c["S"] * c["N"] * c["Hq"], c["L"] + c["N"]
            # within the widest block's products, and the long contexts' cache
            if group * Hkv <= 64 and rows * keys <= 1.2e9 and c["S"] * keys * Hkv <= 5e6:
                break
    elif op == "cache":
        N, S = _log(rng, 1, 4000), _log(rng, 1, 64)
        c = {"op": op, "S": min(S, max(1, 32000 // N)), "N": N, "take": rng.choice([0, min(N, rng.randint(1, 17))]), "Hkv": rng.choice([1, 2, 5, 8, 32]),
             "D": rng.choice([64, 128]), "L": _log(rng, 1, 8000), "page": rng.choice([16, 32, 64, 128]), "kv": rng.choice(["bf16", "e4m3"])}
        c["Hkv"] = c["Hkv"] if c["S"] * N <= 8000 else min(8, c["Hkv"])
        c["rot"] = rng.choice([0, 32, 64])
    elif op == "rope":
        D, Hkv = rng.choice([64, 128]), rng.choice([1, 2, 8])
        c = {"op": op, "T": _log(rng, 1, 32000), "Hq": Hkv * rng.choice([1, 3, 4]), "Hkv": Hkv, "D": D, "rot": rng.choice([D // 4, D // 2, D]),
             "interleaved": rng.random() < 0.5, "factor": rng.choice([1.0, 4.0]), "top": rng.choice([100, 4096, 131072])}
    else:
        V = _log(rng, 500, 128256)
        c = {"op": op, "M": _log(rng, 1, 2816), "V": V, "d": rng.choice([128, 1000, 2048, 4096]), "alt": rng.choice([0, 1, 5, 8, 20])}
    c.pop("name", None)
    return c


# ------------------------------------------------------------------------------------------------ inputs
def _lens(S, L, spread):
    """Context lengths: a fixed ragged pattern, the first sequence the longest."""
    return [L - (s * 7919) % (spread + 1) for s in range(S)]


def _parents(S, N, width, g):
    """[S, N] parent node, -1 for a root: rows of `width` columns, each a chain, or random trees with short branches."""
    j = torch.arange(N)
    if width:
        return torch.where(j % width == 0, -1, j - 1).expand(S, N).contiguous()
    back = torch.minimum(1 + (torch.rand(S, N, generator=g) ** 3 * 8).long(), j.clamp(min=1))
    return torch.where(j == 0, -1, j - back)


def _mask_words(parent):
    """Ancestors of each node, itself included, 32 to a word: [S, N, ceil(N / 32)] int32."""
    S, N = parent.shape
    bits = torch.zeros(S, N, (N + 31) // 32 * 32, dtype=torch.bool, device=parent.device)
    at = torch.arange(N, device=parent.device).expand(S, N).clone()
    rows, nodes = torch.arange(S, device=parent.device)[:, None], torch.arange(N, device=parent.device)[None]
    while bool((at >= 0).any()):
        ok = at >= 0
        bits[rows.expand(S, N)[ok], nodes.expand(S, N)[ok], at[ok]] = True
        at = torch.where(ok, parent.gather(1, at.clamp(min=0)), at)
    words = (bits.view(S, N, -1, 32).long() << torch.arange(32, device=bits.device)).sum(-1)
    return torch.where(words >= 1 << 31, words - (1 << 32), words).int()


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _quantise(x):
    """[..., D] -> E4M3 codes (uint8) and the scale byte of each vector (uint8): the smallest power of two that brings
    the largest magnitude to at most 448."""
    x = x.float()
    amax = x.abs().amax(-1).clamp(max=E4M3_MAX * 2.0 ** E8_TOP)
    m, e = torch.frexp(amax / E4M3_MAX)
    e = torch.where(m == 0.5, e - 1, e).clamp(min=-120, max=E8_TOP)
    e = torch.where(amax > 0, e, torch.zeros_like(e))
    y = torch.ldexp(x, -e[..., None]).clamp(-E4M3_MAX, E4M3_MAX)
    return y.to(torch.float8_e4m3fn).view(torch.uint8), (e + E8_BIAS).to(torch.uint8)


def _dequantise(codes, scale):
    return codes.view(torch.float8_e4m3fn).float() * torch.exp2(scale.float() - E8_BIAS)[..., None]


def _cache(g, S, tokens, Hkv, D, page, kv):
    """A paged cache with room for `tokens` positions of each sequence, its pages handed out in no order."""
    per = max(1, -(-tokens // page))
    k, v = (_randn(g, S * per, Hkv, page, D).bfloat16() for _ in range(2))
    table = torch.randperm(S * per, generator=g, device="cuda").int().view(S, per)
    if kv == "bf16":
        return {"k": k, "v": v, "table": table}
    (k, ks), (v, vs) = _quantise(k), _quantise(v)
    return {"k": k, "v": v, "table": table, "k_exp": ks, "v_exp": vs}


def _handle(V=64, d=64, weight=None):
    """The context that a program keeps for its head."""
    import paper_2411_03786_b200 as ngs
    w = torch.zeros(V, d, dtype=torch.bfloat16, device="cuda") if weight is None else weight
    return ngs.SpecContext(w, w)


def _frequencies(rot, factor, base=10000.0):
    """Rotation per position of each pair, positions stretched by `factor`."""
    return (base ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot) / factor).float().cuda()


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    host = torch.Generator().manual_seed(seed)
    c, s = case, {"case": case}
    if c["op"] == "attention":
        s["lens_host"] = _lens(c["S"], c["L"], c["spread"])
        s["lens"] = torch.tensor(s["lens_host"], dtype=torch.int32, device="cuda")
        s["cache"] = _cache(g, c["S"], c["L"], c["Hkv"], c["D"], c["page"], c["kv"])
        # the block's projections as one matrix product leaves them: queries, keys and values side by side
        qkv = _randn(g, c["S"], c["N"], c["Hq"] + 2 * c["Hkv"], c["D"]).bfloat16()
        qkv[:, :, :c["Hq"]] *= 2.0  # scores of standard deviation 2: some keys weigh much more than others
        s["q"], s["k"], s["v"] = qkv[:, :, :c["Hq"]], qkv[:, :, c["Hq"]:c["Hq"] + c["Hkv"]], qkv[:, :, c["Hq"] + c["Hkv"]:]
        s["mask"] = _mask_words(_parents(c["S"], c["N"], c["width"], host).cuda())
    elif c["op"] == "cache":
        n = c["take"] or c["N"]
        s["cache"] = _cache(g, c["S"], c["L"] + n, c["Hkv"], c["D"], c["page"], c["kv"])
        s["start"] = torch.tensor(_lens(c["S"], c["L"], c["L"] // 2), dtype=torch.int32, device="cuda")
        kv = _randn(g, c["S"], c["N"], 2 * c["Hkv"], c["D"])
        kv = (kv * torch.exp(_randn(g, c["S"], c["N"], 2 * c["Hkv"], 1))).bfloat16()
        s["k"], s["v"] = kv[:, :, :c["Hkv"]], kv[:, :, c["Hkv"]:]
        s["count"] = torch.tensor([n - (i * 31) % min(n, 9) for i in range(c["S"])], dtype=torch.int32, device="cuda")
        s["nodes"] = None
        if c["take"]:  # the accepted nodes: a run inside the block
            first = torch.randint(0, c["N"] - n + 1, (c["S"], 1), generator=host)
            s["nodes"] = (first + torch.arange(n)).int().cuda()
        s["freq"] = _frequencies(c["rot"], 1.0) if c["rot"] else None
    elif c["op"] == "rope":
        qk = _randn(g, c["T"], c["Hq"] + c["Hkv"], c["D"]).bfloat16()
        s["q"], s["k"] = qk[:, :c["Hq"]], qk[:, c["Hq"]:]
        s["pos"] = torch.randint(0, c["top"], (c["T"],), generator=g, device="cuda").int()
        s["freq"] = _frequencies(c["rot"], c["factor"])
        s["gain"] = 1.0 + 0.1 * math.log(c["factor"])
    else:
        # activations and weights on a grid (1/16 and 1/1024): every order of summation gives the same logits, so that
        # the ids of the alternatives depend on the values alone
        s["hidden"] = (_randn(g, c["M"], c["d"]).clamp(-7, 7) * 16).round().div(16).bfloat16()
        s["weight"] = (_randn(g, c["V"], c["d"]).clamp(-6, 6).mul_(0.02 * 1024)).round_().div_(1024).bfloat16()
        s["tokens"] = torch.randint(0, c["V"], (c["M"],), generator=g, device="cuda").int()
    if own:
        s["ctx"] = _handle(c["V"], c["d"], s["weight"]) if c["op"] == "score" else _handle()
        import paper_2411_03786_b200 as ngs
        if "cache" in s:
            s["handle"] = ngs.KVCache(**s["cache"])
        if s.get("freq") is not None:
            s["rope"] = ngs.Rope(s["freq"], interleaved=bool(c.get("interleaved", False)), scale=s.get("gain", 1.0))
    return s


# ------------------------------------------------------------------------------------------------ the plain forms
def _positions(cache, at):
    """Page and slot of the positions `at` [S, n]."""
    page = cache["k"].shape[2]
    return cache["table"].gather(1, (at // page).long()).long(), (at % page).long()


def _gather(cache, at):
    """Keys and values at positions `at` [S, n] as float32 [S, n, Hkv, D]."""
    p, o = _positions(cache, at)
    k, v = cache["k"][p, :, o], cache["v"][p, :, o]
    if "k_exp" in cache:
        return _dequantise(k, cache["k_exp"][p, :, o]), _dequantise(v, cache["v_exp"][p, :, o])
    return k.float(), v.float()


def _rotate(x, pos, freq, interleaved, gain):
    """Rotates the first 2 * len(freq) elements of each head of x [..., heads, D] at positions pos [...]."""
    x, h = x.float(), freq.numel()
    a = pos.float()[..., None, None] * freq
    cos, sin = a.cos() * gain, a.sin() * gain
    r = x[..., : 2 * h]
    x0, x1 = (r[..., 0::2], r[..., 1::2]) if interleaved else (r[..., :h], r[..., h:])
    y0, y1 = x0 * cos - x1 * sin, x0 * sin + x1 * cos
    y = torch.stack([y0, y1], -1).flatten(-2) if interleaved else torch.cat([y0, y1], -1)
    return torch.cat([y, x[..., 2 * h:]], -1).bfloat16()


def _plain_attention(s):
    c, dev = s["case"], s["q"].device
    S, N, Hkv, D, G, L = c["S"], c["N"], c["Hkv"], c["D"], c["Hq"] // c["Hkv"], c["L"]
    kc, vc = _gather(s["cache"], torch.arange(L, device=dev).expand(S, L))
    k, v = torch.cat([kc, s["k"].float()], 1).transpose(1, 2), torch.cat([vc, s["v"].float()], 1).transpose(1, 2)
    q = s["q"].float().reshape(S, N, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(S, Hkv, N * G, D)
    score = (q @ k.transpose(2, 3)).view(S, Hkv, N, G, L + N) * D ** -0.5
    seen = torch.zeros(S, N, L + N, dtype=torch.bool, device=dev)
    seen[:, :, :L] = (torch.arange(L, device=dev) < s["lens"][:, None])[:, None]
    seen[:, :, L:] = ((s["mask"][..., None] >> torch.arange(32, device=dev)) & 1).bool().flatten(2)[:, :, :N]
    score.masked_fill_(~seen[:, None, :, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    score.sub_(top).exp_()
    total = score.sum(-1, keepdim=True)
    out = (score.view(S, Hkv, N * G, L + N) @ v).view(S, Hkv, N, G, D) / total
    lse = (top + total.log()).squeeze(-1)
    return out.permute(0, 2, 1, 3, 4).reshape(S, N, Hkv * G, D).bfloat16(), lse.permute(0, 2, 1, 3).reshape(S, N, Hkv * G)


def _plain_cache(s):
    c, dev = s["case"], s["k"].device
    n = c["take"] or c["N"]
    k, v = s["k"], s["v"]
    if s["nodes"] is not None:
        rows = torch.arange(c["S"], device=dev)[:, None]
        k, v = k[rows, s["nodes"].long()], v[rows, s["nodes"].long()]
    step = torch.arange(n, device=dev)
    at = s["start"][:, None] + step
    if s["freq"] is not None:
        k = _rotate(k, at, s["freq"], False, 1.0)
    keep = step < s["count"][:, None]
    p, o = (t[keep] for t in _positions(s["cache"], at))
    cache = s["cache"]
    if "k_exp" in cache:
        (k, ks), (v, vs) = _quantise(k[keep]), _quantise(v[keep])
        cache["k"][p, :, o], cache["k_exp"][p, :, o], cache["v"][p, :, o], cache["v_exp"][p, :, o] = k, ks, v, vs
    else:
        cache["k"][p, :, o], cache["v"][p, :, o] = k[keep], v[keep]
    k, v = _gather(cache, at)
    return torch.where(keep[..., None, None], k, 0).bfloat16(), torch.where(keep[..., None, None], v, 0).bfloat16()


def _plain_score(s):
    z = s["hidden"].float() @ s["weight"].float().T
    top = z.amax(-1, keepdim=True)
    lse = top + (z - top).exp().sum(-1, keepdim=True).log()
    z -= lse  # log probabilities
    logp = z.gather(1, s["tokens"].long()[:, None])[:, 0]
    entropy = -(z.exp() * z).sum(-1)
    if not s["case"]["alt"]:
        return logp, entropy
    value, index = torch.sort(z, dim=-1, descending=True, stable=True)
    return logp, entropy, index[:, : s["case"]["alt"]].int(), value[:, : s["case"]["alt"]].clone()


def run(s):
    c = s["case"]
    if c["op"] == "attention":
        if own:
            return s["ctx"].tree_attention(s["handle"], s["q"], s["k"], s["v"], s["mask"], s["lens"], with_lse=True)
        return _plain_attention(s)
    if c["op"] == "cache":
        if own:
            s["ctx"].cache_write(s["handle"], s["k"], s["v"], s["start"], count=s["count"], nodes=s["nodes"], rope=s.get("rope"))
            return s["ctx"].cache_read(s["handle"], s["start"], c["take"] or c["N"], count=s["count"])
        return _plain_cache(s)
    if c["op"] == "rope":
        if own:
            return s["ctx"].rope_rows(s["rope"], s["q"], s["k"], s["pos"])
        return tuple(_rotate(x, s["pos"], s["freq"], c["interleaved"], s["gain"]) for x in (s["q"], s["k"]))
    if own:
        return tuple(t for t in s["ctx"].score_tokens(s["hidden"], s["tokens"], n_alt=c["alt"]) if t is not None)
    return _plain_score(s)


# ------------------------------------------------------------------------------------------------ bytes and operations
def work(case):
    c = case
    if c["op"] == "attention":
        lens = _lens(c["S"], c["L"], c["spread"])
        own_keys = (c["width"] + 1) / 2 if c["width"] else min(c["N"], 8)  # ancestors of a node, about
        element = 2 if c["kv"] == "bf16" else 1 + 1 / c["D"]
        flops = 4.0 * c["D"] * c["Hq"] * c["N"] * sum(n + own_keys for n in lens)
        return {"bytes": 2 * element * c["Hkv"] * c["D"] * sum(lens) + c["S"] * c["N"] * c["D"] * (4 * c["Hq"] + 4 * c["Hkv"]) + 4 * c["S"] * c["N"] * c["Hq"], "flops": flops}
    if c["op"] == "cache":
        n = c["S"] * (c["take"] or c["N"]) * 2 * c["Hkv"] * c["D"]
        element = 2 if c["kv"] == "bf16" else 1 + 1 / c["D"]
        return {"bytes": n * (2 + element + element + 2), "flops": 4.0 * n}
    if c["op"] == "rope":
        n = c["T"] * (c["Hq"] + c["Hkv"]) * c["D"]
        return {"bytes": 4.0 * n + 4 * c["T"], "flops": 3.0 * n}
    return {"bytes": 2.0 * c["V"] * c["d"] + 2.0 * c["M"] * c["d"] + c["M"] * (12 + 8 * c["alt"]), "flops": 2.0 * c["M"] * c["V"] * c["d"]}


# ------------------------------------------------------------------------------------------------ 64 bits
def _codes64():
    """The 256 values of E4M3: sign, four exponent bits (bias 7), three mantissa bits."""
    b = torch.arange(256)
    e, m = (b >> 3) & 15, (b & 7).double()
    v = torch.where(e == 0, m * 2.0 ** -9, (1 + m / 8) * torch.exp2(e.double() - 7))
    v = torch.where((b & 127) == 127, torch.full_like(v, math.nan), v)
    return torch.where(b >= 128, -v, v).cuda()


def _held64(store, exp, table, n):
    """The first n positions of one sequence: [heads, n, D] in 64 bits."""
    x = store[table.long()]  # pages, heads, page, D
    x = x.double() if exp is None else _codes64()[x.long()] * torch.exp2(exp[table.long()].double() - 127)[..., None]
    return x.transpose(0, 1).flatten(1, 2)[:, :n]


def _held_as64(x):
    """The nearest values that 8 bits and a power of two hold, halves to the even one."""
    top = x.abs().amax(-1, keepdim=True)
    scale = torch.exp2(torch.ceil(torch.log2(top / 448)).clamp(-120, 7))
    y = x / torch.where(top > 0, scale, 1.0)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return (torch.round(y / step) * step).clamp(-448, 448) * scale


def _turn64(x, pos, freq, interleaved, gain):
    """Rotation as a complex product: (x0 + i x1) * gain * exp(i pos freq)."""
    x, h = x.double(), freq.numel()
    r = x[..., : 2 * h].unflatten(-1, (h, 2)) if interleaved else x[..., : 2 * h].unflatten(-1, (2, h)).transpose(-1, -2)
    w = torch.polar(torch.full_like(pos, gain, dtype=torch.float64)[..., None], pos.double()[..., None] * freq.double())
    z = torch.view_as_real(torch.view_as_complex(r.contiguous()) * w[..., None, :])
    z = z.flatten(-2) if interleaved else z.transpose(-1, -2).flatten(-2)
    return torch.cat([z, x[..., 2 * h:]], -1)


def exact(case, seed):
    s, c = prepare(case, seed), case
    if c["op"] == "attention":
        if c["S"] * c["N"] * c["Hq"] * (c["L"] + c["N"]) * c["D"] > 4e11:
            return None
        G, t = c["Hq"] // c["Hkv"], s["cache"]
        out, lse = [], []
        for i, n in enumerate(s["lens_host"]):
            k, v = (_held64(t[x], t.get(x + "_exp"), t["table"][i], n) for x in "kv")
            word = s["mask"][i].long()
            own_keys = torch.stack([(word >> b) & 1 for b in range(32)], -1).flatten(1)[:, : c["N"]].bool()
            hidden = torch.cat([torch.zeros(c["N"], n, dtype=torch.bool, device="cuda"), ~own_keys], 1)
            o, l = [], []
            for h in range(c["Hq"]):
                kh, vh = torch.cat([k[h // G], s["k"][i, :, h // G].double()]), torch.cat([v[h // G], s["v"][i, :, h // G].double()])
                z = (s["q"][i, :, h].double() @ kh.T / math.sqrt(c["D"])).masked_fill(hidden, -math.inf)
                l.append(torch.logsumexp(z, -1))
                o.append(torch.exp(z - l[-1][:, None]) @ vh)
            out.append(torch.stack(o, 1))
            lse.append(torch.stack(l, 1))
        return torch.stack(out), torch.stack(lse)
    if c["op"] == "cache":
        k, v, n = s["k"], s["v"], c["take"] or c["N"]
        if s["nodes"] is not None:
            k, v = (torch.stack([x[i, s["nodes"][i].long()] for i in range(c["S"])]) for x in (k, v))
        step = torch.arange(n, device="cuda")
        k = k.double() if s["freq"] is None else _turn64(k, s["start"][:, None] + step, s["freq"], False, 1.0)
        keep = (step < s["count"][:, None])[..., None, None]
        if c["kv"] == "bf16":
            return k * keep, v.double() * keep
        return _held_as64(k.bfloat16().double()) * keep, _held_as64(v.double()) * keep
    if c["op"] == "rope":
        return tuple(_turn64(x, s["pos"], s["freq"], c["interleaved"], s["gain"]) for x in (s["q"], s["k"]))
    logp, entropy, value = [], [], []
    for rows, tok in zip(s["hidden"].split(256), s["tokens"].split(256)):
        z = torch.cat([rows.double() @ w.double().T for w in s["weight"].split(8192)], 1)
        p = torch.log_softmax(z, -1)
        logp.append(p[torch.arange(len(tok)), tok.long()])
        entropy.append(torch.special.entr(p.exp()).sum(-1))
        value.append(p.topk(c["alt"], -1).values if c["alt"] else p[:, :0])
    return (torch.cat(logp), torch.cat(entropy)) + ((None, torch.cat(value)) if c["alt"] else ())
