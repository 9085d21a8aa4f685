"""The operators around a cache of 4 bits and its pages, as cases that can be timed and compared.

  attention  ``tree_attention`` over a paged cache of E2M1 codes, a scale byte for each 16 of them
  cache      ``cache_write`` / ``cache_read`` of that cache; of a bfloat16 cache with keys rotated along several axes
  rope       ``rope_rows`` with an axis for each pair: time, height and width of images and video
  pages      ``pages_assign`` / ``pages_reserve`` / ``pages_compact``: forking, extending, freeing and moving together

``run`` computes them in plain torch operations, or with the package's kernels where ``own`` is set.
"""
import math

import torch

own = False

TOP_SCALE = 226  # the largest scale byte, 10240: a code times it stays within half precision


# ------------------------------------------------------------------------------------------------ the cases
def _attention(name, S, N, width, Hq, Hkv, D, L, spread, page):
    """S sequences, N drafted nodes each (width 0: a random tree, else rows of `width` columns), contexts of
    L - spread .. L tokens in pages of `page` tokens."""
    return {"name": name, "op": "attention", "S": S, "N": N, "width": width, "Hq": Hq, "Hkv": Hkv, "D": D, "L": L, "spread": spread, "page": page}


def _pages(name, kind, S, group, L, n, layers, Hkv, D, page, kv):
    return {"name": name, "op": "pages", "kind": kind, "S": S, "group": group, "L": L, "n": n, "layers": layers, "Hkv": Hkv, "D": D, "page": page, "kv": kv}


def listed():
    return [
        # plain decoding of one sequence: one token, the latency of a call
        _attention("attention4-token", 1, 1, 1, 32, 8, 128, 4095, 0, 64),
        # small heads shared by an odd number of queries, a ragged batch of short contexts, a tree of 23 nodes
        _attention("attention4-odd", 8, 23, 0, 14, 2, 64, 777, 700, 32),
        # plain decoding of a serving batch: the time to read the cache once, from the smallest pages
        _attention("attention4-decode", 64, 1, 1, 32, 8, 128, 8192, 2048, 16),
        # the same batch verifying 16 rows of 1 + 8 columns over shorter contexts
        _attention("attention4-batch", 64, 144, 9, 32, 8, 128, 2048, 512, 16),
        # long contexts and a small tree
        _attention("attention4-long", 4, 37, 0, 32, 8, 128, 131072, 1000, 128),
        # the widest draft block (64 rows of 1 + 10 columns) over long contexts: bound by the matrix products
        _attention("attention4-block", 4, 704, 11, 32, 8, 128, 16384, 300, 64),
        # what a step commits: at most 9 accepted nodes of 144 for each of 64 sequences, written and read back
        {"name": "cache4-commit", "op": "cache", "S": 64, "N": 144, "take": 9, "Hkv": 8, "D": 128, "L": 2048, "page": 16, "kv": "e2m1", "axes": 0},
        # prompts written at once, and read back
        {"name": "cache4-prompt", "op": "cache", "S": 8, "N": 4001, "take": 0, "Hkv": 8, "D": 128, "L": 100, "page": 64, "kv": "e2m1", "axes": 0},
        # a decode step's block behind images: 48 tokens, 28 + 4 heads, three axes in sections
        {"name": "rope3-step", "op": "rope", "T": 48, "Hq": 28, "Hkv": 4, "D": 128, "rot": 128, "interleaved": False, "axes": 3, "mixed": False},
        # prompts of text and video frames: the axes dealt out in turn
        {"name": "rope3-prompt", "op": "rope", "T": 32001, "Hq": 28, "Hkv": 4, "D": 128, "rot": 128, "interleaved": False, "axes": 3, "mixed": True},
        # four prompts, eight samples of each: the samples take the prompt's pages and get pages of their own for the next block
        _pages("pages-fork", "fork", 36, 8, 1000, 11, 4, 8, 128, 64, "e2m1"),
        # a pool of 64 sequences of which the older half has ended: the others move to the front, new prompts get what is free
        _pages("pages-compact", "slide", 64, 0, 4100, 0, 16, 8, 128, 16, "e2m1"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attention", "attention", "attention", "cache", "rope", "pages"])
    if op == "attention":
        while True:
            group, Hkv = rng.choice([1, 2, 4, 7, 8, 16]), rng.choice([1, 2, 4, 8, 32])
            width = rng.choice([0, 0, 1, 4, 6, 9, 11])
            N = rng.choice([1, _log(rng, 1, 700)])
            N = max(1, N // width) * width if width else N
            c = _attention("", _log(rng, 1, 64), N, width, group * Hkv, Hkv, rng.choice([64, 128]), _log(rng, 1, 131072), 0, rng.choice([16, 32, 64, 128]))
            c["spread"] = rng.randrange(0, c["L"] + 1)
            rows, keys = c["S"] * c["N"] * c["Hq"], c["L"] + c["N"]
            # within the widest block's products, and the long contexts' cache
            if group * Hkv <= 64 and rows * keys <= 1.2e9 and c["S"] * keys * Hkv <= 4.5e6:
                break
    elif op == "cache":
        N, S = _log(rng, 1, 4000), _log(rng, 1, 64)
        c = {"op": op, "S": min(S, max(1, 32000 // N)), "N": N, "take": rng.choice([0, min(N, rng.randint(1, 17))]), "Hkv": rng.choice([1, 2, 5, 8, 32]),
             "D": rng.choice([64, 128]), "L": _log(rng, 1, 8000), "page": rng.choice([16, 32, 64, 128])}
        c["Hkv"] = c["Hkv"] if c["S"] * N <= 8000 else min(8, c["Hkv"])
        c["axes"] = rng.choice([0, 0, 2, 3])
        c["kv"] = "bf16" if c["axes"] else "e2m1"
    elif op == "rope":
        D, Hkv = rng.choice([64, 80, 128]), rng.choice([1, 2, 8])
        c = {"op": op, "T": _log(rng, 1, 32000), "Hq": Hkv * rng.choice([1, 3, 4]), "Hkv": Hkv, "D": D, "rot": rng.choice([D // 32 * 16, D]),
             "interleaved": rng.random() < 0.5, "axes": rng.choice([2, 3]), "mixed": rng.random() < 0.5}
    else:
        kind = rng.choice(["fork", "slide"])
        group = rng.randint(1, 12) if kind == "fork" else 0
        S = rng.randint(1, 6) * (1 + group) if kind == "fork" else 2 * _log(rng, 1, 32)
        layers = _log(rng, 1, 16)
        c = _pages("", kind, S, group, _log(rng, 1, min(8000, 4000000 // (S * layers))), _log(rng, 1, 300), layers, rng.choice([1, 2, 8]), rng.choice([64, 128]),
                   rng.choice([16, 32, 64, 128]), rng.choice(["bf16", "e2m1", "e2m1"]))
        if c["kv"] == "bf16":
            c["layers"] = max(1, layers // 4)
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


def _scales(dev):
    """What the 256 scale bytes stand for: the upper byte of a half-precision number without its sign; NaN beyond the largest."""
    s = (torch.arange(256, dtype=torch.int16, device=dev) << 7).view(torch.float16).float()
    s[TOP_SCALE + 1:] = math.nan
    return s


def _values(dev):
    v = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=dev)
    return torch.cat([v, -v])


def _quantise(x):
    """[..., D] -> codes (uint8 [..., D / 2], the even element in the low half) and scale bytes (uint8 [..., D / 16]): the
    smallest scale that brings the 16 magnitudes to at most 6, the code nearest to x / scale, halves to the even code."""
    x = x.float().unflatten(-1, (-1, 16))
    top = x.abs().amax(-1)
    scales = _scales(x.device)
    byte = torch.searchsorted(scales[: TOP_SCALE + 1] * 6, top.clamp(max=6 * 10240.0).contiguous())
    s = scales[byte][..., None]
    # (the borders between neighbouring codes, times a scale, are exact in 32 bits; a border itself goes to the even code)
    a, code = x.abs(), torch.zeros_like(x, dtype=torch.uint8)
    for i, border in enumerate((0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)):
        code += (a >= border * s) if i % 2 else (a > border * s)
    code = torch.where(s > 0, code, 0) + 8 * torch.signbit(x).byte()
    nan = x.isnan().any(-1)
    code, byte = torch.where(nan[..., None], 0, code).flatten(-2), torch.where(nan, 255, byte)
    return code[..., 0::2] + 16 * code[..., 1::2], byte.to(torch.uint8)


def _dequantise(codes, scale):
    code = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
    v = _values(codes.device)[code.long()].unflatten(-1, (-1, 16))
    return (v * _scales(codes.device)[scale.long()][..., None]).flatten(-2)


def _cache(g, S, tokens, Hkv, D, page, kv):
    """A paged cache with room for `tokens` positions of each sequence, its pages handed out in no order; some channels of
    the keys are larger than others."""
    per = max(1, -(-tokens // page))
    table = torch.randperm(S * per, generator=g, device="cuda").int().view(S, per)
    gain = torch.exp(0.5 * _randn(g, Hkv, 1, D))
    parts = {"k": [], "v": [], "k_scale": [], "v_scale": []}
    step = max(1, (1 << 26) // (Hkv * page * D))
    for at in range(0, S * per, step):
        for name in "kv":
            x = _randn(g, min(step, S * per - at), Hkv, page, D)
            x = (x * gain if name == "k" else x).bfloat16()
            if kv == "bf16":
                parts[name].append(x)
            else:
                codes, scale = _quantise(x)
                parts[name].append(codes)
                parts[name + "_scale"].append(scale)
    return {"table": table, **{name: torch.cat(p) for name, p in parts.items() if p}}, gain


def _handle():
    """The context that a program keeps."""
    import paper_2411_03786_b200 as ngs
    w = torch.zeros(64, 64, dtype=torch.bfloat16, device="cuda")
    return ngs.SpecContext(w, w)


def _frequencies(rot, base=10000.0):
    return (base ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)).float().cuda()


def _axis(pairs, axes, mixed):
    """The axis that each pair turns by: in sections, the first half as large as the others, or dealt out in turn."""
    if mixed:
        return (torch.arange(pairs) % axes).to(torch.uint8).cuda()
    first = max(1, pairs // (2 * axes - 1))
    rest = (torch.arange(pairs - first) * (axes - 1)) // max(1, pairs - first) + 1
    return torch.cat([torch.zeros(first, dtype=torch.long), rest]).to(torch.uint8).cuda()


def _coordinates(T, axes, host):
    """[axes, T] positions of text, where all axes go on together, and images and frames, whose tokens have the coordinates
    of a grid behind the text."""
    parts, at, have = [], 0, 0
    while have < T:
        n = int(torch.randint(1, 400, (1,), generator=host))
        parts.append((at + torch.arange(n)).expand(axes, n))
        at, have = at + n, have + n
        size = [int(x) for x in torch.randint(1, 40, (axes,), generator=host)]
        size[0] = 1 + size[0] % 4
        grid = torch.stack(torch.meshgrid(*[torch.arange(x) for x in size], indexing="ij")).flatten(1)
        parts.append(at + grid)
        at, have = at + max(size), have + grid.shape[1]
    return torch.cat(parts, 1)[:, :T].int().contiguous().cuda()


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    host = torch.Generator().manual_seed(seed)
    c, s = case, {"case": case}
    if c["op"] == "attention":
        s["lens_host"] = _lens(c["S"], c["L"], c["spread"])
        s["lens"] = torch.tensor(s["lens_host"], dtype=torch.int32, device="cuda")
        s["cache"], gain = _cache(g, c["S"], c["L"], c["Hkv"], c["D"], c["page"], "e2m1")
        # the block's projections as one matrix product leaves them: queries, keys and values side by side
        qkv = _randn(g, c["S"], c["N"], c["Hq"] + 2 * c["Hkv"], c["D"]).bfloat16()
        # scores of standard deviation about 2: some keys weigh much more than others
        qkv[:, :, :c["Hq"]] *= 2.0 / float(gain.square().mean().sqrt())
        qkv[:, :, c["Hq"]:c["Hq"] + c["Hkv"]] *= gain[:, 0]
        s["q"], s["k"], s["v"] = qkv[:, :, :c["Hq"]], qkv[:, :, c["Hq"]:c["Hq"] + c["Hkv"]], qkv[:, :, c["Hq"] + c["Hkv"]:]
        s["mask"] = _mask_words(_parents(c["S"], c["N"], c["width"], host).cuda())
    elif c["op"] == "cache":
        n = c["take"] or c["N"]
        s["cache"], gain = _cache(g, c["S"], c["L"] + n, c["Hkv"], c["D"], c["page"], c["kv"])
        s["start"] = torch.tensor(_lens(c["S"], c["L"], c["L"] // 2), dtype=torch.int32, device="cuda")
        kv = _randn(g, c["S"], c["N"], 2 * c["Hkv"], c["D"])
        kv = (kv * torch.exp(_randn(g, c["S"], c["N"], 2 * c["Hkv"], 1))).bfloat16()
        s["k"], s["v"] = kv[:, :, :c["Hkv"]], kv[:, :, c["Hkv"]:]
        s["count"] = torch.tensor([n - (i * 31) % min(n, 9) for i in range(c["S"])], dtype=torch.int32, device="cuda")
        s["nodes"] = None
        if c["take"]:  # the accepted nodes: a run inside the block
            first = torch.randint(0, c["N"] - n + 1, (c["S"], 1), generator=host)
            s["nodes"] = (first + torch.arange(n)).int().cuda()
        if c["axes"]:
            s["freq"], s["axis"] = _frequencies(c["D"]), _axis(c["D"] // 2, c["axes"], True)
            s["pos"] = _coordinates(c["S"] * c["N"], c["axes"], host).view(c["axes"], c["S"], c["N"])
    elif c["op"] == "rope":
        qk = _randn(g, c["T"], c["Hq"] + c["Hkv"], c["D"]).bfloat16()
        s["q"], s["k"] = qk[:, :c["Hq"]], qk[:, c["Hq"]:]
        s["pos"] = _coordinates(c["T"], c["axes"], host)
        s["freq"], s["axis"] = _frequencies(c["rot"]), _axis(c["rot"] // 2, c["axes"], c["mixed"])
    else:
        _prepare_pages(c, s, g)
    if own:
        import paper_2411_03786_b200 as ngs
        s["ctx"] = _handle()
        if "cache" in s:
            s["handle"] = ngs.KVCache(**s["cache"])
        if s.get("freq") is not None:
            s["rope"] = ngs.Rope(s["freq"], interleaved=bool(c.get("interleaved", False)), axis=s["axis"])
        if "layers" in s:
            s["pool"] = ngs.PagePool([ngs.KVCache(table=s["table"], **{n: x[i] for n, x in s["layers"].items()}) for i in range(c["layers"])], s["refs"])
    return s


def _prepare_pages(c, s, g):
    """A pool in the state that a pass leaves it in, so that every pass does the same work."""
    S, page, lens = c["S"], c["page"], _lens(c["S"], c["L"], c["L"] // 3)
    if c["kind"] == "fork":
        # prompts in the first rows, then the samples of each, whose pages of the last pass are given back first
        P = S // (1 + c["group"])
        parent = [i // c["group"] for i in range(S - P)]
        source, keep = list(range(P)) + parent, lens[:P] + [lens[p] for p in parent]
        start, count = keep, [0] * P + [1 + (i * 5) % c["n"] for i in range(S - P)]
        held = keep
    else:
        # the first half of the rows ends, the second takes its place; as many prompts of the same lengths arrive
        lens = lens[: S // 2] * 2
        source, keep = [s + S // 2 if s < S // 2 else -1 for s in range(S)], [n if s < S // 2 else 0 for s, n in enumerate(lens)]
        start, count = [0] * S, [0 if s < S // 2 else n for s, n in enumerate(lens)]
        held = lens
    need = [-(-(a + b) // page) for a, b in zip(start, count)]
    first, at, rows = [-(-n // page) for n in held], 0, []
    for i in range(S):
        if c["kind"] == "fork" and i >= P:
            rows.append(rows[source[i]])
        else:
            rows.append(list(range(at, at + first[i])))
            at += first[i]
    total = at + sum(need)
    order = torch.randperm(total, generator=g, device="cuda").int()  # prompts lie anywhere in the pool
    width = max(max(need), max(first)) + 1
    table = torch.full((S, width), -1, dtype=torch.int32)
    for i, r in enumerate(rows):
        table[i, : len(r)] = torch.tensor(r, dtype=torch.int32)
    s["table"] = table.cuda()
    if c["kind"] == "fork":
        s["table"] = torch.where(s["table"] >= 0, order[s["table"].long()], -1).int()
    held = s["table"][s["table"] >= 0].long()
    s["refs"] = torch.bincount(held, minlength=total).int()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    s["source"], s["keep"], s["start"], s["count"] = i32(source), i32(keep), i32(start), i32(count)
    shape = (c["layers"], total, c["Hkv"], page)  # all layers share the table
    if c["kv"] == "bf16":
        x = {n: _randn(g, *shape, c["D"]).bfloat16() for n in ("k", "v")}
    else:
        x = {n: torch.randint(0, 256, (*shape, c["D"] // 2), generator=g, device="cuda", dtype=torch.uint8) for n in ("k", "v")}
        x.update({n: torch.randint(100, 130, (*shape, c["D"] // 16), generator=g, device="cuda", dtype=torch.uint8) for n in ("k_scale", "v_scale")})
    s["layers"] = x


# ------------------------------------------------------------------------------------------------ the plain forms
def _positions(cache, at):
    """Page and slot of the positions `at` [S, n]."""
    page = cache["k"].shape[2]
    return cache["table"].gather(1, (at // page).long()).long(), (at % page).long()


def _gather(cache, at):
    """Keys and values at positions `at` [S, n] as float32 [S, n, Hkv, D]."""
    p, o = _positions(cache, at)
    k, v = cache["k"][p, :, o], cache["v"][p, :, o]
    if "k_scale" in cache:
        return _dequantise(k, cache["k_scale"][p, :, o]), _dequantise(v, cache["v_scale"][p, :, o])
    return k.float(), v.float()


def _rotate(x, pos, freq, axis, interleaved):
    """Rotates the first 2 * len(freq) elements of each head of x [..., heads, D]: pair i by pos[axis[i]] * freq[i], the
    angles in 64 bits."""
    x, h = x.float(), freq.numel()
    a = (pos.double()[axis.long()] * freq.double().view(-1, *[1] * (pos.dim() - 1))).movedim(0, -1)[..., None, :]
    cos, sin = a.cos().float(), a.sin().float()
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
    del kc, vc
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
    k, v, pos = s["k"], s["v"], s.get("pos")
    if s["nodes"] is not None:
        rows = torch.arange(c["S"], device=dev)[:, None]
        k, v = k[rows, s["nodes"].long()], v[rows, s["nodes"].long()]
        pos = None if pos is None else pos[:, rows, s["nodes"].long()]
    step = torch.arange(n, device=dev)
    at = s["start"][:, None] + step
    if pos is not None:
        k = _rotate(k, pos, s["freq"], s["axis"], False)
    keep = step < s["count"][:, None]
    p, o = (t[keep] for t in _positions(s["cache"], at))
    cache = s["cache"]
    if "k_scale" in cache:
        (k, ks), (v, vs) = _quantise(k[keep]), _quantise(v[keep])
        cache["k"][p, :, o], cache["k_scale"][p, :, o], cache["v"][p, :, o], cache["v_scale"][p, :, o] = k, ks, v, vs
    else:
        cache["k"][p, :, o], cache["v"][p, :, o] = k[keep], v[keep]
    k, v = _gather(cache, at)
    return torch.where(keep[..., None, None], k, 0).bfloat16(), torch.where(keep[..., None, None], v, 0).bfloat16()


def _plain_assign(s):
    """Row i of the table becomes the pages of row source[i] that its first keep[i] positions lie in."""
    table, refs, page = s["table"], s["refs"], s["case"]["page"]
    new = torch.where((s["source"] >= 0)[:, None], table[s["source"].long().clamp(min=0)], -1)
    index = torch.arange(table.shape[1], device=table.device)
    new = torch.where(index * page < s["keep"][:, None], new, -1)
    refs += torch.bincount(new[new >= 0], minlength=refs.numel()) - torch.bincount(table[table >= 0], minlength=refs.numel())
    table.copy_(new)


def _move(s, src, dst):
    for x in s["layers"].values():
        for layer in x:
            layer[dst] = layer[src]


def _plain_reserve(s):
    """Pages of their own for positions start .. start + count: the lowest free ones, in the order of rows and positions.
    A shared page is copied.  Rows are served until one needs more than is left."""
    table, refs, page = s["table"], s["refs"], s["case"]["page"]
    start, end = s["start"][:, None], (s["start"] + s["count"])[:, None]
    index = torch.arange(table.shape[1], device=table.device)
    mine = (table >= 0) & (refs[table.long().clamp(min=0)] == 1)
    need = (index >= start // page) & (index * page < end) & (end > start) & ~mine
    demand = need.sum(1)
    free = (refs == 0).nonzero().flatten()
    ok = (demand == 0) | (demand.cumsum(0) <= free.numel())
    rows, cols = (need & ok[:, None]).nonzero(as_tuple=True)
    old, new = table[rows, cols].long(), free[: rows.numel()]
    shared = old >= 0
    _move(s, old[shared], new[shared])
    refs -= torch.bincount(old[shared], minlength=refs.numel())
    refs[new] = 1
    table[rows, cols] = new.int()
    return ok.int()


def _plain_compact(s):
    """Pages that are held move to the front: the lowest of those behind it to the lowest free one, and so on."""
    table, refs = s["table"], s["refs"]
    live = refs > 0
    n = live.sum()
    index = torch.arange(refs.numel(), device=refs.device)
    src, dst = (live & (index >= n)).nonzero().flatten(), (~live & (index < n)).nonzero().flatten()
    _move(s, src, dst)
    now = index.clone()
    now[src] = dst
    refs[dst] = refs[src]
    refs[src] = 0
    table.copy_(torch.where(table >= 0, now[table.long().clamp(min=0)].int(), table))
    return n.int().view(1)


def _plain_pages(s):
    _plain_assign(s)
    n = _plain_compact(s) if s["case"]["kind"] == "slide" else None
    return n, _plain_reserve(s)


def run(s):
    c = s["case"]
    if c["op"] == "attention":
        if own:
            return s["ctx"].tree_attention(s["handle"], s["q"], s["k"], s["v"], s["mask"], s["lens"], with_lse=True)
        return _plain_attention(s)
    if c["op"] == "cache":
        if own:
            s["ctx"].cache_write(s["handle"], s["k"], s["v"], s["start"], count=s["count"], nodes=s["nodes"], rope=s.get("rope"), pos=s.get("pos"))
            return s["ctx"].cache_read(s["handle"], s["start"], c["take"] or c["N"], count=s["count"])
        return _plain_cache(s)
    if c["op"] == "rope":
        if own:
            return s["ctx"].rope_rows(s["rope"], s["q"], s["k"], s["pos"])
        return tuple(_rotate(x, s["pos"], s["freq"], s["axis"], c["interleaved"]) for x in (s["q"], s["k"]))
    if own:
        s["ctx"].pages_assign(s["pool"], s["source"], s["keep"])
        n = s["ctx"].pages_compact(s["pool"]) if c["kind"] == "slide" else None
        ok = s["ctx"].pages_reserve(s["pool"], s["start"], s["count"])
    else:
        n, ok = _plain_pages(s)
    return [s["table"], s["refs"], ok] + ([] if n is None else [n]) + list(s["layers"].values())


# ------------------------------------------------------------------------------------------------ bytes and operations
def _element(kv):
    return 2.0 if kv == "bf16" else 0.5 + 1 / 16


def work(case):
    c = case
    if c["op"] == "attention":
        lens = _lens(c["S"], c["L"], c["spread"])
        own_keys = (c["width"] + 1) / 2 if c["width"] else min(c["N"], 8)  # ancestors of a node, about
        flops = 4.0 * c["D"] * c["Hq"] * c["N"] * sum(n + own_keys for n in lens)
        return {"bytes": 2 * _element("e2m1") * c["Hkv"] * c["D"] * sum(lens) + c["S"] * c["N"] * c["D"] * (4 * c["Hq"] + 4 * c["Hkv"]) + 4 * c["S"] * c["N"] * c["Hq"],
                "flops": flops}
    if c["op"] == "cache":
        n = c["S"] * (c["take"] or c["N"]) * 2 * c["Hkv"] * c["D"]
        return {"bytes": n * (4 + 2 * _element(c["kv"])), "flops": 4.0 * n}
    if c["op"] == "rope":
        n = c["T"] * (c["Hq"] + c["Hkv"]) * c["D"]
        return {"bytes": 4.0 * n + 4 * c["axes"] * c["T"], "flops": 3.0 * n}
    S, page = c["S"], c["page"]
    lens = _lens(S, c["L"], c["L"] // 3)
    if c["kind"] == "fork":  # the last page of a prompt, unless it is full, for each sample
        copied = sum(c["group"] for n in lens[: S // (1 + c["group"])] if n % page)
        entries = sum(-(-n // page) for n in lens[: S // (1 + c["group"])]) * (1 + c["group"])
    else:
        copied = sum(-(-n // page) for n in lens[: S // 2])
        entries = 2 * copied
    moved = 2 * 2 * copied * c["layers"] * c["Hkv"] * page * c["D"] * _element(c["kv"])
    return {"bytes": moved + 4 * 4 * entries, "flops": 0.0}


# ------------------------------------------------------------------------------------------------ 64 bits
def _held64(codes, scale, table, n):
    """The first n positions of one sequence: [heads, n, D] in 64 bits."""
    b, e = codes[table.long()].long(), scale[table.long()].long()  # pages, heads, page, D / 2 and D / 16
    c = torch.stack([b % 16, b // 16], -1).flatten(-2)
    exponent, mantissa = (c // 2) % 4, (c % 2).double()
    v = torch.where(exponent == 0, mantissa / 2, (1 + mantissa / 2) * torch.exp2(exponent.double() - 1))
    v = torch.where(c >= 8, -v, v)
    s = torch.where(e < 8, (e % 8).double() / 8 * 2.0 ** -14, (1 + (e % 8).double() / 8) * torch.exp2((e // 8).double() - 15))
    return (v * s.repeat_interleave(16, -1)).transpose(0, 1).flatten(1, 2)[:, :n]


def _held_as64(x):
    """The nearest values that 4 bits and a scale for 16 of them hold, halves to the even code."""
    x = x.unflatten(-1, (-1, 16))
    need = x.abs().amax(-1, keepdim=True) / 6
    # steps of the scale: 3 bits below the leading one, down to 2^-17
    unit = torch.exp2(torch.floor(torch.log2(need.clamp(min=2.0 ** -14))) - 3)
    scale = (torch.ceil(need / unit) * unit).clamp(max=10240.0)
    y = (x / torch.where(scale > 0, scale, 1.0)).clamp(-6, 6)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=1.0))) - 1)
    return (torch.round(y / step) * step * scale).flatten(-2)


def _turn64(x, pos, freq, axis, interleaved):
    """Rotation as a complex product: (x0 + i x1) * exp(i pos[axis] freq)."""
    x, h = x.double(), freq.numel()
    r = x[..., : 2 * h].unflatten(-1, (h, 2)) if interleaved else x[..., : 2 * h].unflatten(-1, (2, h)).transpose(-1, -2)
    a = torch.stack([pos[int(axis[i])].double() * float(freq[i]) for i in range(h)], -1)
    w = torch.polar(torch.ones_like(a), a)
    z = torch.view_as_real(torch.view_as_complex(r.contiguous()) * w[..., None, :])
    z = z.flatten(-2) if interleaved else z.transpose(-1, -2).flatten(-2)
    return torch.cat([z, x[..., 2 * h:]], -1)


def exact(case, seed):
    if case["op"] == "pages":  # whole numbers and copies only
        return None
    s, c = prepare(case, seed), case
    if c["op"] == "attention":
        if c["S"] * c["N"] * c["Hq"] * (c["L"] + c["N"]) * c["D"] > 4e11:
            return None
        G, t = c["Hq"] // c["Hkv"], s["cache"]
        out, lse = [], []
        for i, n in enumerate(s["lens_host"]):
            k, v = (_held64(t[x], t[x + "_scale"], t["table"][i], n) for x in "kv")
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
        k, v, n, pos = s["k"], s["v"], c["take"] or c["N"], s.get("pos")
        if s["nodes"] is not None:
            k, v = (torch.stack([x[i, s["nodes"][i].long()] for i in range(c["S"])]) for x in (k, v))
            pos = None if pos is None else torch.stack([pos[:, i, s["nodes"][i].long()] for i in range(c["S"])], 1)
        k = k.double() if pos is None else _turn64(k, pos, s["freq"], s["axis"], False)
        keep = (torch.arange(n, device="cuda") < s["count"][:, None])[..., None, None]
        if c["kv"] == "bf16":
            return k * keep, v.double() * keep
        return _held_as64(k) * keep, _held_as64(v.double()) * keep
    return tuple(_turn64(x, s["pos"], s["freq"], s["axis"], c["interleaved"]) for x in (s["q"], s["k"]))
