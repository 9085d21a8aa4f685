"""Plain 64-bit forms of the cache, rotary and tree-attention calls, and inputs for their tests."""
import math

import torch

E4M3 = None


def e4m3_values():
    """The 256 values of E4M3 in 64 bits."""
    global E4M3
    if E4M3 is None:
        v = []
        for b in range(256):
            e, m = (b >> 3) & 15, b & 7
            x = math.nan if (b & 127) == 127 else (m * 2.0 ** -9 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
            v.append(-x if b & 128 else x)
        E4M3 = torch.tensor(v, dtype=torch.float64)
    return E4M3


def quantise(x):
    """[..., D] -> (codes, scale bytes), from the definition, in 64 bits on the host: nearest value, ties to the even code."""
    x = x.double().cpu()
    nan = x.isnan().any(-1)
    top = x.nan_to_num(nan=0.0).abs().amax(-1)
    e = torch.ceil(torch.log2(top.clamp(min=1e-60, max=448 * 2.0 ** 7) / 448))
    e = torch.where(top > 0, e.clamp(-120, 7), torch.zeros_like(e))
    y = (x / torch.exp2(e)[..., None]).clamp(-448, 448).nan_to_num(nan=0.0)
    pos = e4m3_values()[:127]
    at = torch.searchsorted(pos, y.abs().contiguous())
    lo, hi = (at - 1).clamp(min=0), at.clamp(max=126)
    dl, dh = y.abs() - pos[lo], pos[hi] - y.abs()
    code = torch.where(dl < dh, lo, torch.where(dh < dl, hi, torch.where(lo % 2 == 0, lo, hi)))
    code = code + 128 * torch.signbit(y).long()
    code = torch.where(nan[..., None], 127, code)
    return code.to(torch.uint8), torch.where(nan, 255, e + 127).to(torch.uint8)


def dequantise(codes, exp):
    s = torch.exp2(exp.cpu().double() - 127)
    s[exp.cpu() == 255] = math.nan
    return e4m3_values()[codes.cpu().long()] * s[..., None]


def make_cache(S, tokens, heads, D, page, quantised, seed, spare=3, fill=None):
    """A cache whose pages are handed out in no order, `spare` of them to nobody.  Returns (KVCache, k, v) with the
    values that it holds as float64 [S, per * page, heads, D] on the host."""
    import paper_2411_03786_b200 as ngs
    g = torch.Generator().manual_seed(seed)
    per = max(1, -(-tokens // page))
    n = S * per + spare
    kv = [torch.randn(n, heads, page, D, generator=g).bfloat16() for _ in range(2)]
    if fill is not None:
        kv = [torch.full_like(x, fill) for x in kv]
    table = torch.randperm(n, generator=g)[: S * per].int().view(S, per)
    if quantised:
        q = [quantise(x) for x in kv]
        held = [dequantise(*x) for x in q]
        cache = ngs.KVCache(q[0][0].cuda(), q[1][0].cuda(), table.cuda(), q[0][1].cuda(), q[1][1].cuda())
    else:
        held = [x.double() for x in kv]
        cache = ngs.KVCache(kv[0].cuda(), kv[1].cuda(), table.cuda())
    # [S, per, heads, page, D] -> [S, per * page, heads, D]
    held = [x[table.long()].permute(0, 1, 3, 2, 4).reshape(S, per * page, heads, D) for x in held]
    return cache, held[0], held[1]


def rotate(x, pos, freq, interleaved, factor):
    """x [..., heads, D] at pos [...], in 64 bits."""
    x, h = x.double().cpu(), freq.numel()
    a = pos.double().cpu()[..., None, None] * freq.double().cpu()
    c, s = torch.cos(a) * factor, torch.sin(a) * factor
    y = x.clone()
    i, j = (slice(0, 2 * h, 2), slice(1, 2 * h, 2)) if interleaved else (slice(0, h), slice(h, 2 * h))
    y[..., i], y[..., j] = x[..., i] * c - x[..., j] * s, x[..., i] * s + x[..., j] * c
    return y


def ancestors(parent):
    """[S, N] parents -> bool [S, N, N]."""
    S, N = parent.shape
    m = torch.zeros(S, N, N, dtype=torch.bool)
    for s in range(S):
        for i in range(N):
            j = i
            while j >= 0:
                m[s, i, j] = True
                j = int(parent[s, j])
    return m


def pack(mask):
    """bool [S, N, N] -> int32 words [S, N, ceil(N / 32)]."""
    S, N, _ = mask.shape
    W = (N + 31) // 32
    b = torch.zeros(S, N, W * 32, dtype=torch.int64)
    b[..., :N] = mask.long()
    w = (b.view(S, N, W, 32) << torch.arange(32)).sum(-1)
    return torch.where(w >= 2 ** 31, w - 2 ** 32, w).int()


def attention(q, k, v, held_k, held_v, mask, lens, scale, live=None):
    """out, lse and sum p |v| in 64 bits.  What a row does not attend to is left out, not multiplied by zero."""
    held_k, held_v, mask = held_k.cuda(), held_v.cuda(), mask.cuda()
    S, N, Hq, D = q.shape
    G = Hq // k.shape[2]
    out, lse, mag = torch.zeros(S, N, Hq, D, dtype=torch.float64), torch.full((S, N, Hq), -math.inf, dtype=torch.float64), torch.zeros(S, N, Hq, D, dtype=torch.float64)
    q, k, v = (x.double().cuda() for x in (q, k, v))
    out, lse, mag = out.cuda(), lse.cuda(), mag.cuda()
    for s in range(S):
        n = int(lens[s])
        for i in range(N if live is None else int(live[s])):
            nodes = mask[s, i].nonzero()[:, 0]
            if live is not None:
                nodes = nodes[nodes < int(live[s])]
            kk = torch.cat([held_k[s, :n], k[s, nodes]]).repeat_interleave(G, 1)  # [keys, Hq, D]
            vv = torch.cat([held_v[s, :n], v[s, nodes]]).repeat_interleave(G, 1)
            if not kk.shape[0]:
                continue
            z = torch.einsum("hd,khd->hk", q[s, i], kk) * scale
            lse[s, i] = torch.logsumexp(z, -1)
            p = torch.exp(z - lse[s, i][:, None])
            out[s, i] = torch.einsum("hk,khd->hd", p, vv)
            mag[s, i] = torch.einsum("hk,khd->hd", p, vv.abs())
    return out.cpu(), lse.cpu(), mag.cpu()


def check_attention(got, ref, score_bound):
    """Weights rounded to bfloat16 (8 significant bits: 2^-8 of each at most, so 2^-8 of sum p |v|), an output rounded to
    bfloat16 (2^-8 of itself), fp32 elsewhere; scores within `score_bound` of the exact ones, which moves a weight by as much."""
    out, lse, mag = ref
    o, l = got[0].double().cpu(), got[1].double().cpu()
    fin = out.isfinite()
    assert torch.equal(o.isnan(), out.isnan()) and torch.equal(o[~fin & ~out.isnan()], out[~fin & ~out.isnan()])
    tol = (2.0 ** -8) * out.abs() + (2.0 ** -8 + 2 * score_bound) * mag + 1e-30
    bad = (o - out).abs() > tol
    assert not (bad & fin).any(), f"worst {((o - out).abs() / tol)[fin].max():.2f} of the tolerance"
    lf = lse.isfinite()
    assert torch.equal(lf, l.isfinite()) and torch.equal(l[lse == -math.inf], lse[lse == -math.inf])
    assert ((l - lse).abs()[lf] <= score_bound + 2.0 ** -20 * (1 + lse.abs()[lf])).all()
