"""Plain forms of a cache of 4 bits, from its definition, in 64 bits on the host."""
import torch

CODES = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)
TOP = 226


def scale_values():
    """What the 256 scale bytes stand for: 5 exponent bits (bias 15, subnormals) and 3 mantissa bits; NaN beyond the largest."""
    b = torch.arange(256)
    e, m = (b // 8).double(), (b % 8).double()
    s = torch.where(b < 8, m / 8 * 2.0 ** -14, (1 + m / 8) * torch.exp2(e - 15))
    s[TOP + 1:] = float("nan")
    return s


def quantise(x):
    """[..., D] -> (packed codes uint8 [..., D / 2], scale bytes uint8 [..., D / 16])."""
    x = x.double().cpu().unflatten(-1, (-1, 16))
    nan = x.isnan().any(-1)
    x = x.nan_to_num(nan=0.0, posinf=1e300, neginf=-1e300)
    scales = scale_values()[: TOP + 1]
    byte = torch.searchsorted(6 * scales, x.abs().amax(-1).contiguous()).clamp(max=TOP)
    s = scales[byte][..., None]
    y = (x.abs() / torch.where(s > 0, s, 1.0)).clamp(max=6.0).contiguous()
    at = torch.searchsorted(CODES, y)
    lo, hi = (at - 1).clamp(min=0), at.clamp(max=7)
    dl, dh = y - CODES[lo], CODES[hi] - y
    code = torch.where(dl < dh, lo, torch.where(dh < dl, hi, torch.where(lo % 2 == 0, lo, hi)))
    code = torch.where(s > 0, code, 0)
    code = (code + 8 * (torch.signbit(x) & (code > 0)).long()).masked_fill(nan[..., None], 0).flatten(-2)
    return (code[..., 0::2] + 16 * code[..., 1::2]).to(torch.uint8), byte.masked_fill(nan, 255).to(torch.uint8)


def dequantise(codes, scale):
    c, s = codes.cpu().long(), scale.cpu().long()
    c = torch.stack([c % 16, c // 16], -1).flatten(-2)
    v = torch.where(c >= 8, -CODES[c % 8], CODES[c % 8])
    return v * scale_values()[s].repeat_interleave(16, -1)


def make_cache(S, tokens, heads, D, page, seed, spare=3, gain=1.0):
    """A cache whose pages are handed out in no order, `spare` of them to nobody.  Returns (KVCache, k, v) with the values that it
    holds as float64 [S, per * page, heads, D] on the host."""
    import paper_2411_03786_b200 as ngs
    g = torch.Generator().manual_seed(seed)
    per = max(1, -(-tokens // page))
    n = S * per + spare
    q = [quantise((torch.randn(n, heads, page, D, generator=g) * gain).bfloat16()) for _ in range(2)]
    table = torch.randperm(n, generator=g)[: S * per].int().view(S, per)
    cache = ngs.KVCache(q[0][0].cuda(), q[1][0].cuda(), table.cuda(), k_scale=q[0][1].cuda(), v_scale=q[1][1].cuda())
    held = [dequantise(*x)[table.long()].permute(0, 1, 3, 2, 4).reshape(S, per * page, heads, D) for x in q]
    return cache, held[0], held[1]
