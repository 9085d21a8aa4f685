"""Rotary positions with several axes against their 64-bit form: rows, keys on their way into a cache, refusals."""
import math

import pytest
import torch

import attn_util as au
import e2m1_util as e4
from test_gpu_cache import near_bf16

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    import paper_2411_03786_b200 as ngs
    w = torch.zeros(64, 64, dtype=torch.bfloat16, device="cuda")
    c = ngs.SpecContext(w, w)
    yield c
    c.close()


def freqs(rot):
    return (10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)).float().cuda()


def rotate(x, pos, freq, axis, interleaved, factor):
    """x [..., heads, D], pos [axes, ...], in 64 bits: pair by pair."""
    x, y, h = x.double().cpu(), x.double().cpu().clone(), freq.numel()
    pos, freq, axis = pos.double().cpu(), freq.double().cpu(), axis.cpu()
    for i in range(h):
        at = pos[int(axis[i])] if int(axis[i]) < pos.shape[0] else torch.zeros_like(pos[0])
        c, s = torch.cos(at * freq[i])[..., None] * factor, torch.sin(at * freq[i])[..., None] * factor
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + h)
        y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
    return y


def axis_of(pairs, axes, kind):
    if kind == "sections":
        return (torch.arange(pairs) * axes // pairs).to(torch.uint8).cuda()
    return (torch.arange(pairs) % axes).to(torch.uint8).cuda()


@pytest.mark.parametrize("kind", ["sections", "turns"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,rot", [(64, 64), (128, 128), (128, 96), (80, 80), (80, 32), (256, 64), (16, 16)])
@pytest.mark.parametrize("T,Hq,Hk,axes", [(1, 1, 1, 1), (5, 7, 2, 3), (33, 4, 0, 2), (700, 3, 3, 8), (1200, 28, 4, 3)])
def test_rows(ctx, T, Hq, Hk, axes, D, rot, interleaved, kind):
    import paper_2411_03786_b200 as ngs
    g = torch.Generator().manual_seed(T + D)
    q = torch.randn(T, Hq, D, generator=g).bfloat16().cuda()
    k = torch.randn(T, Hk, D, generator=g).bfloat16().cuda() if Hk else None
    pos = torch.randint(0, 131072, (axes, T), generator=g).int().cuda()
    f, axis = freqs(rot), axis_of(rot // 2, axes, kind)
    rope = ngs.Rope(f, interleaved, 1.25, axis=axis)
    out = ctx.rope_rows(rope, q, k, pos)
    for x, y in zip((q, k), out):
        if x is not None:
            near_bf16(y, rotate(x, pos, f, axis, interleaved, 1.25), extra=2.0 ** -20 * x.abs().max().item())
            assert torch.equal(y[..., rot:], x[..., rot:])
    ctx.rope_rows(rope, q, k, pos, out=(q, k))  # in place
    assert torch.equal(q, out[0]) and (k is None or torch.equal(k, out[1]))


@pytest.mark.parametrize("interleaved", [False, True])
def test_equal_positions_are_one_axis(ctx, interleaved):
    """Where all axes agree (text) the result is that of one axis, bit for bit, strided inputs among them."""
    import paper_2411_03786_b200 as ngs
    t = torch.randn(3, 40, 9, 64).bfloat16().cuda()
    q, k = t[:, :, :6], t[:, :, 6:]
    pos = torch.randint(-5, 100000, (3, 40)).int().cuda()
    f = freqs(64)
    a = ctx.rope_rows(ngs.Rope(f, interleaved), q, k, pos)
    b = ctx.rope_rows(ngs.Rope(f, interleaved, axis=axis_of(32, 3, "turns")), q, k, pos.expand(3, 3, 40).contiguous())
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_pairs_without_an_axis_pass(ctx):
    import paper_2411_03786_b200 as ngs
    q = torch.randn(10, 2, 64).bfloat16().cuda()
    axis = torch.full((32,), 255, dtype=torch.uint8, device="cuda")
    axis[::4] = 1
    pos = torch.randint(1, 1000, (2, 10)).int().cuda()
    y = ctx.rope_rows(ngs.Rope(freqs(64), axis=axis), q, None, pos)[0]
    still = (axis == 255).repeat(2)
    assert torch.equal(y[..., still], q[..., still])
    near_bf16(y, rotate(q, pos, freqs(64), axis, False, 1.0), extra=2.0 ** -20 * q.abs().max().item())


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("chosen", [False, True])
def test_keys_on_their_way_into_a_cache(ctx, bits, interleaved, chosen):
    """The cache holds what rows rotated beforehand would leave in it."""
    import paper_2411_03786_b200 as ngs
    S, N, heads, D, rot, page = 3, 37, 2, 128, 96, 16
    g = torch.Generator().manual_seed(bits)
    t = torch.randn(S, N, 2 * heads, D, generator=g).bfloat16().cuda()
    k, v = t[:, :, :heads], t[:, :, heads:]
    pos = torch.randint(0, 5000, (3, S, N), generator=g).int().cuda()
    rope = ngs.Rope(freqs(rot), interleaved, 1.125, axis=axis_of(rot // 2, 3, "turns"))
    turned = ctx.rope_rows(rope, k, None, pos)[0]
    start = torch.tensor([0, 21, 5], dtype=torch.int32).cuda()
    nodes = torch.randint(-1, N, (S, 20), generator=g).int().cuda() if chosen else None
    count = torch.tensor([20, 7, 0], dtype=torch.int32).cuda() if chosen else None
    table = torch.randperm(S * 4, generator=g).int().view(S, 4).cuda()
    got = []
    for keys, kw in ((k, {"rope": rope, "pos": pos}), (turned, {})):
        cache = ngs.KVCache.empty(S * 4, heads, page, D, table, bits=bits)
        for x in (cache.k, cache.v, cache.k_exp, cache.v_exp, cache.k_scale, cache.v_scale):
            if x is not None:
                x.zero_()
        ctx.cache_write(cache, keys, v, start, count=count, nodes=nodes, **kw)
        got.append(ctx.cache_read(cache, torch.zeros_like(start), 64))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
    assert ctx.get_status() == 0 and got[0][0].any()


def test_positions_that_are_not_slots(ctx):
    """One axis without a list of axes: rotary positions of their own."""
    import paper_2411_03786_b200 as ngs
    S, N, heads, D = 2, 9, 1, 64
    k = torch.randn(S, N, heads, D).bfloat16().cuda()
    pos = torch.randint(0, 5000, (S, N)).int().cuda()
    rope = ngs.Rope(freqs(D))
    cache = ngs.KVCache.empty(S, heads, 16, D, torch.arange(S, dtype=torch.int32, device="cuda").view(S, 1))
    start = torch.tensor([0, 7], dtype=torch.int32).cuda()
    ctx.cache_write(cache, k, k, start, rope=rope, pos=pos)
    rk, rv = ctx.cache_read(cache, start, N)
    assert torch.equal(rk, ctx.rope_rows(rope, k, None, pos)[0]) and torch.equal(rv, k)


def test_refusals(ctx):
    import paper_2411_03786_b200 as ngs
    f = freqs(64)
    axis = axis_of(32, 3, "turns")
    for bad in (axis[:31], axis.int(), axis.cpu(), axis.view(2, 16), axis.repeat(2)[::2]):
        with pytest.raises(ngs.SpecError):
            ngs.Rope(f, axis=bad)
    rope = ngs.Rope(f, axis=axis)
    q = torch.zeros(6, 2, 64, dtype=torch.bfloat16, device="cuda")
    pos = torch.zeros(3, 6, dtype=torch.int32, device="cuda")
    ctx.rope_rows(rope, q, None, pos)
    for bad in (pos[0], pos[:, :5], pos.long(), pos.T.contiguous().T, pos.cpu(), torch.zeros(9, 6, dtype=torch.int32, device="cuda"), pos[:0]):
        with pytest.raises(ngs.SpecError):
            ctx.rope_rows(rope, q, None, bad)
    cache = ngs.KVCache.empty(2, 2, 16, 64, torch.zeros(1, 2, dtype=torch.int32, device="cuda"))
    k = q.view(1, 6, 2, 64)
    start = torch.zeros(1, dtype=torch.int32, device="cuda")
    for kw in ({"rope": rope}, {"pos": pos.view(3, 1, 6)}, {"rope": rope, "pos": pos}, {"rope": rope, "pos": pos.view(3, 1, 6)[:, :, :5]}, {"rope": ngs.Rope(f), "pos": pos.view(3, 1, 6)}):
        with pytest.raises(ngs.SpecError):
            ctx.cache_write(cache, k, k, start, **kw)
    e = q[:0]
    assert ctx.rope_rows(rope, e, None, pos[:, :0])[0].shape == (0, 2, 64)
    assert ctx.get_status() == 0
