"""The cache of 4 bits: what is written is the nearest that the format holds, what is read is what it stands for."""
import math

import pytest
import torch

import attn_util as au
import e2m1_util as e4

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    import paper_2411_03786_b200 as ngs
    w = torch.zeros(64, 64, dtype=torch.bfloat16, device="cuda")
    c = ngs.SpecContext(w, w)
    yield c
    c.close()


def i32(*x):
    return torch.tensor(x, dtype=torch.int32).cuda()


def kv(S, N, heads, D, seed):
    g = torch.Generator().manual_seed(seed)
    t = torch.randn(S, N, 2 * heads, D, generator=g) * torch.exp(3 * torch.randn(S, N, 2 * heads, D // 16, generator=g)).repeat_interleave(16, -1)
    t = t.bfloat16().cuda()
    return t[:, :, :heads], t[:, :, heads:]


def held(cache, s, n):
    at = torch.arange(n)
    pages = cache.table[s].long().cpu()[at // cache.page]
    return [e4.dequantise(x.cpu()[pages, :, at % cache.page], y.cpu()[pages, :, at % cache.page]) for x, y in ((cache.k, cache.k_scale), (cache.v, cache.v_scale))]


@pytest.mark.parametrize("S,N,heads,D,page,start", [(1, 1, 1, 64, 16, [0]), (2, 7, 3, 128, 16, [13, 0]), (3, 40, 2, 64, 32, [31, 32, 5]), (2, 300, 8, 128, 64, [1, 700]),
                                                    (1, 130, 5, 128, 128, [127])])
def test_write_and_read(ctx, S, N, heads, D, page, start):
    cache, hk, hv = e4.make_cache(S, max(start) + N, heads, D, page, 1)
    k, v = kv(S, N, heads, D, 2)
    before = [t.clone() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale)]
    ctx.cache_write(cache, k, v, i32(*start))
    rk, rv = ctx.cache_read(cache, i32(*start), N)
    for x, r, old, t in ((k, rk, hk, 0), (v, rv, hv, 1)):
        want = e4.dequantise(*e4.quantise(x))
        assert torch.equal(r.double().cpu(), want)
        for s in range(S):
            now = held(cache, s, start[s] + N)[t]
            assert torch.equal(now[start[s]:], want[s]) and torch.equal(now[:start[s]], old[s, :start[s]])
    used = torch.zeros(cache.n_pages, dtype=torch.bool)
    used[cache.table.long().cpu().flatten()] = True
    for was, t in zip(before, (cache.k, cache.v, cache.k_scale, cache.v_scale)):
        assert torch.equal(was.cpu()[~used], t.cpu()[~used])
    assert ctx.get_status() == 0


def test_scale_bytes_are_the_smallest_that_reach(ctx):
    """Every bfloat16 magnitude as the largest of its group: the scale byte is that of the definition."""
    bits = torch.arange(0x7F81, dtype=torch.int32)  # zero to infinity
    x = torch.zeros(1, (len(bits) + 3) // 4 * 4, dtype=torch.int16)
    x[0, : len(bits)] = bits.to(torch.int16)
    n = x.shape[1] // 4
    k = torch.zeros(1, n, 1, 64, dtype=torch.int16)
    k[0, :, 0, 3::16] = x.view(n, 4)
    k = k.view(torch.bfloat16).cuda()
    cache, _, _ = e4.make_cache(1, n, 1, 64, 128, 0)
    ctx.cache_write(cache, k, -k, i32(0))
    codes, byte = e4.quantise(k[0, :, 0])
    pages, at = cache.table[0].long(), torch.arange(n, device="cuda")
    assert torch.equal(cache.k_scale[pages[at // 128], 0, at % 128].cpu(), byte)
    assert torch.equal(cache.v_scale[pages[at // 128], 0, at % 128].cpu(), byte)
    assert torch.equal(e4.dequantise(cache.k[pages[at // 128], 0, at % 128], byte), e4.dequantise(codes, byte))
    # no code is off by more than half of the widest step: from 4 to 6 it is two scales, so by one scale; none below the largest
    # scale is cut off
    fin = k[0, :, 0].double().cpu()
    err = (e4.dequantise(codes, byte) - fin).abs()
    ok = fin.abs() <= 61440
    assert (err[ok] <= e4.scale_values()[byte.long()].repeat_interleave(16, -1)[ok]).all()


def test_codes_of_all_quotients(ctx):
    """With 6 times a scale in each group the scale is that one: all bfloat16 below it are rounded to the nearest code, borders to the even
    one."""
    rows = []
    for byte in (1, 3, 7, 8, 11, 120, 125, 127, 130, 226):
        s = float(e4.scale_values()[byte])
        y = torch.cat([torch.linspace(0, 6, 1500), torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])]).double() * s
        y = torch.cat([y.bfloat16(), torch.nextafter(y.bfloat16(), torch.tensor(1e9).bfloat16()), torch.nextafter(y.bfloat16(), torch.tensor(-1.0).bfloat16())])
        y = y[(y >= 0) & (y.double() <= 6 * s)]
        y = y[: len(y) // 15 * 15].view(-1, 15)
        y = torch.cat([torch.full((len(y), 1), 6 * s).bfloat16(), y], 1)
        assert (y[:, 0].double() == 6 * s).all()
        rows += [y, -y]
    x = torch.cat(rows)
    x = torch.cat([x, torch.zeros(-len(x) % 8, 16).bfloat16()]).view(1, -1, 1, 128).cuda()
    n = x.shape[1]
    cache, _, _ = e4.make_cache(1, n, 1, 128, 64, 0)
    ctx.cache_write(cache, x, x.flip(1), i32(0))
    rk, rv = ctx.cache_read(cache, i32(0), n)
    want = e4.dequantise(*e4.quantise(x))
    assert torch.equal(rk.double().cpu(), want) and torch.equal(rv.double().cpu(), want.flip(1))


def test_values_at_the_ends(ctx):
    """Zeros, the smallest numbers, numbers beyond the format, infinities and NaN: a NaN takes its group of 16 and no other."""
    x = torch.randn(1, 8, 1, 64, generator=torch.Generator().manual_seed(3)).bfloat16().cuda()
    x[0, 0] = 0
    x[0, 1] = -0.0
    x[0, 2, 0, ::3] = 9.2e-41  # a subnormal
    x[0, 3, 0, 5] = math.inf
    x[0, 4, 0, 40] = -math.inf
    x[0, 5, 0, 17] = math.nan
    x[0, 6] = 3.3e38
    x[0, 7] = 2.0 ** -18
    cache, _, _ = e4.make_cache(1, 8, 1, 64, 16, 0)
    ctx.cache_write(cache, x, x, i32(0))
    k, v = ctx.cache_read(cache, i32(0), 8)
    want = e4.dequantise(*e4.quantise(x))
    for got in (k, v):
        got = got.double().cpu()
        assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(), want.nan_to_num())
    assert want.isnan().sum() == 16 and k[0, 3, 0, 5] == 61440 and k[0, 4, 0, 40] == -61440 and (k[0, 6] == 61440).all()


def test_scale_bytes_beyond_the_largest_read_as_nan(ctx):
    cache, _, _ = e4.make_cache(1, 64, 1, 64, 64, 0)
    page = int(cache.table[0, 0])
    cache.k_scale[page, 0, :, 1] = torch.arange(64, dtype=torch.uint8, device="cuda") + 192
    k, v = ctx.cache_read(cache, i32(0), 64)
    nan = k[0, :, 0].isnan()
    want = torch.zeros(64, 64, dtype=torch.bool)
    want[227 - 192:, 16:32] = True
    assert torch.equal(nan.cpu(), want) and v.isfinite().all()


@pytest.mark.parametrize("interleaved", [False, True])
def test_keys_are_rotated_before_they_are_held(ctx, interleaved):
    import paper_2411_03786_b200 as ngs
    S, N, heads, D = 2, 50, 2, 128
    cache, _, _ = e4.make_cache(S, 100, heads, D, 16, 5)
    k, v = kv(S, N, heads, D, 6)
    start = i32(40, 3)
    rope = ngs.Rope((10000.0 ** (-torch.arange(0, 64, 2, dtype=torch.float64) / 64)).float().cuda(), interleaved)
    ctx.cache_write(cache, k, v, start, rope=rope)
    turned, _ = ctx.rope_rows(rope, k, None, start[:, None] + torch.arange(N, device="cuda").int())
    rk, rv = ctx.cache_read(cache, start, N)
    assert torch.equal(rk.double().cpu(), e4.dequantise(*e4.quantise(turned))) and torch.equal(rv.double().cpu(), e4.dequantise(*e4.quantise(v)))


def test_commit_of_chosen_nodes(ctx):
    S, N, heads, D = 3, 24, 2, 128
    cache, hk, hv = e4.make_cache(S, 48, heads, D, 16, 3)
    k, v = kv(S, N, heads, D, 4)
    nodes = torch.tensor([[0, 1, 2, -1], [6, 7, -1, -1], [23, 0, 5, 24]], dtype=torch.int32).cuda()
    start, count = [10, 31, 0], [3, 2, 9]
    ctx.cache_write(cache, k, v, i32(*start), count=i32(*count), nodes=nodes)
    for s in range(S):
        want = [hk[s, :48].clone(), hv[s, :48].clone()]
        for i in range(min(4, count[s])):
            node = int(nodes[s, i])
            if 0 <= node < N:
                for w, x in zip(want, (k, v)):
                    w[start[s] + i] = e4.dequantise(*e4.quantise(x[s, node]))
        assert all(torch.equal(a, b) for a, b in zip(held(cache, s, 48), want))
    rk, rv = ctx.cache_read(cache, i32(*start), 4, count=i32(4, 0, 2))
    assert (rk[1] == 0).all() and (rv[2, 2:] == 0).all() and torch.equal(rk[0].double().cpu(), held(cache, 0, 14)[0][10:])


def test_positions_without_a_page(ctx):
    import paper_2411_03786_b200 as ngs
    cache, _, _ = e4.make_cache(2, 32, 1, 64, 16, 3)
    before = [t.clone() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale)]
    cache.table[1] = i32(-1, cache.n_pages)
    k, v = kv(2, 4, 1, 64, 4)
    ctx.cache_write(cache, k, v, i32(31, 14))
    assert ctx.get_status() == ngs.STATUS_CAPACITY
    page = int(cache.table[0, 1])
    for was, t in zip(before, (cache.k, cache.v, cache.k_scale, cache.v_scale)):
        was[page, 0, 15] = t[page, 0, 15]
        assert torch.equal(was, t)
    rk, _ = ctx.cache_read(cache, i32(0, 0), 32)
    assert (rk[1] == 0).all() and ctx.get_status() == ngs.STATUS_CAPACITY


def test_empty_and_odd_calls(ctx):
    import paper_2411_03786_b200 as ngs
    cache = ngs.KVCache.empty(4, 2, 16, 64, torch.arange(4, dtype=torch.int32, device="cuda").view(2, 2), bits=4)
    assert cache.k.shape == (4, 2, 16, 32) and cache.k_scale.shape == (4, 2, 16, 4) and cache.head_dim == 64
    z = torch.zeros(2, 0, 2, 64, dtype=torch.bfloat16, device="cuda")
    ctx.cache_write(cache, z, z, i32(0, 0))
    assert ctx.cache_read(cache, i32(0, 0), 0)[0].shape == (2, 0, 2, 64)
    for kw in ({"k_scale": cache.k_scale}, {"k_scale": cache.k_scale, "v_scale": cache.v_scale[..., :2].contiguous()}, {"k_scale": cache.k_scale.cpu(), "v_scale": cache.v_scale},
               {"k_scale": cache.k_scale.float(), "v_scale": cache.v_scale.float()}, {"k_scale": cache.k_scale, "v_scale": cache.v_scale, "k_exp": cache.k_scale[..., 0].contiguous()},
               {"v_scale": cache.v_scale}):
        with pytest.raises(ngs.SpecError):
            ngs.KVCache(cache.k, cache.v, cache.table, **kw)
    with pytest.raises(ngs.SpecError):
        ngs.KVCache(cache.k.bfloat16(), cache.v.bfloat16(), cache.table, k_scale=cache.k_scale, v_scale=cache.v_scale)
    with pytest.raises(ngs.SpecError):
        ngs.KVCache.empty(4, 2, 16, 64, cache.table, bits=2)
    assert ctx.get_status() == 0
