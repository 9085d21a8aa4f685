"""Rotary positions, the paged cache and tree masks against their plain 64-bit forms."""
import math

import pytest
import torch

import attn_util as au

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    import paper_2411_03786_b200 as ngs
    w = torch.zeros(64, 64, dtype=torch.bfloat16, device="cuda")
    c = ngs.SpecContext(w, w)
    yield c
    c.close()


def freqs(rot, stretch=1.0):
    return (10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot) / stretch).float().cuda()


def near_bf16(got, ref, extra=0.0):
    """Rounded once to bfloat16: off by half the spacing of bfloat16 at the exact value (2^-7 of its power of two), and by
    what fp32 leaves before it: cos, sin and products within a few 2^-23 of the pair's length."""
    ref = ref.cpu()
    half = torch.exp2(torch.floor(torch.log2(ref.abs().clamp(min=2.0 ** -126))) - 8)
    assert ((got.double().cpu() - ref).abs() <= half + extra).all()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,rot", [(64, 64), (64, 16), (128, 128), (128, 96), (80, 32), (256, 64), (16, 16)])
@pytest.mark.parametrize("T,Hq,Hk", [(1, 1, 1), (5, 7, 2), (33, 4, 0), (700, 3, 3)])
def test_rope_rows(ctx, T, Hq, Hk, D, rot, interleaved):
    import paper_2411_03786_b200 as ngs
    g = torch.Generator().manual_seed(T + D)
    q = torch.randn(T, Hq, D, generator=g).bfloat16().cuda()
    k = torch.randn(T, Hk, D, generator=g).bfloat16().cuda() if Hk else None
    pos = torch.randint(0, 131072, (T,), generator=g).int().cuda()
    f = freqs(rot, 2.0)
    out = ctx.rope_rows(ngs.Rope(f, interleaved, 1.25), q, k, pos)
    for x, y in zip((q, k), out):
        if x is not None:
            near_bf16(y, au.rotate(x, pos, f, interleaved, 1.25), extra=2.0 ** -20 * x.abs().max().item())
            assert torch.equal(y[..., rot:], x[..., rot:])
    ctx.rope_rows(ngs.Rope(f, interleaved, 1.25), q, k, pos, out=(q, k))  # in place
    assert torch.equal(q, out[0]) and (k is None or torch.equal(k, out[1]))


def test_rope_strides_and_identity(ctx):
    import paper_2411_03786_b200 as ngs
    t = torch.randn(3, 4, 9, 64).bfloat16().cuda()
    q, k = t[:, :, :6], t[:, :, 6:]
    pos = torch.arange(12).int().view(3, 4).cuda()
    f = freqs(64)
    a = ctx.rope_rows(ngs.Rope(f), q, k, pos)
    b = ctx.rope_rows(ngs.Rope(f), q.contiguous(), k.contiguous(), pos)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    z = ctx.rope_rows(ngs.Rope(f), q, None, torch.zeros_like(pos))[0]
    assert torch.equal(z, q)


def kv(S, N, heads, D, seed, wide=True):
    g = torch.Generator().manual_seed(seed)
    t = torch.randn(S, N, 2 * heads, D, generator=g)
    if wide:
        t = t * torch.exp(4 * torch.randn(S, N, 2 * heads, 1, generator=g))
    t = t.bfloat16().cuda()
    return t[:, :, :heads], t[:, :, heads:]


def held(cache, s, n):
    """What positions 0 .. n-1 of a sequence hold, float64 [n, heads, D]."""
    at = torch.arange(n)
    pages = cache.table[s].long().cpu()[at // cache.page]
    k, v = (t.cpu()[pages, :, at % cache.page] for t in (cache.k, cache.v))
    if cache.k_exp is None:
        return k.double(), v.double()
    return au.dequantise(k, cache.k_exp.cpu()[pages, :, at % cache.page]), au.dequantise(v, cache.v_exp.cpu()[pages, :, at % cache.page])


@pytest.mark.parametrize("quantised", [False, True])
@pytest.mark.parametrize("S,N,heads,D,page,start", [(1, 1, 1, 64, 16, [0]), (2, 7, 3, 128, 16, [13, 0]), (3, 40, 2, 64, 32, [31, 32, 5]), (2, 300, 8, 128, 64, [1, 700])])
def test_write_and_read(ctx, S, N, heads, D, page, start, quantised):
    tokens = max(start) + N
    cache, hk, hv = au.make_cache(S, tokens, heads, D, page, quantised, 1)
    k, v = kv(S, N, heads, D, 2)
    st = torch.tensor(start, dtype=torch.int32).cuda()
    before = [t.clone() for t in (cache.k, cache.v)]
    ctx.cache_write(cache, k, v, st)
    rk, rv = ctx.cache_read(cache, st, N)
    for x, r, old, t in ((k, rk, hk, 0), (v, rv, hv, 1)):
        want = au.dequantise(*au.quantise(x)) if quantised else x.double().cpu()
        assert torch.equal(r.double().cpu(), want)
        for s in range(S):
            now = held(cache, s, tokens)[t]
            assert torch.equal(now[start[s]:start[s] + N], want[s]) and torch.equal(now[:start[s]], old[s, :start[s]])
    used = torch.zeros(cache.n_pages, dtype=torch.bool)
    used[cache.table.long().cpu().flatten()] = True
    assert torch.equal(cache.k.cpu()[~used], before[0].cpu()[~used]) and torch.equal(cache.v.cpu()[~used], before[1].cpu()[~used])
    assert ctx.get_status() == 0


@pytest.mark.parametrize("quantised", [False, True])
def test_commit_of_chosen_nodes(ctx, quantised):
    S, N, heads, D = 4, 24, 2, 128
    cache, hk, hv = au.make_cache(S, 40, heads, D, 16, quantised, 3)
    k, v = kv(S, N, heads, D, 4)
    nodes = torch.tensor([[0, 1, 2, -1], [6, 7, -1, -1], [23, 0, 5, 24], [-1, 9, 1 << 30, 3]], dtype=torch.int32).cuda()
    start, count = [10, 31, 0, 36], [3, 2, 4, 9]
    ctx.cache_write(cache, k, v, torch.tensor(start, dtype=torch.int32).cuda(), count=torch.tensor(count, dtype=torch.int32).cuda(), nodes=nodes)
    for s in range(S):
        gk, gv = held(cache, s, 48)
        wk, wv = hk[s, :48].clone(), hv[s, :48].clone()
        for i in range(min(4, count[s])):
            node = int(nodes[s, i])
            if 0 <= node < N:
                wk[start[s] + i] = au.dequantise(*au.quantise(k[s, node])) if quantised else k[s, node].double().cpu()
                wv[start[s] + i] = au.dequantise(*au.quantise(v[s, node])) if quantised else v[s, node].double().cpu()
        assert torch.equal(gk, wk) and torch.equal(gv, wv)
    assert ctx.get_status() == 0


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,rot", [(64, 32), (128, 128), (128, 96)])
def test_write_rotates_as_rope_rows_does(ctx, D, rot, interleaved):
    import paper_2411_03786_b200 as ngs
    S, N, heads = 2, 21, 3
    rope = ngs.Rope(freqs(rot), interleaved, 0.9)
    k, v = kv(S, N, heads, D, 5)
    start = torch.tensor([100, 7], dtype=torch.int32).cuda()
    pos = start[:, None] + torch.arange(N, device="cuda").int()
    turned = ctx.rope_rows(rope, k, None, pos.contiguous())[0]
    for quantised in (False, True):
        a, b = (au.make_cache(S, 130, heads, D, 16, quantised, 6)[0] for _ in range(2))
        ctx.cache_write(a, k, v, start, rope=rope)
        ctx.cache_write(b, turned, v, start)
        assert torch.equal(a.k, b.k) and torch.equal(a.v, b.v)
        assert not quantised or (torch.equal(a.k_exp, b.k_exp) and torch.equal(a.v_exp, b.v_exp))


def test_special_values(ctx):
    """Zeros, infinities, NaN, magnitudes beyond both ends of the scales, and ties between codes."""
    D = 64
    x = torch.zeros(1, 10, 1, D)
    x[0, 1, 0, 3], x[0, 1, 0, 4] = math.inf, -1.0
    x[0, 2, 0, 5] = math.nan
    x[0, 3, 0, :2] = torch.tensor([3e38, -57344.0])
    x[0, 4, 0, :2] = torch.tensor([1e-38, 2e-38])
    x[0, 5, 0, :3] = torch.tensor([448.0, 432.0, -0.0])
    x[0, 6, 0, :3] = torch.tensor([450.0, 17.0, 19.0])
    x[0, 7, 0] = torch.arange(D) * 8.0 - 252
    x[0, 8, 0] = 2.0 ** -133
    x[0, 9, 0] = -torch.arange(D) / 64.0
    x = x.bfloat16().cuda()
    cache, _, _ = au.make_cache(1, 16, 1, D, 16, True, 1)
    zero = torch.zeros(1, dtype=torch.int32).cuda()
    ctx.cache_write(cache, x, x, zero)
    codes, exp = au.quantise(x)
    rk, rv = ctx.cache_read(cache, zero, 10)
    want = au.dequantise(codes, exp)
    for r in (rk, rv):
        r = r.double().cpu()
        assert torch.equal(r.isnan(), want.isnan()) and torch.equal(r.nan_to_num(nan=0.0), want.nan_to_num(nan=0.0))
    assert rk[0, 1, 0, 3] == 57344 and rk[0, 2].isnan().all() and rk[0, 3, 0, 0] == 57344 and (rk[0, 0] == 0).all()
    page = int(cache.table[0, 0])
    assert torch.equal(cache.k_exp[page, 0, :10].cpu(), exp[0, :, 0]) and torch.equal(cache.v_exp[page, 0, :10].cpu(), exp[0, :, 0])


def test_every_code_survives(ctx):
    """All finite codes at a scale byte come back bit for bit after read and write."""
    codes = torch.tensor([b for b in range(256) if b & 127 != 127], dtype=torch.uint8)
    rows = torch.zeros(4, 64, dtype=torch.uint8)
    rows[:, :62] = torch.cat([codes, codes[-(4 * 62 - codes.numel()):] if codes.numel() < 248 else codes[:0]])[:248].view(4, 62)
    rows[:, 63] = 126  # 448: the scale is what it was
    for exp in (7, 100, 127, 134):
        c, _, _ = au.make_cache(1, 4, 1, 64, 16, True, 1, spare=0)
        c.k[0, 0, :4], c.v[0, 0, :4] = rows.cuda(), rows.cuda()
        c.k_exp[0, 0, :4], c.v_exp[0, 0, :4] = exp, exp
        zero = torch.zeros(1, dtype=torch.int32).cuda()
        k, v = ctx.cache_read(c, zero, 4)
        d, _, _ = au.make_cache(1, 4, 1, 64, 16, True, 2, spare=0)
        ctx.cache_write(d, k, v, zero)
        assert torch.equal(d.k[0, 0, :4], rows.cuda()) and (d.k_exp[0, 0, :4] == exp).all()


def test_read_counts_and_status(ctx):
    import paper_2411_03786_b200 as ngs
    cache, hk, hv = au.make_cache(3, 32, 2, 64, 16, False, 9)
    st = torch.tensor([30, 0, 5], dtype=torch.int32).cuda()
    k, v = ctx.cache_read(cache, st, 6, count=torch.tensor([2, 0, 99], dtype=torch.int32).cuda())
    assert torch.equal(k[0, :2].double().cpu(), hk[0, 30:32]) and (k[0, 2:] == 0).all() and (v[1] == 0).all()
    assert torch.equal(v[2].double().cpu(), hv[2, 5:11]) and ctx.get_status() == 0
    k, v = ctx.cache_read(cache, st, 6)  # the first sequence runs out of pages
    assert (k[0, 2:] == 0).all() and ctx.get_status() == ngs.STATUS_CAPACITY
    before = cache.k.clone()
    x = torch.ones(3, 1, 2, 64, dtype=torch.bfloat16).cuda()
    ctx.cache_write(cache, x, x, torch.tensor([32, -1, 1 << 30], dtype=torch.int32).cuda())
    assert torch.equal(before, cache.k) and ctx.get_status() == ngs.STATUS_CAPACITY
    cache.table[1, 0] = cache.n_pages
    ctx.cache_write(cache, x, x, torch.zeros(3, dtype=torch.int32).cuda(), count=torch.tensor([0, 1, -4], dtype=torch.int32).cuda())
    assert torch.equal(before, cache.k) and ctx.get_status() == ngs.STATUS_CAPACITY


@pytest.mark.parametrize("N", [1, 31, 32, 33, 64, 200, 1088, 4096])
def test_tree_mask(ctx, N):
    g = torch.Generator().manual_seed(N)
    j = torch.arange(N).expand(3, N)
    par = (torch.rand(3, N, generator=g) * (j + 1)).long() - 1
    par[1] = j[1] - 1  # one chain
    par[2] = -1        # all roots
    mask, depth = ctx.tree_mask(par.int().cuda())
    if N <= 200:
        assert torch.equal(mask.cpu(), au.pack(au.ancestors(par)))
    chain = torch.tril(torch.ones(N, N, dtype=torch.bool))[None]
    assert torch.equal(mask[1:2].cpu(), au.pack(chain)) and torch.equal(depth[1].cpu(), torch.arange(N).int())
    assert torch.equal(mask[2:].cpu(), au.pack(torch.eye(N, dtype=torch.bool)[None])) and (depth[2] == 0).all()


def test_tree_mask_of_broken_trees(ctx):
    par = torch.tensor([[-1, 0, 2, 2, 1, -7, 9, 5], [-1, 0, 1, 2, 3, 4, 5, 6]], dtype=torch.int32).cuda()
    mask, depth = ctx.tree_mask(par, n_nodes=torch.tensor([8, 3], dtype=torch.int32).cuda())
    assert mask[0, :, 0].tolist() == [1, 3, 0, 0, 0b10011, 0, 0, 0] and depth[0].tolist() == [0, 1, -1, -1, 2, -1, -1, -1]
    assert mask[1, :, 0].tolist() == [1, 3, 7, 0, 0, 0, 0, 0] and depth[1].tolist() == [0, 1, 2, -1, -1, -1, -1, -1]


def test_refusals(ctx):
    import paper_2411_03786_b200 as ngs
    cache, _, _ = au.make_cache(2, 32, 2, 64, 16, False, 9)
    x = torch.ones(2, 3, 2, 64, dtype=torch.bfloat16).cuda()
    st = torch.zeros(2, dtype=torch.int32).cuda()
    bad = [lambda: ctx.cache_write(cache, x[:1], x[:1], st), lambda: ctx.cache_write(cache, x.float(), x.float(), st), lambda: ctx.cache_write(cache, x, x, st.long()),
           lambda: ctx.cache_write(cache, x, x, st, nodes=st), lambda: ctx.cache_write(cache, x, x, st, rope=ngs.Rope(freqs(128))),
           lambda: ctx.cache_read(cache, st[:1], 3), lambda: ctx.rope_rows(ngs.Rope(freqs(24)), x, None, torch.zeros(2, 3).int().cuda()),
           lambda: ctx.rope_rows(ngs.Rope(freqs(64)), x, None, st), lambda: ctx.rope_rows(ngs.Rope(freqs(64)), x[..., :40], None, torch.zeros(2, 3).int().cuda()),
           lambda: ngs.Rope(freqs(64).double()), lambda: ctx.tree_mask(torch.zeros(1, 4097, dtype=torch.int32).cuda()), lambda: ctx.tree_mask(st.long()[None])]
    for f in bad:
        with pytest.raises((ngs.SpecError, IndexError)):
            f()
    assert ctx.get_status() == 0


@pytest.mark.parametrize("D", [64, 128])
def test_attention_and_cache_read_hold_the_same(ctx, D):
    """One key to a sequence: attention gives its value vector as it is.  All finite codes, all scale bytes of the format
    down to 2^-100 (below, products of the smallest codes are not numbers that fp32 holds in full), and those beyond it."""
    import paper_2411_03786_b200 as ngs
    finite = torch.tensor([b for b in range(256) if b & 127 != 127], dtype=torch.uint8)
    per = -(-finite.numel() // D)
    rows = torch.cat([finite, finite[: per * D - finite.numel()]]).view(per, D)
    scales = list(range(27, 135)) + [135, 200, 254, 255]
    S = per * len(scales)
    codes = rows.repeat(len(scales), 1)
    exp = torch.tensor(scales, dtype=torch.uint8).repeat_interleave(per)
    cache = ngs.KVCache.empty(S, 1, 16, D, torch.arange(S, dtype=torch.int32, device="cuda").view(S, 1), True)
    cache.k.zero_(), cache.k_exp.fill_(127), cache.v.fill_(255), cache.v_exp.fill_(255)
    cache.v[:, 0, 0], cache.v_exp[:, 0, 0] = codes.cuda(), exp.cuda()
    zero, one = torch.zeros(S, dtype=torch.int32).cuda(), torch.ones(S, dtype=torch.int32).cuda()
    read = ctx.cache_read(cache, zero, 1)[1][:, 0, 0]
    want = au.dequantise(codes, exp)
    want[exp > 134] = math.nan
    q, kv = torch.ones(S, 1, 2, D).bfloat16().cuda(), torch.ones(S, 1, 1, D).bfloat16().cuda()
    seen = ctx.tree_attention(cache, q, kv, kv, torch.zeros(S, 1, 1, dtype=torch.int32).cuda(), one)[0][:, 0]
    for got in (read, seen[:, 0], seen[:, 1]):
        got = got.double().cpu()
        assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(nan=0.0), want.nan_to_num(nan=0.0))
    # and as keys: a vector that is NaN is NaN to every row
    cache.k_exp.fill_(127), cache.v.zero_(), cache.v_exp.fill_(127)
    cache.k_exp[:, 0, 0] = exp.cuda()
    lse = ctx.tree_attention(cache, q, kv, kv, torch.zeros(S, 1, 1, dtype=torch.int32).cuda(), one, with_lse=True)[1]
    assert torch.equal(lse.isnan().all(-1).flatten().cpu(), exp > 134) and ctx.get_status() == 0
