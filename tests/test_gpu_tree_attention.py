"""Tree attention against a plain 64-bit form: sizes, masks, page layouts and values where it can go wrong."""
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


def block(S, N, Hq, Hkv, D, seed, strided=False):
    g = torch.Generator().manual_seed(seed)
    t = torch.randn(S, N, Hq + 2 * Hkv, D, generator=g).bfloat16()
    if strided:
        t = t.cuda()
        return t[:, :, :Hq], t[:, :, Hq:Hq + Hkv], t[:, :, Hq + Hkv:]
    return tuple(x.contiguous().cuda() for x in (t[:, :, :Hq], t[:, :, Hq:Hq + Hkv], t[:, :, Hq + Hkv:]))


def parents(S, N, kind, seed):
    g = torch.Generator().manual_seed(seed)
    j = torch.arange(N).expand(S, N)
    if kind == "chain":
        return (j - 1).int()
    if kind == "rows":
        return torch.where(j % 5 == 0, -1, j - 1).int()
    up = (torch.rand(S, N, generator=g) * (j + 1)).long() - 1  # anything before the node, or a root
    return torch.where(j == 0, -1, up).int()


# fp32 sums of D products of values around 1, |score| around 10 at most: 2^-24 * D * sum |q k| * scale stays under this
SCORE = 2.0 ** -14


def run(ctx, S, N, Hq, Hkv, D, lens, page, quantised, kind="tree", seed=0, strided=False, live=None, scale=None, tokens=None):
    cache, hk, hv = au.make_cache(S, max(tokens or max(lens), 1), Hkv, D, page, quantised, seed)
    q, k, v = block(S, N, Hq, Hkv, D, seed + 1, strided)
    par = parents(S, N, kind, seed + 2)
    mask = au.ancestors(par)
    nn = None if live is None else torch.tensor(live, dtype=torch.int32).cuda()
    got = ctx.tree_attention(cache, q, k, v, au.pack(mask).cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), n_nodes=nn,
                             scale=scale, with_lse=True)
    ref = au.attention(q, k, v, hk, hv, mask, lens, scale or D ** -0.5, live)
    au.check_attention(got, ref, SCORE)
    assert ctx.get_status() == 0
    return got


@pytest.mark.parametrize("quantised", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("length", [0, 1, 15, 16, 17, 63, 64, 127, 128, 129, 255, 256, 257, 385, 1000])
def test_lengths(ctx, length, D, quantised):
    run(ctx, 1, 5, 4, 2, D, [length], 16, quantised, seed=length)


@pytest.mark.parametrize("quantised", [False, True])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_pages(ctx, page, quantised):
    run(ctx, 3, 9, 6, 2, 128, [page - 1, 3 * page, 2 * page + 5], page, quantised, seed=page)


@pytest.mark.parametrize("N,Hq,Hkv", [(1, 1, 1), (1, 32, 8), (2, 7, 1), (31, 4, 4), (32, 8, 2), (33, 3, 1), (43, 6, 2), (64, 4, 2), (65, 2, 1),
                                      (127, 1, 1), (128, 2, 2), (129, 1, 1), (130, 4, 2), (257, 2, 1), (300, 5, 1)])
@pytest.mark.parametrize("quantised", [False, True])
def test_blocks(ctx, N, Hq, Hkv, quantised):
    """Rows of a tile that are not there, tiles of several heads' rows, masks of one word and of many."""
    run(ctx, 2, N, Hq, Hkv, 64, [70, 200], 32, quantised, seed=N)


@pytest.mark.parametrize("kind", ["chain", "rows", "tree"])
def test_trees(ctx, kind):
    run(ctx, 2, 150, 4, 2, 128, [130, 0], 64, False, kind=kind, seed=5)


@pytest.mark.parametrize("quantised", [False, True])
def test_ragged_batch(ctx, quantised):
    lens = [0, 1, 900, 5, 64, 333, 2, 2000, 128, 0, 77]
    run(ctx, len(lens), 6, 8, 2, 128, lens, 32, quantised, seed=3)


@pytest.mark.parametrize("quantised", [False, True])
@pytest.mark.parametrize("N,Hq,Hkv", [(1, 8, 1), (3, 4, 4), (200, 2, 1)])
def test_long_context_is_split_and_joined(ctx, quantised, N, Hq, Hkv):
    run(ctx, 1, N, Hq, Hkv, 128, [6000 + N], 128, quantised, seed=N)


@pytest.mark.parametrize("quantised", [False, True])
@pytest.mark.parametrize("D,N,Hq,Hkv", [(128, 2, 16, 8), (64, 3, 8, 8), (128, 150, 8, 4)])
def test_many_tiles_per_cta(ctx, quantised, D, N, Hq, Hkv):
    """Some thousand key tiles: every CTA walks several heads and sequences, rings wrap around, contexts end on and off
    tile borders."""
    g = torch.Generator().manual_seed(N)
    S = 40 if N < 100 else 12
    lens = torch.randint(0, 2500, (S,), generator=g)
    lens[::3] = lens[::3] // 128 * 128
    lens[1::7] = lens[1::7] % 300
    run(ctx, S, N, Hq, Hkv, D, lens.tolist(), 64, quantised, seed=N, kind="rows")


def test_strided_projections(ctx):
    run(ctx, 2, 20, 6, 3, 64, [40, 140], 16, False, strided=True)


def test_live_nodes(ctx):
    """Nodes beyond n_nodes give empty rows and are attended by nobody."""
    got = run(ctx, 4, 40, 4, 2, 64, [50, 0, 0, 130], 16, False, live=[40, 1, 0, 17], kind="chain")
    assert (got[0][2] == 0).all() and (got[1][2] == -math.inf).all()


@pytest.mark.parametrize("quantised", [False, True])
def test_live_nodes_over_row_tiles(ctx, quantised):
    """Sequences whose live rows fill three row tiles, end in the third, the second or the first, side by side."""
    run(ctx, 6, 150, 4, 2, 128, [300, 40, 1000, 257, 0, 129], 64, quantised, live=[150, 129, 128, 65, 64, 3], seed=6)


@pytest.mark.parametrize("quantised", [False, True])
@pytest.mark.parametrize("N,Hq,length", [(415, 7, 0), (415, 7, 300), (700, 4, 1), (520, 1, 129), (1100, 1, 64)])
def test_wide_blocks_of_rows(ctx, quantised, N, Hq, length):
    """Blocks of many tiles of which a row attends to one or two, from the front, the middle or the end."""
    run(ctx, 2, N, Hq, 1, 64, [length, length + 200], 32, quantised, kind="rows", seed=N, live=[N, N - 130])


def test_scale_argument(ctx):
    run(ctx, 1, 8, 2, 1, 64, [300], 16, False, scale=0.02)


def test_empty_rows(ctx):
    """No context and a mask without a bit: zeros and -inf; other rows of the tile as usual."""
    S, N, D = 1, 40, 128
    cache, hk, hv = au.make_cache(S, 1, 2, D, 16, False, 0)
    q, k, v = block(S, N, 4, 2, D, 1)
    mask = au.ancestors(parents(S, N, "tree", 2))
    mask[0, 3], mask[0, 17], mask[0, 39] = False, False, False
    lens = torch.zeros(S, dtype=torch.int32).cuda()
    got = ctx.tree_attention(cache, q, k, v, au.pack(mask).cuda(), lens, with_lse=True)
    au.check_attention(got, au.attention(q, k, v, hk, hv, mask, [0], D ** -0.5), SCORE)
    assert (got[0][0, 17] == 0).all() and (got[1][0, 39] == -math.inf).all()


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf, -3.3895313892515355e38])
@pytest.mark.parametrize("length", [0, 5, 129])
def test_masked_places_do_not_count(ctx, bad, length):
    """Non-finite keys and values in nodes that a row does not attend to, in dead nodes and in unused slots of pages."""
    S, N, Hq, Hkv, D = 2, 37, 4, 2, 128
    cache, hk, hv = au.make_cache(S, 200, Hkv, D, 32, False, 7)
    for s in range(S):  # everything from `length` on
        at = torch.arange(length, cache.table.shape[1] * 32)
        pages = cache.table[s].long().cpu()[at // 32]
        cache.k[pages.cuda(), :, (at % 32).cuda()] = bad
        cache.v[pages.cuda(), :, (at % 32).cuda()] = bad
    q, k, v = block(S, N, Hq, Hkv, D, 8)
    live = [30, 37]
    mask = torch.zeros(S, N, N, dtype=torch.bool)
    mask[:, :, :] = torch.eye(N, dtype=torch.bool)
    mask[:, :, 0] = True
    k[0, 5], v[0, 5] = bad, bad      # attended by itself only
    v[1, 36, 0, 3] = bad             # one element, attended by itself only
    k[0, 30:], v[0, 30:] = bad, bad  # dead
    lens = [length] * S
    got = ctx.tree_attention(cache, q, k, v, au.pack(mask).cuda(), torch.tensor(lens, dtype=torch.int32).cuda(),
                             n_nodes=torch.tensor(live, dtype=torch.int32).cuda(), with_lse=True)
    ref = au.attention(q, k, v, hk, hv, mask, lens, D ** -0.5, live)
    clean = torch.ones(S, N, dtype=torch.bool)
    clean[0, 5], clean[1, 36] = False, False
    au.check_attention((got[0].cpu()[clean], got[1].cpu()[clean]), tuple(x[clean] for x in ref), SCORE)
    if not math.isfinite(bad):  # a row that does attend to it shows it
        o = got[0][1, 36, 0, 3].item()
        assert math.isnan(o) if math.isnan(bad) else o == bad
        assert torch.isfinite(got[0][1, 36, 0, 4:]).all() and torch.isfinite(got[0][1, 36, 2:]).all()


def test_quantised_nan_and_garbage_scales(ctx):
    """Unused slots of an E4M3 cache hold anything; a NaN vector in use shows."""
    S, N, D = 1, 3, 128
    cache, hk, hv = au.make_cache(S, 100, 1, D, 16, True, 1)
    at = torch.arange(61, 112)
    pages = cache.table[0].long()[(at // 16).cuda()]
    for t in (cache.k, cache.v):
        t[pages, :, (at % 16).cuda()] = 127
    cache.k_exp[pages, :, (at % 16).cuda()] = 255
    cache.v_exp[pages, :, (at % 16).cuda()] = 255
    q, k, v = block(S, N, 2, 1, D, 2)
    mask = au.ancestors(parents(S, N, "chain", 0))
    args = (q, k, v, au.pack(mask).cuda())
    got = ctx.tree_attention(cache, *args, torch.tensor([61], dtype=torch.int32).cuda(), with_lse=True)
    au.check_attention(got, au.attention(q, k, v, hk, hv, mask, [61], D ** -0.5), SCORE)
    got = ctx.tree_attention(cache, *args, torch.tensor([62], dtype=torch.int32).cuda(), with_lse=True)
    assert got[0].isnan().all()


def test_extreme_scores(ctx):
    """Scores of some thousands: one key takes all the weight, the maximum moves far between tiles."""
    S, N, D, L = 1, 4, 64, 700
    cache, hk, hv = au.make_cache(S, L, 1, D, 64, False, 2)
    q, k, v = block(S, N, 2, 1, D, 3)
    q *= 256
    ramp = torch.linspace(0.1, 3.0, hk.shape[1])[:, None, None]
    flat = (hk * ramp).bfloat16()
    table = cache.table[0].long().cpu()
    for p in range(hk.shape[1] // 64):
        cache.k[table[p]] = flat[0, p * 64:(p + 1) * 64].transpose(0, 1).cuda()
    mask = au.ancestors(parents(S, N, "chain", 0))
    got = ctx.tree_attention(cache, q, k, v, au.pack(mask).cuda(), torch.tensor([L], dtype=torch.int32).cuda(), with_lse=True)
    # scores near 2000: fp32 leaves 2^-24 * 64 * 2000 of them at most
    au.check_attention(got, au.attention(q, k, v, flat.double(), hv, mask, [L], D ** -0.5), 2.0 ** -7)


@pytest.mark.parametrize("quantised", [False, True])
def test_offsets_beyond_32_bits(ctx, quantised):
    """A pool of pages in which bytes (and, in bfloat16, elements) are numbered beyond 2^31: its last pages behave like the first of a small one."""
    import paper_2411_03786_b200 as ngs
    S, N, Hkv, D, page, L = 2, 9, 4, 128, 64, 300
    n_pages = (1 << 16) + 70  # 16.8 million vectors of 128
    per = -(-(L + 3) // page)
    small, _, _ = au.make_cache(S, L + 3, Hkv, D, page, quantised, 3, spare=0)
    table = (small.table.long() + n_pages - S * per).int()
    big = ngs.KVCache.empty(n_pages, Hkv, page, D, table, quantised)
    for a, b in ((small.k, big.k), (small.v, big.v), (small.k_exp, big.k_exp), (small.v_exp, big.v_exp)):
        if a is not None:
            b[n_pages - S * per:] = a
    assert big.k.numel() > 1 << 31
    q, k, v = block(S, N, 8, Hkv, D, 4)
    mask = au.pack(au.ancestors(parents(S, N, "tree", 5))).cuda()
    lens = torch.tensor([L, 130], dtype=torch.int32).cuda()
    out = []
    for c in (small, big):
        a = ctx.tree_attention(c, q, k, v, mask, lens, with_lse=True)
        ctx.cache_write(c, k, v, lens, count=torch.full((S,), 3, dtype=torch.int32).cuda())
        out.append((*a, *ctx.cache_read(c, torch.zeros_like(lens), L + 3)))
    assert all(torch.equal(x, y) for x, y in zip(*out)) and ctx.get_status() == 0


def test_same_result_every_time_and_on_another_stream(ctx):
    cache, _, _ = au.make_cache(3, 3000, 2, 128, 64, True, 4)
    q, k, v = block(3, 50, 8, 2, 128, 5)
    mask = au.pack(au.ancestors(parents(3, 50, "tree", 6))).cuda()
    lens = torch.tensor([3000, 17, 1234], dtype=torch.int32).cuda()
    a = ctx.tree_attention(cache, q, k, v, mask, lens, with_lse=True)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        b = ctx.tree_attention(cache, q, k, v, mask, lens, with_lse=True)
    torch.cuda.current_stream().wait_stream(st)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_inside_a_graph(ctx):
    cache, _, _ = au.make_cache(2, 500, 2, 64, 32, False, 4)
    q, k, v = block(2, 10, 4, 2, 64, 5)
    mask = au.pack(au.ancestors(parents(2, 10, "tree", 6))).cuda()
    lens = torch.tensor([500, 100], dtype=torch.int32).cuda()
    want = ctx.tree_attention(cache, q, k, v, mask, lens, with_lse=True)
    out = tuple(torch.zeros_like(t) for t in want)
    work = torch.empty(ctx._lib.spec_tree_attention_bytes(ctx._h, cache._ref, 2, 10, 4) or 16, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ctx.tree_attention(cache, q, k, v, mask, lens, out=out, work=work)
    for n in (500, 33):  # the lengths are read on the device
        lens[0] = n
        g.replay()
        want = ctx.tree_attention(cache, q, k, v, mask, lens, with_lse=True)
        assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])


def test_bad_lengths_and_pages_set_the_status(ctx):
    import paper_2411_03786_b200 as ngs
    cache, _, _ = au.make_cache(3, 64, 1, 64, 16, False, 4)
    q, k, v = block(3, 2, 1, 1, 64, 5)
    mask = au.pack(au.ancestors(parents(3, 2, "chain", 6))).cuda()
    out = ctx.tree_attention(cache, q, k, v, mask, torch.tensor([64, 65, -1], dtype=torch.int32).cuda(), with_lse=True)
    assert (out[0][1:] == 0).all() and (out[1][1:] == -math.inf).all() and out[0][0].isfinite().all()
    assert ctx.get_status() == ngs.STATUS_CAPACITY
    cache.table[0, 1] = 1 << 30
    cache.table[1, 0] = -1
    ctx.tree_attention(cache, q, k, v, mask, torch.tensor([64, 64, 64], dtype=torch.int32).cuda())
    assert ctx.get_status() == ngs.STATUS_CAPACITY


def test_refusals(ctx):
    import paper_2411_03786_b200 as ngs
    cache, _, _ = au.make_cache(2, 64, 2, 64, 16, False, 4)
    q, k, v = block(2, 3, 4, 2, 64, 5)
    mask = au.pack(au.ancestors(parents(2, 3, "chain", 6))).cuda()
    lens = torch.tensor([64, 3], dtype=torch.int32).cuda()
    ok = lambda **kw: ctx.tree_attention(kw.get("cache", cache), kw.get("q", q), kw.get("k", k), kw.get("v", v), kw.get("mask", mask), kw.get("lens", lens),
                                         scale=kw.get("scale"), work=kw.get("work"))
    ok()
    odd = block(2, 3, 3, 2, 64, 5)[0]
    shifted = torch.empty(2 * 3 * 4 * 64 + 4, dtype=torch.bfloat16, device="cuda")[4:].view(2, 3, 4, 64)
    for kw in ({"q": odd}, {"q": q.float()}, {"q": shifted}, {"q": q.transpose(2, 3).contiguous().transpose(2, 3)}, {"k": k[:, :2]}, {"lens": lens.long()},
               {"mask": mask[:1]}, {"scale": 0.0}, {"scale": math.nan}, {"work": torch.empty(8, dtype=torch.uint8, device="cuda")}, {"lens": lens.cpu()}):
        with pytest.raises(ngs.SpecError):
            ok(**kw)
    with pytest.raises(ngs.SpecError):
        ngs.KVCache(cache.k, cache.v, cache.table, torch.zeros(1, dtype=torch.uint8).cuda(), None)
    for shape in ((4, 2, 8, 64), (4, 2, 16, 96)):  # page and head sizes that no kernel is made for
        t = torch.zeros(shape, dtype=torch.bfloat16, device="cuda")
        c = ngs.KVCache(t, t.clone(), cache.table)
        x = torch.zeros(2, 3, 2, shape[3], dtype=torch.bfloat16, device="cuda")
        with pytest.raises(ngs.SpecError):
            ctx.tree_attention(c, x, x, x, mask, lens)
    assert ctx.get_status() == 0
