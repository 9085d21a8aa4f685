"""Tree attention over a cache of 4 bits against a plain 64-bit form: sizes, masks, page layouts and values where it can go wrong."""
import math

import pytest
import torch

import attn_util as au
import e2m1_util as e4
from test_gpu_tree_attention import SCORE, block, parents

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    import paper_2411_03786_b200 as ngs
    w = torch.zeros(64, 64, dtype=torch.bfloat16, device="cuda")
    c = ngs.SpecContext(w, w)
    yield c
    c.close()


def i32(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


def with_small_weights(ref, held_v, v):
    """Weights for the cached values are held in half precision with the largest at 2^6 or more: below 2^-14 they are off by up to
    2^-25, which is 2^-31 of the largest weight, which is at most 1 of their sum.  So an output is off by up to 2^-31 of the sum of all |v|, which
    counts where the values that matter are 0.  `check_attention` allows 2^-8 of the magnitude."""
    S, _, Hq, _ = ref[0].shape
    total = held_v.abs().sum(1) + v.double().cpu().abs().sum(1)  # [S, heads, D]
    return ref[0], ref[1], ref[2] + 2.0 ** (8 - 31) * total.repeat_interleave(Hq // v.shape[2], 1)[:, None]


def run(ctx, S, N, Hq, Hkv, D, lens, page, kind="tree", seed=0, strided=False, live=None, scale=None, gain=1.0, bound=SCORE):
    cache, hk, hv = e4.make_cache(S, max(max(lens), 1), Hkv, D, page, seed, gain=gain)
    q, k, v = block(S, N, Hq, Hkv, D, seed + 1, strided)
    mask = au.ancestors(parents(S, N, kind, seed + 2))
    got = ctx.tree_attention(cache, q, k, v, au.pack(mask).cuda(), i32(lens), n_nodes=None if live is None else i32(live), scale=scale, with_lse=True)
    au.check_attention(got, au.attention(q, k, v, hk, hv, mask, lens, scale or D ** -0.5, live), bound)
    assert ctx.get_status() == 0
    return got


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("N,Hq", [(1, 2), (5, 4), (12, 8), (40, 4)])
@pytest.mark.parametrize("length", [0, 1, 15, 16, 17, 63, 64, 127, 128, 129, 255, 256, 257, 385, 1000])
def test_lengths(ctx, length, N, Hq, D):
    run(ctx, 1, N, Hq, 2, D, [length], 16, seed=length)


@pytest.mark.parametrize("N", [2, 20])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_pages(ctx, page, N):
    run(ctx, 3, N, 6, 2, 128, [page - 1, 3 * page, 2 * page + 5], page, seed=page)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("N,Hq,Hkv", [(1, 1, 1), (1, 32, 8), (1, 16, 1), (1, 17, 1), (1, 64, 2), (2, 7, 1), (3, 8, 2), (4, 4, 1), (5, 13, 1), (8, 1, 1), (9, 1, 1), (16, 2, 2), (17, 1, 1),
                                      (31, 4, 4), (32, 8, 2), (33, 3, 1), (43, 6, 2), (64, 4, 2), (65, 2, 1), (127, 1, 1), (128, 2, 2), (129, 1, 1), (130, 4, 2), (257, 2, 1), (300, 5, 1)])
def test_blocks(ctx, N, Hq, Hkv, D):
    """Rows of a tile that are not there, tiles of several heads' rows, masks of one word and of many."""
    run(ctx, 2, N, Hq, Hkv, D, [70, 200], 32, seed=N)


@pytest.mark.parametrize("N", [1, 2, 6, 60])
def test_ragged_batch(ctx, N):
    lens = [0, 1, 900, 5, 64, 333, 2, 2000, 128, 0, 77]
    run(ctx, len(lens), N, 8, 2, 128, lens, 32, seed=3)


@pytest.mark.parametrize("N,Hq,Hkv", [(1, 8, 1), (1, 4, 4), (3, 4, 4), (2, 16, 2), (200, 2, 1)])
def test_long_context_is_split_and_joined(ctx, N, Hq, Hkv):
    run(ctx, 1, N, Hq, Hkv, 128, [6000 + N], 128, seed=N)


@pytest.mark.parametrize("D,N,Hq,Hkv", [(128, 1, 16, 8), (128, 2, 16, 8), (64, 3, 8, 8), (128, 150, 8, 4)])
def test_many_tiles_per_cta(ctx, D, N, Hq, Hkv):
    """Every CTA walks several heads and sequences, rings wrap around, contexts end on and off tile borders."""
    g = torch.Generator().manual_seed(N)
    S = 40 if N < 100 else 12
    lens = torch.randint(0, 2500, (S,), generator=g)
    lens[::3] = lens[::3] // 128 * 128
    lens[1::7] = lens[1::7] % 300
    run(ctx, S, N, Hq, Hkv, D, lens.tolist(), 64, seed=N, kind="rows")


@pytest.mark.parametrize("N", [4, 20])
def test_strided_projections(ctx, N):
    run(ctx, 2, N, 6, 3, 64, [40, 140], 16, strided=True)


@pytest.mark.parametrize("N,live", [(40, [40, 1, 0, 17]), (6, [6, 1, 0, 3])])
def test_live_nodes(ctx, N, live):
    """Nodes beyond n_nodes give empty rows and are attended by nobody."""
    got = run(ctx, 4, N, 4, 2, 64, [50, 0, 0, 130], 16, live=live, kind="chain")
    assert (got[0][2] == 0).all() and (got[1][2] == -math.inf).all()


@pytest.mark.parametrize("N", [8, 40])
def test_scale_argument(ctx, N):
    run(ctx, 1, N, 2, 1, 64, [300], 16, scale=0.02)


@pytest.mark.parametrize("N,Hq,length", [(415, 7, 0), (700, 4, 1), (1100, 1, 64)])
def test_wide_blocks_of_rows(ctx, N, Hq, length):
    """Blocks of many tiles of which a row attends to one or two, from the front, the middle or the end."""
    run(ctx, 2, N, Hq, 1, 64, [length, length + 200], 32, kind="rows", seed=N, live=[N, N - 130])


@pytest.mark.parametrize("D,N", [(64, 9), (128, 5), (64, 2)])
def test_rows_on_both_sides_of_the_two_forms(ctx, D, N):
    """One row tile, two, and the first sizes that the form for many rows takes."""
    for Hq in (7, 8, 9):
        run(ctx, 2, N, Hq, 1, D, [333, 40], 16, seed=Hq)
    run(ctx, 3, 1, 16 if D == 128 else 32, 1, D, [333, 0, 16], 16, seed=3)
    run(ctx, 3, 1, 17 if D == 128 else 33, 1, D, [333, 0, 16], 16, seed=3)


@pytest.mark.parametrize("N", [5, 40])
def test_empty_rows(ctx, N):
    """No context and a mask without a bit: zeros and -inf; other rows of the tile as usual."""
    S, D = 1, 128
    cache, hk, hv = e4.make_cache(S, 1, 2, D, 16, 0)
    q, k, v = block(S, N, 4, 2, D, 1)
    mask = au.ancestors(parents(S, N, "tree", 2))
    mask[0, 1], mask[0, N - 1] = False, False
    got = ctx.tree_attention(cache, q, k, v, au.pack(mask).cuda(), i32([0]), with_lse=True)
    au.check_attention(got, au.attention(q, k, v, hk, hv, mask, [0], D ** -0.5), SCORE)
    assert (got[0][0, 1] == 0).all() and (got[1][0, N - 1] == -math.inf).all()


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf, -3.3895313892515355e38])
@pytest.mark.parametrize("N", [7, 37])
@pytest.mark.parametrize("length", [0, 5, 129])
def test_masked_places_do_not_count(ctx, bad, N, length):
    """Non-finite keys and values in nodes that a row does not attend to, in dead nodes and in unused slots of pages."""
    S, Hq, Hkv, D = 2, 4, 2, 128
    cache, hk, hv = e4.make_cache(S, 200, Hkv, D, 32, 7)
    for s in range(S):  # everything from `length` on reads as NaN
        at = torch.arange(length, cache.table.shape[1] * 32)
        pages = cache.table[s].long().cpu()[at // 32]
        cache.k_scale[pages.cuda(), :, (at % 32).cuda()] = 255
        cache.v_scale[pages.cuda(), :, (at % 32).cuda()] = 255
    q, k, v = block(S, N, Hq, Hkv, D, 8)
    live = [N - 2, N]
    mask = torch.eye(N, dtype=torch.bool).expand(S, N, N).clone()
    mask[:, :, 0] = True
    k[0, 2], v[0, 2] = bad, bad              # attended by itself only
    v[1, N - 1, 0, 3] = bad                  # one element, attended by itself only
    k[0, N - 2:], v[0, N - 2:] = bad, bad    # dead
    got = ctx.tree_attention(cache, q, k, v, au.pack(mask).cuda(), i32([length] * S), n_nodes=i32(live), with_lse=True)
    ref = au.attention(q, k, v, hk, hv, mask, [length] * S, D ** -0.5, live)
    clean = torch.ones(S, N, dtype=torch.bool)
    clean[0, 2], clean[1, N - 1] = False, False
    au.check_attention((got[0].cpu()[clean], got[1].cpu()[clean]), tuple(x[clean] for x in ref), SCORE)
    if not math.isfinite(bad):  # a row that does attend to it shows it
        o = got[0][1, N - 1, 0, 3].item()
        assert math.isnan(o) if math.isnan(bad) else o == bad
        assert torch.isfinite(got[0][1, N - 1, 0, 4:]).all() and torch.isfinite(got[0][1, N - 1, 2:]).all()


@pytest.mark.parametrize("N", [3, 40])
def test_nan_in_the_context_shows(ctx, N):
    S, D = 2, 128
    cache, hk, hv = e4.make_cache(S, 100, 1, D, 16, 1)
    q, k, v = block(S, N, 2, 1, D, 2)
    mask = au.ancestors(parents(S, N, "chain", 0))
    page = int(cache.table[0, 3])
    cache.v_scale[page, 0, 13, 2] = 230  # position 61, elements 32 to 47
    args = (q, k, v, au.pack(mask).cuda())
    got = ctx.tree_attention(cache, *args, i32([61, 61]), with_lse=True)
    au.check_attention(got, au.attention(q, k, v, hk, hv, mask, [61, 61], D ** -0.5), SCORE)
    got = ctx.tree_attention(cache, *args, i32([62, 62]), with_lse=True)
    assert got[0][0, :, :, 32:48].isnan().all() and got[0][0, :, :, :32].isfinite().all() and got[0][0, :, :, 48:].isfinite().all() and got[0][1].isfinite().all()
    cache.k_scale[page, 0, 13, 2] = 255
    got = ctx.tree_attention(cache, *args, i32([62, 62]), with_lse=True)
    assert got[0][0].isnan().all() and got[0][1].isfinite().all()


@pytest.mark.parametrize("N", [1, 4, 40])
@pytest.mark.parametrize("gain", [2.0 ** -15, 2.0 ** -9, 300.0])
def test_small_and_large_values(ctx, gain, N):
    """Scales from the smallest to the largest of the format; queries of a size that keeps the scores around 1."""
    S, Hq, D, L = 1, 2, 64, 500
    cache, hk, hv = e4.make_cache(S, L, 1, D, 64, 2, gain=gain)
    q, k, v = block(S, N, Hq, 1, D, 3)
    k, v = k * gain, v * gain
    mask = au.ancestors(parents(S, N, "chain", 0))
    got = ctx.tree_attention(cache, q, k, v, au.pack(mask).cuda(), i32([L]), scale=D ** -0.5 / gain, with_lse=True)
    au.check_attention(got, au.attention(q, k, v, hk, hv, mask, [L], D ** -0.5 / gain), SCORE)


@pytest.mark.parametrize("N", [1, 4, 40])
@pytest.mark.parametrize("size", [1e-30, 1e30])
def test_queries_of_any_size(ctx, size, N):
    S, Hq, D, L = 1, 3, 128, 300
    cache, hk, hv = e4.make_cache(S, L, 1, D, 64, 2)
    q, k, v = block(S, N, Hq, 1, D, 3)
    q = (q.double() * size).bfloat16()
    q[0, 0, 1] = 0
    scale = float(torch.tensor(D ** -0.5 / size, dtype=torch.float32))
    mask = au.ancestors(parents(S, N, "chain", 0))
    got = ctx.tree_attention(cache, q, k, v, au.pack(mask).cuda(), i32([L]), scale=scale, with_lse=True)
    au.check_attention(got, au.attention(q, k, v, hk, hv, mask, [L], scale), SCORE)


@pytest.mark.parametrize("N", [1, 4, 40])
def test_extreme_scores(ctx, N):
    """Scores of some thousands: one key takes all the weight, the maximum moves far between tiles."""
    import paper_2411_03786_b200 as ngs
    S, D, L = 1, 64, 700
    g = torch.Generator().manual_seed(2)
    ramp = torch.linspace(0.1, 3.0, 704)[:, None, None]
    x = (torch.randn(704, 1, D, generator=g) * ramp).bfloat16()
    y = torch.randn(704, 1, D, generator=g).bfloat16()
    parts = [e4.quantise(t.view(11, 64, 1, D).transpose(1, 2)) for t in (x, y)]
    cache = ngs.KVCache(parts[0][0].cuda(), parts[1][0].cuda(), torch.arange(11, dtype=torch.int32, device="cuda").view(1, 11), k_scale=parts[0][1].cuda(), v_scale=parts[1][1].cuda())
    hk, hv = (e4.dequantise(*p).transpose(1, 2).reshape(1, 704, 1, D) for p in parts)
    q, k, v = block(S, N, 2, 1, D, 3)
    q *= 256
    mask = au.ancestors(parents(S, N, "chain", 0))
    got = ctx.tree_attention(cache, q, k, v, au.pack(mask).cuda(), i32([L]), with_lse=True)
    # scores near 2000: fp32 leaves 2^-24 * 64 * 2000 of them at most
    au.check_attention(got, with_small_weights(au.attention(q, k, v, hk, hv, mask, [L], D ** -0.5), hv, v), 2.0 ** -7)


@pytest.mark.parametrize("N", [2, 40])
def test_offsets_beyond_32_bits(ctx, N):
    """A pool whose elements are numbered beyond 2^32 and bytes beyond 2^31: its last pages behave like the first of a small one."""
    import paper_2411_03786_b200 as ngs
    S, Hkv, D, page, L = 2, 4, 128, 64, 300
    n_pages = (1 << 17) + 70  # 33.5 million vectors of 128
    per = -(-(L + 3) // page)
    small, _, _ = e4.make_cache(S, L + 3, Hkv, D, page, 3, spare=0)
    big = ngs.KVCache.empty(n_pages, Hkv, page, D, (small.table.long() + n_pages - S * per).int(), bits=4)
    for a, b in ((small.k, big.k), (small.v, big.v), (small.k_scale, big.k_scale), (small.v_scale, big.v_scale)):
        b[n_pages - S * per:] = a
    assert big.k.numel() > 1 << 31
    q, k, v = block(S, N, 8, Hkv, D, 4)
    mask = au.pack(au.ancestors(parents(S, N, "tree", 5))).cuda()
    lens = i32([L, 130])
    out = []
    for c in (small, big):
        a = ctx.tree_attention(c, q, k, v, mask, lens, with_lse=True)
        ctx.cache_write(c, k, v, lens, count=torch.full((S,), 2, dtype=torch.int32).cuda())
        out.append((*a, *ctx.cache_read(c, torch.zeros_like(lens), L + 3)))
    assert all(torch.equal(x, y) for x, y in zip(*out)) and ctx.get_status() == 0


@pytest.mark.parametrize("N", [1, 50])
def test_same_result_every_time_on_another_stream_and_in_a_graph(ctx, N):
    cache, _, _ = e4.make_cache(3, 3000, 2, 128, 64, 4)
    q, k, v = block(3, N, 8, 2, 128, 5)
    mask = au.pack(au.ancestors(parents(3, N, "tree", 6))).cuda()
    lens = i32([3000, 17, 1234])
    a = ctx.tree_attention(cache, q, k, v, mask, lens, with_lse=True)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        b = ctx.tree_attention(cache, q, k, v, mask, lens, with_lse=True)
    torch.cuda.current_stream().wait_stream(st)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    out = tuple(torch.zeros_like(t) for t in a)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ctx.tree_attention(cache, q, k, v, mask, lens, out=out)
    for n in (3000, 33):  # the lengths are read on the device
        lens[0] = n
        g.replay()
        want = ctx.tree_attention(cache, q, k, v, mask, lens, with_lse=True)
        assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])


@pytest.mark.parametrize("N", [2, 40])
@pytest.mark.parametrize("length", [64, 61, 33])
def test_missing_pages_and_bad_lengths(ctx, N, length):
    """Positions in pages that are not in the pool are left out; a length that the pages cannot hold gives empty rows."""
    import paper_2411_03786_b200 as ngs
    cache, hk, hv = e4.make_cache(4, 64, 1, 64, 16, 4)
    q, k, v = block(4, N, 2, 1, 64, 5)
    mask = au.ancestors(parents(4, N, "chain", 6))
    cache.table[0, 1], cache.table[3, 0], cache.table[3, 1] = 1 << 30, -1, cache.n_pages
    got = ctx.tree_attention(cache, q, k, v, au.pack(mask).cuda(), i32([length, 65, -1, length]), with_lse=True)
    assert ctx.get_status() == ngs.STATUS_CAPACITY
    assert (got[0][1:3] == 0).all() and (got[1][1:3] == -math.inf).all()
    for s, gone in ((0, range(16, 32)), (3, range(32))):
        keep = [p for p in range(length) if p not in gone]
        ref = au.attention(q[s:s + 1], k[s:s + 1], v[s:s + 1], hk[s:s + 1, keep], hv[s:s + 1, keep], mask[s:s + 1], [len(keep)], 64 ** -0.5)
        au.check_attention((got[0][s:s + 1], got[1][s:s + 1]), ref, SCORE)
