"""Forking, extending, freeing and moving the pages of a cache against a plain form, and together with the calls that read and write them."""
import random

import numpy as np
import pytest
import torch

import attn_util as au
import e2m1_util as e4
from pages_util import Pool

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


def tensors(pool):
    return [t for c in pool.caches for t in (c.k, c.v, c.k_exp, c.v_exp, c.k_scale, c.v_scale) if t is not None]


def filled(pool, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    for t in tensors(pool):
        t.view(torch.uint8).copy_(torch.randint(0, 256, t.view(torch.uint8).shape, generator=g, device="cuda", dtype=torch.uint8))
    return pool


def plain(pool):
    as_bytes = [t.view(t.shape[0], -1).view(torch.uint8).cpu().numpy() for t in tensors(pool)]
    return Pool(pool.table.cpu().numpy(), pool.refs.cpu().numpy(), pool.page, as_bytes)


def same(pool, ref, contents=True):
    assert np.array_equal(pool.table.cpu().numpy(), ref.table) and np.array_equal(pool.refs.cpu().numpy(), ref.refs)
    if contents:
        for t, x in zip(tensors(pool), ref.layers):
            assert np.array_equal(t.view(t.shape[0], -1).view(torch.uint8).cpu().numpy(), x)


@pytest.mark.parametrize("bits,layers,heads,D,page", [(16, 1, 1, 64, 16), (8, 3, 2, 128, 32), (4, 2, 3, 64, 16), (4, 20, 1, 128, 64), (16, 2, 8, 128, 128)])
@pytest.mark.parametrize("S,width,n_pages", [(1, 1, 1), (7, 5, 24), (40, 9, 300)])
def test_any_mixture_of_calls(ctx, S, width, n_pages, bits, layers, heads, D, page):
    import paper_2411_03786_b200 as ngs
    rng = random.Random(S * bits + page)
    pool = filled(ngs.PagePool.empty(layers, n_pages, S, width, heads, page, D, bits=bits), 1)
    ref = plain(pool)
    lens = [0] * S
    for step in range(12):
        count = [rng.choice([0, 1, rng.randint(0, 2 * page), rng.randint(0, width * page)]) for _ in range(S)]
        ok = ctx.pages_reserve(pool, i32(lens), i32(count))
        want = ref.reserve(lens, count)
        assert ok.tolist() == want
        assert (ctx.get_status() != 0) == (0 in want)
        lens = [n + c if good else n for n, c, good in zip(lens, count, want)]
        same(pool, ref)
        source = [rng.choice([s, s, rng.randrange(S), -1, S + 3]) for s in range(S)]
        lens = [rng.choice([lens[x], rng.randint(0, lens[x])]) if 0 <= x < S else 0 for x in source]
        asked = [n if 0 <= x < S else 1000 for n, x in zip(lens, source)]
        ctx.pages_assign(pool, i32(source), i32(asked))
        ref.assign(source, asked)
        same(pool, ref, False)
        assert ref.consistent()
        if step % 2:
            assert ctx.pages_compact(pool).tolist() == [ref.compact()]
            same(pool, ref)
    assert ctx.get_status() == 0


def test_many_sequences_and_a_large_pool(ctx):
    """Rows beyond what a CTA has side by side, more pages than threads, free pages far apart."""
    import paper_2411_03786_b200 as ngs
    S, width, n_pages = 5000, 12, 70001
    rng = np.random.default_rng(3)
    table = np.full((S, width), -1, np.int32)
    have = rng.integers(0, width, S)
    pages = rng.permutation(n_pages)[: have.sum()]
    table[np.arange(width) < have[:, None]] = pages
    t = torch.from_numpy(table).cuda()
    pool = filled(ngs.PagePool([ngs.KVCache.empty(n_pages, 1, 16, 64, t, bits=4)]), 2)
    ref = plain(pool)
    source = np.where(rng.random(S) < 0.5, rng.integers(0, S, S), np.arange(S)).astype(np.int32)
    lens = (have[source] * 16 - rng.integers(0, 16, S)).clip(0).astype(np.int32)
    ctx.pages_assign(pool, i32(source), i32(lens))
    ref.assign(source, lens)
    same(pool, ref, False)
    count = rng.integers(0, 17, S).astype(np.int32)
    assert ctx.pages_reserve(pool, i32(lens), i32(count)).tolist() == ref.reserve(lens.tolist(), count.tolist())
    same(pool, ref)
    assert ctx.pages_compact(pool).item() == ref.compact()
    same(pool, ref)
    assert ctx.pages_compact(pool).item() == (ref.refs > 0).sum()  # nothing is left to do
    same(pool, ref)
    assert ctx.get_status() == 0


def test_one_long_row(ctx):
    """A prompt of many pages for one sequence, beside a pool in which every second page is taken."""
    import paper_2411_03786_b200 as ngs
    n_pages, width = 6000, 2500
    table = torch.full((2, width), -1, dtype=torch.int32)
    table[1, :] = torch.arange(width) * 2
    pool = filled(ngs.PagePool([ngs.KVCache.empty(n_pages, 1, 16, 64, table.cuda())]), 2)
    ref = plain(pool)
    assert ctx.pages_reserve(pool, i32([3, 0]), i32([16 * width - 3, 0])).tolist() == ref.reserve([3, 0], [16 * width - 3, 0]) == [1, 1]
    same(pool, ref)
    assert ctx.pages_compact(pool).item() == ref.compact() == 2 * width
    same(pool, ref)


def test_pool_that_runs_out(ctx):
    """Rows are served in order until one needs more than is left; that one and all later ones that need pages stay as they are."""
    import paper_2411_03786_b200 as ngs
    pool = ngs.PagePool.empty(1, 6, 5, 4, 1, 16, 64)
    ok = ctx.pages_reserve(pool, i32([0, 0, 0, 0, 0]), i32([32, 16, 64, 16, 0]))
    assert ok.tolist() == [1, 1, 0, 0, 1] and ctx.get_status() == ngs.STATUS_CAPACITY
    assert pool.table[2:].eq(-1).all() and pool.refs.tolist() == [1, 1, 1, 0, 0, 0]
    for start, count in (([0, 0, 60, -1, 0], [0, 0, 5, 1, -1]),):  # beyond a row, before it, less than nothing
        assert ctx.pages_reserve(pool, i32(start), i32(count)).tolist() == [1, 1, 0, 0, 0]
        assert ctx.get_status() == ngs.STATUS_CAPACITY and pool.refs.tolist() == [1, 1, 1, 0, 0, 0]
    assert ctx.pages_reserve(pool, i32([0, 0, 0, 2147483600, 0]), i32([0, 0, 0, 2147483600, 0])).tolist() == [1, 1, 1, 0, 1]
    assert ctx.get_status() == ngs.STATUS_CAPACITY


def test_held_pages_are_not_given_away(ctx):
    """A holder of the caller's own keeps a page, and makes others copy it."""
    import paper_2411_03786_b200 as ngs
    pool = filled(ngs.PagePool.empty(1, 4, 2, 2, 1, 16, 64), 1)
    ctx.pages_reserve(pool, i32([0, 0]), i32([10, 0]))
    pool.refs[0] += 1  # the prompt is kept
    was = pool.caches[0].k[0].clone()
    assert ctx.pages_reserve(pool, i32([10, 0]), i32([1, 16])).tolist() == [1, 1]
    assert pool.table.tolist() == [[1, -1], [2, -1]] and pool.refs.tolist() == [1, 1, 1, 0]
    assert torch.equal(pool.caches[0].k[1].view(torch.uint8), was.view(torch.uint8))
    ctx.pages_assign(pool, i32([-1, -1]), i32([5, 5]))
    assert pool.refs.tolist() == [1, 0, 0, 0] and ctx.pages_compact(pool).item() == 1


def test_copies(ctx):
    import paper_2411_03786_b200 as ngs
    pool = filled(ngs.PagePool.empty(3, 50, 1, 1, 2, 32, 128, bits=8), 5)
    ref = plain(pool)
    order = torch.randperm(50, generator=torch.Generator().manual_seed(1)).int()
    src, dst = order[:20].contiguous(), order[20:40].contiguous()
    ctx.pages_copy(pool, src.cuda(), dst.cuda(), n=i32([13]))
    ref.copy(list(zip(src.tolist()[:13], dst.tolist()[:13])))
    same(pool, ref)
    ctx.pages_copy(pool, i32([3, -1, 50, 7]), i32([3, 5, 6, 1 << 30]))  # itself, and pairs that are not in the pool
    same(pool, ref)
    assert ctx.get_status() == ngs.STATUS_CAPACITY
    ctx.pages_copy(pool, i32([])[:0], i32([])[:0])
    one = order[40:41].expand(9).contiguous().cuda()  # one page to many
    ctx.pages_copy(pool, one, order[41:50].contiguous().cuda())
    ref.copy([(int(order[40]), int(d)) for d in order[41:50]])
    same(pool, ref)


def test_samples_of_a_prompt(ctx):
    """A prompt in a cache of 4 bits, three samples of it that go on differently, one that is dropped, the rest moved together: each
    sequence's attention is that over its own tokens."""
    import paper_2411_03786_b200 as ngs
    S, Hq, Hkv, D, page, L = 4, 8, 2, 128, 16, 45
    g = torch.Generator().manual_seed(0)
    pool = ngs.PagePool.empty(2, 40, S, 8, Hkv, page, D, bits=4)
    for t in tensors(pool):
        t.fill_(255)  # whatever is not written reads as NaN
    ctx.pages_assign(pool, i32([-1] * S), i32([0] * S))
    new = lambda n: [torch.randn(S, n, Hkv, D, generator=g).bfloat16().cuda() for _ in range(4)]
    held = [[[torch.zeros(0, Hkv, D, dtype=torch.float64) for _ in range(S)] for _ in "kv"] for _ in range(2)]
    lens = [0] * S

    def extend(n, count):
        assert ctx.pages_reserve(pool, i32(lens), i32(count)).tolist() == [1] * S
        x = new(n)
        for layer in range(2):
            k, v = x[2 * layer], x[2 * layer + 1]
            ctx.cache_write(pool.caches[layer], k, v, i32(lens), count=i32(count))
            for which, t in enumerate((k, v)):
                q = e4.dequantise(*e4.quantise(t))
                for s in range(S):
                    held[layer][which][s] = torch.cat([held[layer][which][s], q[s, : count[s]]])
        for s in range(S):
            lens[s] += count[s]

    def assign(source, keep):
        ctx.pages_assign(pool, i32(source), i32(keep))
        for layer in range(2):
            for which in range(2):
                held[layer][which] = [held[layer][which][x][:n] if x >= 0 else held[layer][which][0][:0] for x, n in zip(source, keep)]
        lens[:] = keep

    def check():
        q = torch.randn(S, 3, Hq, D, generator=g).bfloat16().cuda()
        k, v = (torch.randn(S, 3, Hkv, D, generator=g).bfloat16().cuda() for _ in range(2))
        mask = torch.ones(S, 3, 3).tril().bool()
        for layer in range(2):
            got = ctx.tree_attention(pool.caches[layer], q, k, v, au.pack(mask).cuda(), i32(lens), with_lse=True)
            width = max(max(lens), 1)
            hk, hv = (torch.stack([torch.cat([x, torch.zeros(width - len(x), Hkv, D, dtype=torch.float64)]) for x in h]) for h in held[layer])
            au.check_attention(got, au.attention(q, k, v, hk, hv, mask, lens, D ** -0.5), 2.0 ** -14)

    extend(L, [L, 0, 0, 0])
    check()
    assign([0, 0, 0, 0], [L, L, L, L - 20])
    assert int(pool.refs.max()) == 4 and int((pool.refs > 0).sum()) == 3
    extend(9, [0, 9, 1, 6])
    check()
    assign([3, -1, 2, 1], [L - 14, 0, L + 1, L + 9])
    check()
    before = int((pool.refs > 0).sum())
    assert ctx.pages_compact(pool).item() == before and (pool.refs[:before] > 0).all()
    check()
    extend(30, [30, 30, 0, 7])
    check()
    assert ctx.get_status() == 0


def test_inside_a_graph_and_on_another_stream(ctx):
    """A captured step decides anew with every replay; two captured steps share a workspace one after the other."""
    import paper_2411_03786_b200 as ngs
    S = 6
    pool = filled(ngs.PagePool.empty(2, 64, S, 8, 1, 16, 64, bits=4), 1)
    ref = plain(pool)
    start, count = i32([0] * S), i32([20] * S)
    source, keep = i32(list(range(S))), i32([100] * S)
    ok, live = torch.zeros(S, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    work = torch.empty(1 << 16, dtype=torch.uint8, device="cuda")
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    torch.cuda.synchronize()
    with torch.cuda.graph(graphs[0], stream=st):
        ctx.pages_assign(pool, source, keep)
        ctx.pages_reserve(pool, start, count, out=ok, work=work)
    with torch.cuda.graph(graphs[1], stream=st):
        ctx.pages_compact(pool, out=live, work=work)
    same(pool, ref)  # capturing runs nothing
    for step in range(5):
        lens = [20 * step - 7 * ((s + step) % 2) for s in range(S)] if step else [0] * S
        src = [(s + step) % S for s in range(S)]
        source.copy_(i32(src)), keep.copy_(i32(lens)), start.copy_(i32(lens))
        with torch.cuda.stream(st):
            st.wait_stream(torch.cuda.current_stream())
            graphs[0].replay()
            graphs[1].replay()
        torch.cuda.current_stream().wait_stream(st)
        ref.assign(src, lens)
        assert ok.tolist() == ref.reserve(lens, [20] * S) and live.tolist() == [ref.compact()]
        same(pool, ref)
    ctx.get_status()


def test_empty_calls_and_refusals(ctx):
    import paper_2411_03786_b200 as ngs
    e = i32([])[:0]
    pool = ngs.PagePool.empty(1, 3, 0, 2, 1, 16, 64)
    ctx.pages_assign(pool, e, e)
    assert ctx.pages_reserve(pool, e, e).shape == (0,) and ctx.pages_compact(pool).tolist() == [0]
    pool = ngs.PagePool.empty(2, 3, 2, 2, 1, 16, 64)
    z = i32([0, 0])
    for call in (lambda: ctx.pages_assign(pool, z[:1], z), lambda: ctx.pages_assign(pool, z, z.long()), lambda: ctx.pages_reserve(pool, z.cpu(), z),
                 lambda: ctx.pages_reserve(pool, z, z, out=z.long()), lambda: ctx.pages_reserve(pool, z, z, work=torch.empty(8, dtype=torch.uint8, device="cuda")),
                 lambda: ctx.pages_compact(pool, out=z), lambda: ctx.pages_copy(pool, z, z[:1]), lambda: ctx.pages_copy(pool, z, z, n=z)):
        with pytest.raises(ngs.SpecError):
            call()
    a, b = pool.caches
    other = ngs.KVCache.empty(3, 1, 16, 64, b.table.clone())
    more = ngs.KVCache.empty(4, 1, 16, 64, a.table)
    for caches, refs in (([], None), ([a, other], None), ([a, more], None), ([a], pool.refs[:2]), ([a], pool.refs.long()), ([a], pool.refs.cpu())):
        with pytest.raises(ngs.SpecError):
            ngs.PagePool(caches, refs)
    with pytest.raises(ngs.SpecError):
        big = ngs.PagePool([a] * 129, pool.refs)
        ctx.pages_compact(big)
    assert ctx.get_status() == 0
