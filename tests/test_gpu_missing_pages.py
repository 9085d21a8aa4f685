"""Pages that are not in the pool: attention leaves their positions out, whatever lies in the pool's other pages."""
import math

import pytest
import torch

import attn_util as au

pytestmark = pytest.mark.gpu
SCORE = 2.0 ** -14  # fp32 sums of products around 1, as in the tests of whole caches


@pytest.fixture(scope="module")
def ctx():
    import paper_2411_03786_b200 as ngs
    w = torch.zeros(64, 64, dtype=torch.bfloat16, device="cuda")
    c = ngs.SpecContext(w, w)
    yield c
    c.close()


def without(held, lens, page, missing):
    """The positions that are left, packed together: [S, tokens, heads, D] and their numbers."""
    out, n = torch.zeros_like(held), []
    for s, length in enumerate(lens):
        at = torch.tensor([i for i in range(length) if i // page not in missing[s]], dtype=torch.long)
        out[s, : at.numel()] = held[s, at]
        n.append(at.numel())
    return out, n


@pytest.mark.parametrize("quantised", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("page,lens,missing", [
    (16, [300, 17, 40], [{0, 3, 4, 18}, {1}, set()]),     # first, inside a tile, the last and partial one
    (16, [1000, 16, 0], [set(range(8, 16)), {0}, {0}]),   # a whole tile; all of a sequence; none of its positions
    (32, [900, 65, 31], [{5, 27, 28}, {0, 1, 2}, set()]),
    (64, [700, 129, 64], [{0}, {2}, {0}]),
    (128, [3000, 128, 200], [{0, 11, 23}, {0}, {1}]),
])
def test_their_positions_are_left_out(ctx, page, lens, missing, D, quantised):
    import paper_2411_03786_b200 as ngs
    S, N, Hq, Hkv = 3, 9, 6, 2
    cache, hk, hv = au.make_cache(S, max(lens), Hkv, D, page, quantised, page + D)
    if quantised:  # (a page that the table does not name holds vectors that read as NaN)
        free = [p for p in range(cache.n_pages) if p not in set(cache.table.flatten().tolist())]
        swap = cache.table == 0  # page 0 is made one of them
        for t in (cache.k, cache.v, cache.k_exp, cache.v_exp):
            t[free[0]] = t[0]
        cache.table[swap] = free[0]
        cache.k_exp[0], cache.v_exp[0] = 255, 255
    numbers = [cache.n_pages, -1, 1 << 30, -(1 << 31)]
    i = 0
    for s, m in enumerate(missing):
        for p in m:
            cache.table[s, p] = numbers[i % 4]
            i += 1
    g = torch.Generator().manual_seed(D)
    q, k, v = (torch.randn(S, N, h, D, generator=g).bfloat16().cuda() for h in (Hq, Hkv, Hkv))
    mask = au.ancestors(torch.where(torch.arange(N) % 4 == 0, -1, torch.arange(N) - 1).int().expand(S, N))
    mask[1, 2] = False  # where the context is gone too, an empty row
    got = ctx.tree_attention(cache, q, k, v, au.pack(mask).cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), with_lse=True)
    named = any(p * page < lens[s] for s, m in enumerate(missing) for p in m)
    assert named and ctx.get_status() == ngs.STATUS_CAPACITY
    (hk, left), (hv, _) = without(hk, lens, page, missing), without(hv, lens, page, missing)
    au.check_attention(got, au.attention(q, k, v, hk, hv, mask, left, D ** -0.5), SCORE)
    if left[1] == 0:
        assert (got[0][1, 2] == 0).all() and (got[1][1, 2] == -math.inf).all()


@pytest.mark.parametrize("quantised", [False, True])
def test_over_many_ctas_and_rings(ctx, quantised):
    """Long and ragged: missing pages in some of a CTA's segments and not in the next, joins of partly missing contexts."""
    import paper_2411_03786_b200 as ngs
    S, N, Hq, Hkv, D, page = 24, 2, 8, 8, 128, 64
    g = torch.Generator().manual_seed(9)
    lens = torch.randint(1, 2500, (S,), generator=g).tolist()
    cache, hk, hv = au.make_cache(S, max(lens), Hkv, D, page, quantised, 3)
    missing = [set() if s % 3 else set(torch.randint(0, 1 + lens[s] // page, (5,), generator=g).tolist()) for s in range(S)]
    for s, m in enumerate(missing):
        for p in m:
            if p < cache.table.shape[1]:
                cache.table[s, p] = cache.n_pages + s
    q, k, v = (torch.randn(S, N, h, D, generator=g).bfloat16().cuda() for h in (Hq, Hkv, Hkv))
    mask = au.ancestors(torch.tensor([[-1, 0]] * S))
    got = ctx.tree_attention(cache, q, k, v, au.pack(mask).cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), with_lse=True)
    assert ctx.get_status() == ngs.STATUS_CAPACITY
    (hk, left), (hv, _) = without(hk, lens, page, missing), without(hv, lens, page, missing)
    au.check_attention(got, au.attention(q, k, v, hk, hv, mask, left, D ** -0.5), SCORE)
