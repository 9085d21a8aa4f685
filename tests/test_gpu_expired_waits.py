"""Device-side waits that run out: the call returns, says so, and the next one is right.

The waits are made to run out by the host: a limit of nothing, with which a CTA starts as if one of its waits had expired
and gives up at the first barrier that is not complete yet.
"""
import pytest
import torch

import attn_util as au

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("quantised", [False, True])
@pytest.mark.parametrize("D,S,N,Hq,Hkv,lens", [(128, 3, 150, 8, 2, [1000, 0, 333]), (64, 6, 1, 4, 4, [5000, 17, 64, 0, 900, 128]), (128, 1, 700, 4, 1, [200])])
def test_tree_attention_gives_up_together(D, S, N, Hq, Hkv, lens, quantised):
    import paper_2411_03786_b200 as ngs
    w = torch.zeros(64, 64, dtype=torch.bfloat16, device="cuda")
    ctx = ngs.SpecContext(w, w)
    cache, _, _ = au.make_cache(S, max(lens), Hkv, D, 32, quantised, 1)
    g = torch.Generator().manual_seed(2)
    q, k, v = (torch.randn(S, N, h, D, generator=g).bfloat16().cuda() for h in (Hq, Hkv, Hkv))
    parent = torch.where(torch.arange(N) % 5 == 0, -1, torch.arange(N) - 1).int().expand(S, N).contiguous().cuda()
    mask, _ = ctx.tree_mask(parent)
    n = torch.tensor(lens, dtype=torch.int32).cuda()
    want = ctx.tree_attention(cache, q, k, v, mask, n, with_lse=True)
    assert ctx.get_status() == 0
    for limit in (0, 1):
        ctx.debug_wait_limit(limit)
        for _ in range(10):
            ctx.tree_attention(cache, q, k, v, mask, n, with_lse=True)
        bits = ctx.get_status()
        assert bits == ngs.STATUS_TIMEOUT if limit == 0 else bits in (0, ngs.STATUS_TIMEOUT)
    ctx.debug_wait_limit()
    got = ctx.tree_attention(cache, q, k, v, mask, n, with_lse=True)
    assert ctx.get_status() == 0 and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    ctx.close()


def test_the_limit_is_checked():
    import paper_2411_03786_b200 as ngs
    w = torch.zeros(64, 64, dtype=torch.bfloat16, device="cuda")
    ctx = ngs.SpecContext(w, w)
    with pytest.raises(ngs.SpecError):
        ctx.debug_wait_limit(2_000_000_001)
    ctx.close()


@pytest.mark.parametrize("V,d,M", [(5003, 256, 7), (1000, 1000, 300), (32000, 512, 129)])
def test_head_calls_give_up_together(V, d, M):
    import paper_2411_03786_b200 as ngs
    g = torch.Generator().manual_seed(V)
    w = (torch.randn(V, d, generator=g) / 32).bfloat16().cuda()
    h = torch.randn(M, d, generator=g).bfloat16().cuda()
    tok = torch.randint(0, V, (M,), generator=g).int().cuda()
    ctx = ngs.SpecContext(w, w)
    calls = [lambda n=n: ctx.score_tokens(h, tok, n_alt=n) for n in (0, 5, 20)] + [lambda: ctx.verify_lmhead_argmax(h, with_max=True)]
    want = [f() for f in calls]
    assert ctx.get_status() == 0
    for limit in (0, 1):
        ctx.debug_wait_limit(limit)
        for f in calls:
            for _ in range(5):
                out = f()
            bits = ctx.get_status()
            assert bits == ngs.STATUS_TIMEOUT if limit == 0 else bits in (0, ngs.STATUS_TIMEOUT)
        if limit == 0:
            assert (out[0] == -1).all()  # an incomplete verification does not pass for a result
    ctx.debug_wait_limit()
    for f, a in zip(calls, want):
        assert all(x is None and y is None or torch.equal(x, y) for x, y in zip(f(), a))
    assert ctx.get_status() == 0
    ctx.close()
