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
