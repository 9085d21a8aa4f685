"""What the calls around the model's attention take from a user, and what they refuse."""
import pytest
import torch

import attn_util as au

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    import paper_2411_03786_b200 as ngs
    g = torch.Generator().manual_seed(0)
    w = torch.randn(100, 64, generator=g).bfloat16().cuda()
    c = ngs.SpecContext(w, w)
    yield c
    c.close()


def operands(S=2, N=3, Hq=4, Hkv=2, D=64, tokens=64):
    cache, _, _ = au.make_cache(S, tokens, Hkv, D, 16, False, 4)
    g = torch.Generator().manual_seed(5)
    q, k, v = (torch.randn(S, N, h, D, generator=g).bfloat16().cuda() for h in (Hq, Hkv, Hkv))
    mask = au.pack(torch.eye(N, dtype=torch.bool).expand(S, N, N)).cuda()
    return cache, q, k, v, mask, torch.full((S,), min(20, tokens), dtype=torch.int32).cuda()


def rope(ngs, D=64):
    return ngs.Rope((10000.0 ** (-torch.arange(0, D, 2) / D)).float().cuda())


def test_outputs_and_workspaces_in_host_memory_are_refused(ctx):
    import paper_2411_03786_b200 as ngs
    cache, q, k, v, mask, lens = operands()
    pos = torch.zeros(2, 3, dtype=torch.int32).cuda()
    h, tok = torch.randn(4, 64).bfloat16().cuda(), torch.zeros(4, dtype=torch.int32).cuda()
    ok = ctx.rope_rows(rope(ngs), q, k, pos)
    scores = ctx.score_tokens(h, tok, n_alt=2)
    att = ctx.tree_attention(cache, q, k, v, mask, lens, with_lse=True)
    read = ctx.cache_read(cache, lens, 2)
    big = torch.empty(1 << 27, dtype=torch.uint8)
    for f in (lambda: ctx.rope_rows(rope(ngs), q, k, pos, out=(ok[0].cpu(), ok[1])),
              lambda: ctx.rope_rows(rope(ngs), q, k, pos, out=(ok[0], ok[1].cpu())),
              lambda: ctx.rope_rows(rope(ngs), q, k, pos, out=(ok[0], None)),
              lambda: ctx.score_tokens(h, tok, work=big),
              lambda: ctx.score_tokens(h, tok, n_alt=2, out=(scores[0].cpu(), *scores[1:])),
              lambda: ctx.score_tokens(h, tok, n_alt=2, out=(*scores[:2], None, None)),
              lambda: ctx.score_tokens(h, tok, n_alt=2, out=scores[:2]),
              lambda: ctx.cache_read(cache, lens, 2, out=(read[0], read[1].cpu())),
              lambda: ctx.tree_attention(cache, q, k, v, mask, lens, work=big),
              lambda: ctx.tree_attention(cache, q, k, v, mask, lens, work=big.cuda()[::2]),
              lambda: ctx.tree_attention(cache, q, k, v, mask, lens, out=(None, att[1])),
              lambda: ctx.tree_attention(cache, q, k, v, mask, lens, out=(att[0], att[1].cpu()))):
        with pytest.raises(ngs.SpecError):
            f()
    # a workspace counts by its bytes, whatever its type
    need = ctx._lib.spec_tree_attention_bytes(ctx._h, cache._ref, 2, 3, 4)
    got = ctx.tree_attention(cache, q, k, v, mask, lens, with_lse=True, work=torch.empty((need + 3) // 4, dtype=torch.float32, device="cuda"))
    assert torch.equal(got[0], att[0]) and torch.equal(got[1], att[1])
    with pytest.raises(ngs.SpecError):
        ctx.tree_attention(cache, q, k, v, mask, lens, work=torch.empty(need // 4 - 4, dtype=torch.float32, device="cuda"))
    assert ctx.get_status() == 0


def test_outputs_in_pinned_host_memory(ctx):
    """As the older calls allow: results that reach the host without a copy."""
    import paper_2411_03786_b200 as ngs
    cache, q, k, v, mask, lens = operands()
    pos = torch.arange(6, dtype=torch.int32).view(2, 3).cuda()
    h, tok = torch.randn(4, 64).bfloat16().cuda(), torch.zeros(4, dtype=torch.int32).cuda()
    calls = (lambda out: ctx.rope_rows(rope(ngs), q, k, pos, out=out), lambda out: ctx.score_tokens(h, tok, n_alt=2, out=out),
             lambda out: ctx.cache_read(cache, lens, 2, out=out), lambda out: ctx.tree_attention(cache, q, k, v, mask, lens, with_lse=True, out=out))
    for f in calls:
        want = f(None)
        got = tuple(torch.empty_like(t, device="cpu").pin_memory() for t in want)
        f(got)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b.cpu()) for a, b in zip(got, want))
    assert ctx.get_status() == 0


def test_one_node_of_each_sequence_out_of_a_fused_projection(ctx):
    """Plain decoding: queries, keys and values cut out of one [S, Hq + 2 Hkv, D] product."""
    import paper_2411_03786_b200 as ngs
    S, Hq, Hkv, D = 5, 8, 2, 64
    cache, _, _ = au.make_cache(S, 40, Hkv, D, 16, False, 4)
    qkv = torch.randn(S, Hq + 2 * Hkv, D, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    cut = tuple(t.unsqueeze(1) for t in qkv.split([Hq, Hkv, Hkv], 1))
    pos = torch.arange(S, dtype=torch.int32).view(S, 1).cuda()
    lens = (torch.arange(S) * 7).int().cuda()
    mask = torch.ones(S, 1, 1, dtype=torch.int32).cuda()
    out = []
    for q, k, v in (cut, tuple(t.contiguous() for t in cut)):
        r = ctx.rope_rows(rope(ngs), q, k, pos)
        a = ctx.tree_attention(cache, q, k, v, mask, lens, with_lse=True)
        c = ngs.KVCache(cache.k.clone(), cache.v.clone(), cache.table)
        ctx.cache_write(c, k, v, lens, rope=rope(ngs))
        out.append((*r, *a, c.k, c.v))
    assert all(torch.equal(x, y) for x, y in zip(*out)) and ctx.get_status() == 0
    # the last of several nodes, likewise
    t = torch.randn(S, 3, Hq + 2 * Hkv, D).bfloat16().cuda()[:, -1:]
    q, k, v = t.split([Hq, Hkv, Hkv], 2)
    a = ctx.tree_attention(cache, q, k, v, mask, lens)[0]
    assert torch.equal(a, ctx.tree_attention(cache, q.contiguous(), k.contiguous(), v.contiguous(), mask, lens)[0])


def test_rope_of_more_dimensions(ctx):
    """Tokens in several dimensions are taken where they are one stride apart, and refused where not."""
    import paper_2411_03786_b200 as ngs
    t = torch.randn(2, 3, 4, 6, 64).bfloat16().cuda()
    pos = torch.arange(24, dtype=torch.int32).view(2, 3, 4).cuda()
    want = ctx.rope_rows(rope(ngs), t.view(24, 6, 64), None, pos.view(24))[0].view(t.shape)
    assert torch.equal(ctx.rope_rows(rope(ngs), t, None, pos)[0], want)
    assert torch.equal(ctx.rope_rows(rope(ngs), t[:, :, :, 2:], None, pos)[0], want[:, :, :, 2:])
    assert torch.equal(ctx.rope_rows(rope(ngs), t[:, :1, 3:], None, pos[:, :1, 3:].contiguous())[0], want[:, :1, 3:])
    for x in (t[:, :, :2], t[:, :2], t.transpose(1, 2), t[0, 0, 0]):
        with pytest.raises(ngs.SpecError):
            ctx.rope_rows(rope(ngs), x, None, torch.zeros(x.shape[:-2], dtype=torch.int32).cuda())
    assert ctx.get_status() == 0


def test_a_refused_cache_does_not_spoil_the_next_call(ctx):
    """A cache that is refused for its pages, then a good one of the same sizes."""
    import paper_2411_03786_b200 as ngs
    cache, q, k, v, mask, lens = operands(S=2, N=5, Hq=6, Hkv=2)
    t = torch.zeros(8, 2, 8, 64, dtype=torch.bfloat16, device="cuda")  # pages of 8
    with pytest.raises(ngs.SpecError):
        ctx.tree_attention(ngs.KVCache(t, t.clone(), cache.table), q, k, v, mask, lens)
    assert ctx.tree_attention(cache, q, k, v, mask, lens)[0].isfinite().all()
    assert ctx.get_status() == 0


def test_empty_calls_do_nothing(ctx):
    """No sequences, no nodes, no tokens, no rows: tensors without an address."""
    import paper_2411_03786_b200 as ngs
    D, before = 64, ctx.launch_count()
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")
    rows = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device="cuda")
    f = rope(ngs)
    a, b = ctx.rope_rows(f, rows(0, 4, D), rows(0, 2, D), i32(0))
    assert a.shape == (0, 4, D) and b.shape == (0, 2, D)
    assert ctx.rope_rows(f, rows(3, 0, 4, D), None, i32(3, 0))[0].shape == (3, 0, 4, D)
    assert [t.shape for t in ctx.score_tokens(rows(0, 64), i32(0), n_alt=3)] == [(0,), (0,), (0, 3), (0, 3)]
    for quantised in (False, True):
        none = ngs.KVCache.empty(2, 2, 16, D, i32(0, 4), quantised)
        ctx.cache_write(none, rows(0, 3, 2, D), rows(0, 3, 2, D), i32(0), rope=f)
        assert ctx.cache_read(none, i32(0), 5)[0].shape == (0, 5, 2, D)
        mask, depth = ctx.tree_mask(i32(0, 3))
        assert mask.shape == (0, 3, 1) and depth.shape == (0, 3)
        o, l = ctx.tree_attention(none, rows(0, 3, 4, D), rows(0, 3, 2, D), rows(0, 3, 2, D), mask, i32(0), with_lse=True)
        assert o.shape == (0, 3, 4, D) and l.shape == (0, 3, 4)
        some = ngs.KVCache.empty(2, 2, 16, D, i32(3, 1), quantised)
        some.k.zero_()
        ctx.cache_write(some, rows(3, 0, 2, D), rows(3, 0, 2, D), i32(3))
        ctx.cache_write(some, rows(3, 0, 2, D), rows(3, 0, 2, D), i32(3), nodes=i32(3, 2))  # nodes that there are not
        ctx.cache_write(some, rows(3, 2, 2, D) + 1, rows(3, 2, 2, D) + 1, i32(3), nodes=i32(3, 0))
        assert (some.k == 0).all()
        assert ctx.cache_read(some, i32(3), 0)[1].shape == (3, 0, 2, D)
        mask, depth = ctx.tree_mask(i32(3, 0))
        assert mask.shape == (3, 0, 0) and depth.shape == (3, 0)
        o, l = ctx.tree_attention(some, rows(3, 0, 4, D), rows(3, 0, 2, D), rows(3, 0, 2, D), mask, i32(3), with_lse=True)
        assert o.shape == (3, 0, 4, D) and l.shape == (3, 0, 4)
    assert ctx.launch_count() == before and ctx.get_status() == 0
    with pytest.raises(ngs.SpecError):  # sizes are looked at all the same
        ctx.tree_attention(some, rows(3, 0, 3, D), rows(3, 0, 2, D), rows(3, 0, 2, D), mask, i32(3))
    with pytest.raises(ngs.SpecError):
        ctx.score_tokens(rows(0, 64), i32(0), n_alt=33)
