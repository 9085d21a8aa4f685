"""The far ends of the model call's operators: blocks of thousands of nodes, more row tiles than SMs, many heads."""
import pytest
import torch

import attn_util as au

pytestmark = pytest.mark.gpu
SCORE = 2.0 ** -14  # fp32 sums of products around 1, as in the tests of small blocks


@pytest.fixture(scope="module")
def ctx():
    import paper_2411_03786_b200 as ngs
    w = torch.zeros(64, 64, dtype=torch.bfloat16, device="cuda")
    c = ngs.SpecContext(w, w)
    yield c
    c.close()


def some_rows(got, rows, q, k, v, held_k, held_v, bits, lens, scale):
    """Compares `rows` of nodes with the definition, in 64 bits: bits[s, i] is the list of nodes that node i attends to."""
    G = q.shape[2] // k.shape[2]
    held_k, held_v, k64, v64 = held_k.cuda(), held_v.cuda(), k.double(), v.double()
    out, lse, mag = [], [], []
    for s, i in rows:
        at = torch.tensor(bits(s, i), dtype=torch.long, device="cuda")
        kk = torch.cat([held_k[s, : lens[s]], k64[s, at]]).repeat_interleave(G, 1)
        vv = torch.cat([held_v[s, : lens[s]], v64[s, at]]).repeat_interleave(G, 1)
        z = torch.einsum("hd,khd->hk", q[s, i].double(), kk) * scale
        lse.append(torch.logsumexp(z, -1))
        p = torch.exp(z - lse[-1][:, None])
        out.append(torch.einsum("hk,khd->hd", p, vv))
        mag.append(torch.einsum("hk,khd->hd", p, vv.abs()))
    pick = lambda t: torch.stack([t[s, i] for s, i in rows])
    au.check_attention((pick(got[0]), pick(got[1])), tuple(torch.stack(x).cpu() for x in (out, lse, mag)), SCORE)


def sample(S, N, seed):
    """The first and last nodes, those around multiples of 128, and some in between."""
    g = torch.Generator().manual_seed(seed)
    i = {0, 1, N - 1, N - 2, 127, 128, 129, N // 2, N - 128, N - 129} | set(torch.randint(0, N, (25,), generator=g).tolist())
    return [(s, n) for s in range(S) for n in sorted(i) if 0 <= n < N]


def call(ctx, S, N, Hq, Hkv, D, lens, quantised, parent, seed, page=64):
    cache, hk, hv = au.make_cache(S, max(max(lens), 1), Hkv, D, page, quantised, seed)
    g = torch.Generator().manual_seed(seed + 1)
    q, k, v = (torch.randn(S, N, h, D, generator=g).bfloat16().cuda() for h in (Hq, Hkv, Hkv))
    mask, depth = ctx.tree_mask(parent.int().expand(S, N).contiguous().cuda())
    got = ctx.tree_attention(cache, q, k, v, mask, torch.tensor(lens, dtype=torch.int32).cuda(), with_lse=True)

    def bits(s, i):
        path = []
        while i >= 0:
            path.append(i)
            i = int(parent[i])
        return path
    some_rows(got, sample(S, N, seed), q, k, v, hk, hv, bits, lens, D ** -0.5)
    assert got[0].isfinite().all() and got[1].isfinite().all() and ctx.get_status() == 0


@pytest.mark.parametrize("quantised", [False, True])
@pytest.mark.parametrize("N,Hq,Hkv,D,lens", [
    (4096, 10, 1, 64, [70]),       # 160 row-tile pairs: two passes of one group of CTAs, nothing joined
    (4096, 5, 1, 64, [0, 300]),    # 80: one group in one pass, two sequences
    (4000, 2, 2, 128, [129]),      # 32 tiles of the block, masks of 125 words
    (4096, 1, 1, 128, [200]),      # rows of which a CTA does not look through the masks
])
def test_prompts(ctx, N, Hq, Hkv, D, lens, quantised):
    """Blocks that are one chain, up to the longest: every node sees all before it."""
    call(ctx, len(lens), N, Hq, Hkv, D, lens, quantised, torch.arange(N) - 1, N + Hq)


@pytest.mark.parametrize("quantised", [False, True])
@pytest.mark.parametrize("N,Hq,Hkv,D,lens", [(4096, 10, 1, 64, [1000]), (3969, 3, 1, 128, [0, 17]), (2300, 34, 2, 64, [128])])
def test_wide_drafts(ctx, N, Hq, Hkv, D, lens, quantised):
    """Thousands of nodes in rows of 11: each attends to a tile or two of the block's 18 to 32."""
    j = torch.arange(N)
    call(ctx, len(lens), N, Hq, Hkv, D, lens, quantised, torch.where(j % 11 == 0, -1, j - 1), N)


@pytest.mark.parametrize("rot", [0, 64])
@pytest.mark.parametrize("quantised", [False, True])
@pytest.mark.parametrize("S,N,heads,D,page", [(2, 40, 96, 128, 16), (1, 1, 200, 64, 16), (3, 33, 1, 64, 32), (8, 2500, 2, 64, 128)])
def test_cache_write_of_many_heads_and_tokens(ctx, S, N, heads, D, page, rot, quantised):
    """More vectors than a CTA has in flight for one token, and as many tokens to a CTA as its tables hold."""
    import paper_2411_03786_b200 as ngs
    start = [(7 * s) % 50 for s in range(S)]
    g = torch.Generator().manual_seed(heads)
    cache = ngs.KVCache.empty(S * (-(-(50 + N) // page)), heads, page, D, torch.randperm(S * (-(-(50 + N) // page)), generator=g).int().view(S, -1).cuda(), quantised)
    k, v = ((torch.randn(S, N, heads, D, generator=g) * torch.exp(2 * torch.randn(S, N, heads, 1, generator=g))).bfloat16().cuda() for _ in range(2))
    st = torch.tensor(start, dtype=torch.int32).cuda()
    rope = ngs.Rope((10000.0 ** (-torch.arange(0, rot, 2) / rot)).float().cuda()) if rot else None
    ctx.cache_write(cache, k, v, st, rope=rope)
    got = ctx.cache_read(cache, st, N)
    if rot:  # (rotation in the write is that of rope_rows, which has its own tests)
        pos = (st[:, None] + torch.arange(N, device="cuda").int()).contiguous()
        k = ctx.rope_rows(rope, k, None, pos)[0]
    for x, y in zip((k, v), got):
        want = au.dequantise(*au.quantise(x)) if quantised else x.double().cpu()
        assert torch.equal(y.double().cpu(), want)
    assert ctx.get_status() == 0


def test_every_finite_code_survives(ctx):
    """Five rows of 64 hold all 254 of them."""
    finite = torch.tensor([b for b in range(256) if b & 127 != 127], dtype=torch.uint8)
    rows = torch.cat([finite, finite[:66]]).view(5, 64).clone()
    rows[:, 63] = 126  # 448: the scale is what it was
    assert set(rows.flatten().tolist()) >= set(finite.tolist()) - {finite[63].item(), finite[127].item(), finite[191].item()}
    rows[4, :3] = finite[[63, 127, 191]]  # (what the column of 448 took the place of)
    assert set(rows.flatten().tolist()) == set(finite.tolist())
    for exp in (7, 100, 127, 134):
        c, _, _ = au.make_cache(1, 5, 1, 64, 16, True, 1, spare=0)
        c.k[0, 0, :5], c.v[0, 0, :5] = rows.cuda(), rows.cuda()
        c.k_exp[0, 0, :5], c.v_exp[0, 0, :5] = exp, exp
        zero = torch.zeros(1, dtype=torch.int32).cuda()
        k, v = ctx.cache_read(c, zero, 5)
        d, _, _ = au.make_cache(1, 5, 1, 64, 16, True, 2, spare=0)
        ctx.cache_write(d, k, v, zero)
        assert torch.equal(d.k[0, 0, :5], rows.cuda()) and torch.equal(d.v[0, 0, :5], rows.cuda()) and (d.v_exp[0, 0, :5] == exp).all()
