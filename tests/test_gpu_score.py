"""Scores of given tokens (log probability, entropy, alternatives) against a plain 64-bit form."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


def head(V, d, seed, grid=True):
    """Weights and activations on a grid (1/1024, 1/16): sums of products are exact in fp32 in any order, so ids are too."""
    import paper_2411_03786_b200 as ngs
    g = torch.Generator().manual_seed(seed)
    w = ((torch.randn(V, d, generator=g) * 20).round() / 1024).bfloat16().cuda()
    return ngs.SpecContext(w, w), w


def rows(M, d, seed):
    g = torch.Generator().manual_seed(seed)
    return ((torch.randn(M, d, generator=g).clamp(-7, 7) * 16).round() / 16).bfloat16().cuda()


def check(ctx, w, h, tok, n_alt):
    logp, ent, idx, val = ctx.score_tokens(h, tok, n_alt=n_alt)
    z = h.double() @ w.double().T
    p = torch.log_softmax(z, -1)
    M, V = z.shape
    # fp32 statistics: exponentials within 2^-21, sums of up to V positive terms within V 2^-24 / 32 (chunks of 32 columns), results
    # of a size up to log V + |z| rounded to fp32
    tol = 2.0 ** -20 + V * 2.0 ** -29 + 2.0 ** -22 * (1 + z.abs().amax(-1))
    ok = (tok >= 0) & (tok < V)
    want = p.gather(1, tok.long().clamp(0, V - 1)[:, None])[:, 0]
    assert ((logp.double() - want).abs()[ok] <= tol[ok]).all()
    assert (logp[tok == -1] == 0).all() and (logp[~ok & (tok != -1)] == -math.inf).all()
    h64 = torch.special.entr(p.exp()).sum(-1)
    assert ((ent.double() - h64).abs() <= tol * (2 + h64)).all()
    if n_alt:
        order = torch.sort(z, dim=-1, descending=True, stable=True)
        assert torch.equal(idx.long(), order.indices[:, :n_alt])
        assert ((val.double() - p.gather(1, order.indices[:, :n_alt])).abs() <= tol[:, None]).all()
    else:
        assert idx is None and val is None


@pytest.mark.parametrize("V,d", [(1, 8), (31, 64), (33, 72), (500, 128), (1000, 1000), (5003, 256), (32000, 512)])
@pytest.mark.parametrize("M", [1, 7, 48, 128, 129, 300])
def test_sizes(V, d, M):
    ctx, w = head(V, d, V)
    h = rows(M, d, M)
    g = torch.Generator().manual_seed(3)
    tok = torch.randint(0, V, (M,), generator=g).int().cuda()
    for n_alt in sorted({0, 1, min(5, V), min(8, V), min(9, V), min(32, V)}):
        check(ctx, w, h, tok, n_alt)
    assert ctx.get_status() == 0
    ctx.close()


def test_large_block():
    ctx, w = head(20011, 192, 5)
    h = rows(2816, 192, 6)
    tok = torch.randint(0, 20011, (2816,), generator=torch.Generator().manual_seed(1)).int().cuda()
    check(ctx, w, h, tok, 8)
    ctx.close()


def test_peaked_and_flat_rows():
    """One token with all the probability, and all tokens alike; the entropies' two ends."""
    ctx, w = head(4096, 64, 9)
    h = rows(3, 64, 1)
    h[0] *= 8  # logits of some tens
    h[1] = 0
    tok = torch.tensor([0, 4095, 77], dtype=torch.int32).cuda()
    check(ctx, w, h, tok, 4)
    logp, ent, idx, _ = ctx.score_tokens(h, tok, n_alt=4)
    assert abs(ent[1].item() - math.log(4096)) < 1e-5 and abs(logp[1].item() + math.log(4096)) < 1e-5
    assert idx[1].tolist() == [0, 1, 2, 3]  # equal logits: lowest ids
    ctx.close()


def test_first_last_and_unused_tokens():
    import paper_2411_03786_b200 as ngs
    ctx, w = head(1003, 64, 2)
    h = rows(6, 64, 2)
    check(ctx, w, h, torch.tensor([0, 1002, -1, 31, 32, -1], dtype=torch.int32).cuda(), 3)
    assert ctx.get_status() == 0
    check(ctx, w, h, torch.tensor([1003, -2, 5, 1 << 30, 0, 1], dtype=torch.int32).cuda(), 3)
    assert ctx.get_status() == ngs.STATUS_TOKEN_RANGE
    ctx.close()


def test_agrees_with_the_arg_max():
    ctx, w = head(9000, 256, 4)
    h = rows(200, 256, 5)
    am, _ = ctx.verify_lmhead_argmax(h)
    logp, _, idx, val = ctx.score_tokens(h, am, n_alt=1)
    assert torch.equal(idx[:, 0], am) and torch.equal(val[:, 0], logp)
    ctx.close()


def test_refusals():
    import paper_2411_03786_b200 as ngs
    ctx, w = head(100, 64, 4)
    h, tok = rows(4, 64, 1), torch.zeros(4, dtype=torch.int32).cuda()
    for f in (lambda: ctx.score_tokens(h[:, :32].contiguous(), tok), lambda: ctx.score_tokens(h, tok[:3]), lambda: ctx.score_tokens(h, tok.long()),
              lambda: ctx.score_tokens(h, tok, n_alt=33), lambda: ctx.score_tokens(h, tok, n_alt=-1),
              lambda: ctx.score_tokens(h, tok, work=torch.empty(8, dtype=torch.uint8, device="cuda"))):
        with pytest.raises((ngs.SpecError, RuntimeError)):
            f()
    assert ctx.get_status() == 0
    ctx.close()
