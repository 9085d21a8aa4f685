"""Scores of rows and vocabularies with NaN and infinities."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


def grid(shape, scale, seed):
    """Multiples of 1/16 (activations) and 1/1024 (weights): every order of summation gives the same logits."""
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g).clamp(-6, 6) * scale).round() / (16 if scale == 16 else 1024)


@pytest.mark.parametrize("V,d,M", [(40, 64, 3), (1000, 64, 50), (5003, 128, 200)])
@pytest.mark.parametrize("n_alt", [1, 5, 20, 32])
def test_ids_of_rows_that_are_not_numbers(V, d, M, n_alt):
    """A NaN in one row's activations: no id of it is one of a token, and the other rows do not change."""
    import paper_2411_03786_b200 as ngs
    w, h = grid((V, d), 20, V).bfloat16().cuda(), grid((M, d), 16, M).bfloat16().cuda()
    ctx = ngs.SpecContext(w, w)
    tok = torch.arange(M).int().cuda() % V
    want = ctx.score_tokens(h, tok, n_alt=n_alt)
    bad = M // 2
    x = h.clone()
    x[bad, 7] = math.nan
    got = ctx.score_tokens(x, tok, n_alt=n_alt)
    rest = torch.arange(M, device="cuda") != bad
    assert all(torch.equal(a[rest], b[rest]) for a, b in zip(got, want))
    assert got[0][bad].isnan() and got[1][bad].isnan()
    assert (got[2][bad] == -1).all() and (got[3][bad] == -math.inf).all()
    assert ctx.get_status() == 0
    ctx.close()


def test_fewer_numbers_than_alternatives():
    """All but three tokens' logits are NaN: those three, then -1."""
    import paper_2411_03786_b200 as ngs
    V, d = 700, 64
    w, h = grid((V, d), 20, 1).bfloat16(), grid((2, d), 16, 2).bfloat16().cuda()
    keep = torch.zeros(V, dtype=torch.bool)
    keep[[3, 64, 699]] = True
    w[~keep, 0] = math.nan
    w = w.cuda()
    ctx = ngs.SpecContext(w, w)
    _, _, ids, logp = ctx.score_tokens(h, torch.zeros(2, dtype=torch.int32, device="cuda"), n_alt=6)
    z = (h.double() @ w.double().T).nan_to_num(nan=-math.inf)
    assert torch.equal(ids[:, :3].long(), torch.sort(z, dim=-1, descending=True, stable=True).indices[:, :3])
    assert (ids[:, 3:] == -1).all() and (logp[:, 3:] == -math.inf).all()
    ctx.close()


@pytest.mark.parametrize("hidden", [[0], [5002], list(range(0, 64)), list(range(990, 1500)), list(range(32, 5003, 3)), list(range(5002))])
@pytest.mark.parametrize("n_alt", [0, 6])
def test_tokens_without_a_chance(hidden, n_alt):
    """Logits of -inf (a vocabulary with tokens masked in its weights): no weight, no part in the entropy."""
    import paper_2411_03786_b200 as ngs
    V, d, M = 5003, 64, 40
    w, h = grid((V, d), 20, 3).bfloat16(), grid((M, d), 16, 4).bfloat16().cuda()
    w[hidden, 0] = -math.inf
    h[:, 0] = 1.0
    w = w.cuda()
    ctx = ngs.SpecContext(w, w)
    tok = (torch.arange(M) * 127 % V).int().cuda()
    tok[0] = hidden[0]
    logp, ent, ids, val = ctx.score_tokens(h, tok, n_alt=n_alt)
    z = h.double() @ w.double().T
    p = torch.log_softmax(z, -1)
    want = p.gather(1, tok.long()[:, None])[:, 0]
    h64 = torch.special.entr(p.exp()).sum(-1)
    # as for finite logits: exponentials within 2^-21, sums of V terms in chunks of 32, results of a size up to log V + |z|
    tol = 2.0 ** -20 + V * 2.0 ** -29 + 2.0 ** -22 * (1 + z.nan_to_num(neginf=0.0).abs().amax(-1))
    there = want > -math.inf
    assert (logp[~there] == -math.inf).all() and ((logp.double() - want).abs()[there] <= tol[there]).all()
    assert ((ent.double() - h64).abs() <= tol * (2 + h64)).all()
    if n_alt:
        order = torch.sort(z, dim=-1, descending=True, stable=True).indices[:, :n_alt]
        real = z.gather(1, order) > -math.inf
        assert torch.equal(ids.long(), torch.where(real, order, -1))
        assert ((val.double() - p.gather(1, order)).abs() <= tol[:, None])[real].all() and (val[~real] == -math.inf).all()
    assert ctx.get_status() == 0
    ctx.close()


def test_logits_further_apart_than_fp32_reaches():
    """2^127 and -2^127: the differences overflow, the statistics do not."""
    import paper_2411_03786_b200 as ngs
    V, d = 3000, 64
    w, h = torch.zeros(V, d), torch.zeros(2, d)
    w[:, 0] = -(2.0 ** 120)
    w[[5, 1700], 0] = 2.0 ** 120
    h[0, 0], h[1, 0] = 128.0, -128.0
    w, h = w.bfloat16().cuda(), h.bfloat16().cuda()
    ctx = ngs.SpecContext(w, w)
    logp, ent, ids, val = ctx.score_tokens(h, torch.tensor([1700, 9], dtype=torch.int32).cuda(), n_alt=2)
    want = torch.tensor([math.log(2), math.log(V - 2)])
    # (2^127 is beyond where logarithms of sums can show beside it: the log probabilities are those of the sums alone)
    assert (ent.cpu() - want).abs().max() < 1e-5 and (logp.cpu() + want).abs().max() < 1e-5
    assert ids.tolist() == [[5, 1700], [0, 1]] and (val.cpu() + want[:, None]).abs().max() < 1e-5
    ctx.close()
