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
