"""The operators together as a program uses them: speculative decoding whose caches' pages are handed out while sequences grow."""
import pytest
import torch

from test_gpu_speculative_transformer import example  # noqa: F401

pytestmark = pytest.mark.gpu


def prompts(model):
    torch.manual_seed(1)
    return torch.randint(0, model.V, (3, 20), device="cuda").int().repeat(1, 3)


@pytest.mark.parametrize("bits", [16, 8])
def test_pages_that_come_as_needed_change_nothing(example, bits):  # noqa: F811
    """The same text and scores, bit for bit, as with a table that is filled beforehand."""
    model = example.Model()
    a = example.decode(model, prompts(model), 25, quantised=bits == 8)
    b = example.decode(model, prompts(model), 25, bits=bits)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and torch.equal(a[2], b[2])


def test_decodes_over_a_cache_of_4_bits(example):  # noqa: F811
    """Twice the same; the first step, whose block attends to the prompt's cache, is plain decoding's up to what 4 bits leave of keys and values."""
    model = example.Model()
    runs = [example.decode(model, prompts(model), 25, bits=4) for _ in range(2)]
    assert all(torch.equal(x, y) for x, y in zip(runs[0][:3], runs[1][:3]))
    hist, lens, logp, rate = runs[0]
    L = 60
    assert 1.0 <= rate <= 5.0 and logp.isfinite().all() and (lens > L).all()
    for s in range(hist.shape[0]):
        n = int(lens[s])
        z = model.reference_logits(hist[s:s + 1, :n - 1])[0, L - 1:]
        behind = z.amax(-1) - z.gather(1, hist[s, L:n].long()[:, None])[:, 0]
        # E4M3 may move a logit by 0.3 (the tolerance of its test, 2^-4 of each value at most); E2M1 is off by a fifth at most (5 where 4 or 6 is held), 3.2 times as much: two logits
        # differ by 2 x 0.3 x 3.2 at most
        assert (behind <= 1.92).all(), behind.max()


def test_a_pool_that_is_too_small_is_reported(example):  # noqa: F811
    import paper_2411_03786_b200 as ngs
    model = example.Model()
    pool = ngs.PagePool.empty(len(model.layers), 3, 2, 8, model.Hkv, 16, model.D, bits=4)
    ok = model.ctx.pages_reserve(pool, torch.zeros(2, dtype=torch.int32, device="cuda"), torch.tensor([33, 20], dtype=torch.int32, device="cuda"))
    assert ok.tolist() == [1, 0] and model.ctx.get_status() == ngs.STATUS_CAPACITY
