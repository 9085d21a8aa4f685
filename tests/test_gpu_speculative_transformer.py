"""The operators together: speculative decoding of a small transformer gives what plain float32 decoding would."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    path = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples", "speculative_transformer.py")
    spec = importlib.util.spec_from_file_location("speculative_transformer", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def run(example, quantised, steps=25):
    torch.manual_seed(1)
    model = example.Model()
    prompt = torch.randint(0, model.V, (3, 20), device="cuda").int().repeat(1, 3)
    return model, prompt, example.decode(model, prompt, steps, quantised=quantised)


@pytest.mark.parametrize("quantised", [False, True])
def test_decodes_what_plain_decoding_would(example, quantised):
    model, prompt, (hist, lens, logp, rate) = run(example, quantised)
    assert 1.0 <= rate <= 5.0
    L = prompt.shape[1]
    for s in range(hist.shape[0]):
        n = int(lens[s])
        z = model.reference_logits(hist[s:s + 1, :n - 1])[0, L - 1:]
        took = hist[s, L:n].long()
        # logits of standard deviation about 1: bfloat16 activations (2^-9 of each, two layers) move one by some hundredths, E4M3 keys and
        # values (2^-4 of each) by some tenths, so a token may trail the float32 winner by no more than twice that
        tol = 0.6 if quantised else 0.1
        behind = z.amax(-1) - z.gather(1, took[:, None])[:, 0]
        assert (behind <= tol).all(), behind.max()
        want = torch.log_softmax(z, -1).gather(1, took[:, None])[:, 0]
        got = logp[s][logp[s] < 0]
        assert got.numel() == took.numel() and ((got - want).abs() <= tol).all()


def test_blocks_of_one_token_agree_with_rows(example):
    """The same tokens committed by blocks of one node (plain decoding) and by wide blocks, teacher-forced."""
    model = example.Model(seed=3)
    torch.manual_seed(2)
    tokens = torch.randint(0, model.V, (2, 40), device="cuda").int()
    ctx = model.ctx
    whole = model.read_prompt(model.caches(2, 64), tokens)
    caches = model.caches(2, 64)
    model.read_prompt(caches, tokens[:, :30].contiguous())
    mask, depth = ctx.tree_mask(torch.full((2, 1), -1, dtype=torch.int32, device="cuda"))
    for i in range(30, 40):
        lens = torch.full((2,), i, dtype=torch.int32, device="cuda")
        hidden, kv = model.call(caches, tokens[:, i:i + 1], lens, mask, depth)
        for cache, (k, v) in zip(caches, kv):
            ctx.cache_write(cache, k, v, lens)
        # normalised activations (of size 1): bfloat16 in two orders of summation
        assert (hidden[:, 0].float() - whole[:, i].float()).abs().max() < 0.1
    assert ctx.get_status() == 0


@pytest.mark.parametrize("quantised", [False, True])
def test_drafts_are_accepted(example, quantised):
    """A model that says what follows each token (its head is its next token's embedding) on a text that goes round in
    circles: drafts from the history are accepted, and several nodes of a row are committed at once."""
    import paper_2411_03786_b200 as ngs
    torch.manual_seed(3)
    model = example.Model(V=500, seed=5)
    for w in model.layers:  # the residual stream is the last token's embedding alone
        w["out"].zero_(), w["down"].zero_()
    after = (torch.arange(model.V) * 7 + 3) % 12  # every token leads into a circle within the first 12
    model.unembed.zero_()
    for a in range(12):
        model.unembed[after[a]] += model.embed[a]
    prompt = torch.arange(36, device="cuda").int().view(1, 36) % 12
    model.ctx.close()
    model.ctx = ngs.SpecContext(model.embed, model.unembed)
    hist, lens, logp, rate = example.decode(model, prompt.expand(2, 36).contiguous(), 20, quantised=quantised)
    assert rate > 2.0
    for s in range(2):
        text = hist[s, : int(lens[s])].tolist()
        assert all(text[i + 1] == int(after[text[i]]) for i in range(36, len(text) - 1))
