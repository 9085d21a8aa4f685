"""Speculative decoding of a small transformer: drafting, the model call on the block of draft rows, acceptance.

    python examples/speculative_transformer.py [--cache e4m3] [--steps 40]

A step drafts B rows of w tokens from the sequence's own history and the model's bigrams, runs the model on the block of
B * (w + 1) nodes behind the cached context (``rope_rows``, ``tree_attention``), takes the arg max of every node,
accepts the longest agreeing prefix, and writes what was accepted - and nothing else of the block - to the cache
(``cache_write``).  ``score_tokens`` gives the log probabilities of the tokens it committed.  Weights are random: the
text means nothing, but what is decoded is what plain decoding, one token at a time, would give.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
import paper_2411_03786_b200 as ngs  # noqa: E402


class Model:
    """A decoder of `layers` blocks with grouped heads, random bfloat16 weights and a paged cache per layer."""

    def __init__(self, V=2000, d=512, layers=2, Hq=8, Hkv=2, D=64, seed=0):
        g = torch.Generator().manual_seed(seed)
        w = lambda *s: (torch.randn(*s, generator=g) * s[-1] ** -0.5).bfloat16().cuda()
        self.V, self.d, self.Hq, self.Hkv, self.D = V, d, Hq, Hkv, D
        self.embed, self.unembed = w(V, d), w(V, d)
        self.layers = [{"qkv": w((Hq + 2 * Hkv) * D, d), "out": w(d, Hq * D), "up": w(4 * d, d), "down": w(d, 4 * d)} for _ in range(layers)]
        self.freq = (10000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)).float().cuda()
        self.rope = ngs.Rope(self.freq)
        self.ctx = ngs.SpecContext(self.embed, self.unembed)

    def caches(self, S, tokens, page=16, quantised=False):
        per = -(-tokens // page)
        table = torch.randperm(S * per, device="cuda").int().view(S, per)  # pages in any order
        return [ngs.KVCache.empty(S * per, self.Hkv, page, self.D, table, quantised) for _ in self.layers]

    @staticmethod
    def norm(x):
        return torch.nn.functional.rms_norm(x.float(), x.shape[-1:]).to(x.dtype)

    def forward(self, tokens, attend):
        """Hidden states [S, N, d] of tokens [S, N]; attend(layer, q, k, v) is the attention of one layer."""
        x = self.embed[tokens.long()] * self.d ** 0.5
        for i, w in enumerate(self.layers):
            qkv = (self.norm(x) @ w["qkv"].T).unflatten(-1, (-1, self.D))
            q, k, v = qkv.split([self.Hq, self.Hkv, self.Hkv], -2)
            x = x + attend(i, q, k, v).flatten(-2) @ w["out"].T
            x = x + torch.nn.functional.gelu(self.norm(x) @ w["up"].T) @ w["down"].T
        return self.norm(x)

    def call(self, caches, tokens, lens, mask, depth):
        """The model on a block of nodes behind `lens` cached tokens.  Returns hidden states and each layer's (k, v)."""
        pos = lens[:, None] + depth
        block = []

        def attend(i, q, k, v):
            q, k = self.ctx.rope_rows(self.rope, q, k, pos)
            block.append((k, v))
            return self.ctx.tree_attention(caches[i], q, k, v, mask, lens)[0]

        return self.forward(tokens, attend), block

    def read_prompt(self, caches, tokens):
        """Fills the caches with a prompt: a block that is one chain, behind nothing."""
        S, L = tokens.shape
        chain = (torch.arange(L, device="cuda") - 1).int().expand(S, L).contiguous()
        mask, depth = self.ctx.tree_mask(chain)
        zero = torch.zeros(S, dtype=torch.int32, device="cuda")

        def attend(i, q, k, v):
            self.ctx.cache_write(caches[i], k, v, zero, rope=self.rope)  # rotated on the way
            q, k = self.ctx.rope_rows(self.rope, q, k, depth)
            return self.ctx.tree_attention(caches[i], q, k, v, mask, zero)[0]

        return self.forward(tokens, attend)

    def reference_logits(self, tokens):
        """Plain float32 logits [S, N, V] of a whole sequence: no cache, no block."""
        S, N = tokens.shape
        x = self.embed[tokens.long()].float() * self.d ** 0.5
        a = torch.arange(N, device="cuda")[:, None, None] * self.freq
        cos, sin = a.cos(), a.sin()
        turn = lambda t: torch.cat([t[..., : self.D // 2] * cos - t[..., self.D // 2:] * sin, t[..., : self.D // 2] * sin + t[..., self.D // 2:] * cos], -1)
        for w in self.layers:
            qkv = (torch.nn.functional.rms_norm(x, x.shape[-1:]) @ w["qkv"].float().T).unflatten(-1, (-1, self.D))
            q, k, v = qkv.split([self.Hq, self.Hkv, self.Hkv], -2)
            q, k = turn(q).transpose(1, 2), turn(k).repeat_interleave(self.Hq // self.Hkv, 2).transpose(1, 2)
            v = v.repeat_interleave(self.Hq // self.Hkv, 2).transpose(1, 2)
            s = (q @ k.transpose(2, 3) * self.D ** -0.5).masked_fill(torch.ones(N, N, dtype=torch.bool, device="cuda").triu(1), float("-inf"))
            x = x + (s.softmax(-1) @ v).transpose(1, 2).flatten(-2) @ w["out"].float().T
            x = x + torch.nn.functional.gelu(torch.nn.functional.rms_norm(x, x.shape[-1:]) @ w["up"].float().T) @ w["down"].float().T
        return torch.nn.functional.rms_norm(x, x.shape[-1:]) @ self.unembed.float().T


def decode(model, prompt, steps, B=6, w=4, quantised=False):
    """`steps` speculative steps after prompt [S, L].  Returns the histories [S, cap], their lengths, the log probabilities
    of the committed tokens, and tokens per step."""
    ctx, (S, L) = model.ctx, prompt.shape
    cap = (L + steps * (w + 1) + 3) // 4 * 4
    hist = torch.zeros(S, cap, dtype=torch.int32, device="cuda")
    hist[:, :L] = prompt
    lens = torch.full((S,), L, dtype=torch.int32, device="cuda")
    caches = model.caches(S, cap, quantised=quantised)
    ctx.build_model_ngram_tables(8, w_ext=w)
    model.read_prompt(caches, prompt[:, :-1].contiguous())
    N = B * (w + 1)
    node = torch.arange(N, device="cuda")
    mask, depth = ctx.tree_mask(torch.where(node % (w + 1) == 0, -1, node - 1).int().expand(S, N).contiguous())
    logps = []
    for _ in range(steps):
        drafts, n_drafts, _, _ = ctx.draft_context_ngrams(hist, lens, [3, 2, 1], B, B, w)
        last = hist.gather(1, lens.long()[:, None] - 1)
        block = torch.cat([last[:, None].expand(S, B, 1), drafts.clamp(min=0)], 2).view(S, N)
        cached = lens - 1  # the last token's keys are the block's: they are not in the cache yet
        hidden, kv = model.call(caches, block, cached, mask, depth)
        rows = hidden.view(S * N, model.d)
        argmax, _ = ctx.verify_lmhead_argmax(rows)
        accepted, best, committed = ctx.accept_and_commit(drafts, n_drafts, argmax.view(S, B, w + 1), hist, lens)
        # the accepted path: column 0 and the accepted drafts of the best row
        step = torch.arange(w + 1, device="cuda")
        nodes = torch.where(step <= accepted[:, None], best[:, None] * (w + 1) + step, -1).int()
        for cache, (k, v) in zip(caches, kv):
            ctx.cache_write(cache, k, v, cached, count=accepted + 1, nodes=nodes)
        at = (torch.arange(S, device="cuda")[:, None] * N + nodes.clamp(min=0)).view(-1)
        logps.append(ctx.score_tokens(rows[at], committed.view(-1))[0].view(S, w + 1))
    assert ctx.get_status() == 0
    return hist, lens, torch.stack(logps, 1), (lens - L).float().mean().item() / steps


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--cache", choices=("bf16", "e4m3"), default="bf16")
    ap.add_argument("--steps", type=int, default=40)
    a = ap.parse_args()
    torch.manual_seed(0)
    model = Model()
    prompt = torch.randint(0, model.V, (4, 24), device="cuda").int().repeat(1, 3)  # something to find again
    hist, lens, logp, rate = decode(model, prompt, a.steps, quantised=a.cache == "e4m3")
    print(f"{rate:.2f} tokens per model call, mean log probability {logp[logp < 0].mean().item():.2f}")
    for s in range(hist.shape[0]):
        print(hist[s, prompt.shape[1]: min(int(lens[s]), prompt.shape[1] + 16)].tolist(), "...")


if __name__ == "__main__":
    main()
