"""Speculative decoding on a paged MXFP4 cache: a small decoder with random MXFP4 weights drafts with its first layer and
verifies with all of them.  A request's prompt goes through in one pass; every step then

    forks the sequence, drafts a few tokens on the fork (one at a time), drops the fork,
    makes room for the drafted tokens on the sequence itself and runs them through all layers at once,
    picks and compares with the draft (mxfp4_woq_gemm_verify), and gives back the rejected tokens' pages.

    python examples/speculative_cache.py [--tokens 64] [--drafts 4]

Needs a GPU and the built library.  The tokens are those of the same model decoded one token at a time, up to near ties of its
logits (a product of five rows may round differently from one of a single row)."""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2503_13565_amd import binding as b  # noqa: E402

DEV = "cuda"
LAYERS, HIDDEN, HEADS, KV_HEADS, DIM, MLP, VOCAB = 3, 1024, 16, 4, 64, 2048, 4096
PAGE, PAGES, WIDTH, LENGTH = 16, 256, 64, 1024


def ints(*values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


class Decoder:
    """Weights, and the cache with two table rows: 0 is the request, 1 its draft."""

    def __init__(self, seed=0):
        gen = torch.Generator().manual_seed(seed)

        def linear(n, k, scale=1.0):
            return b.mxfp4_direct_cast((torch.randn((n, k), generator=gen) * scale * k ** -0.5).to(torch.bfloat16).to(DEV))

        # the later layers add little, so that the first one is a draft worth having
        self.layers = [dict(qkv=linear((HEADS + 2 * KV_HEADS) * DIM, HIDDEN), out=linear(HIDDEN, HEADS * DIM, 0.5 if i == 0 else 0.1),
                            up=linear(2 * MLP, HIDDEN), down=linear(HIDDEN, MLP, 0.5 if i == 0 else 0.1)) for i in range(LAYERS)]
        self.embed = torch.randn((VOCAB, HIDDEN), generator=gen).to(torch.bfloat16).to(DEV)
        self.head = linear(VOCAB, HIDDEN)
        angle = torch.arange(LENGTH, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(DIM // 2, dtype=torch.float64) / (DIM // 2))
        self.rope = (angle.cos().float().to(DEV), angle.sin().float().to(DEV))
        self.cache = b.mxfp4_kv_cache(PAGES, KV_HEADS, PAGE, DIM, layers=LAYERS)
        self.whole = b.mxfp4_kv_all_layers(self.cache)
        self.pool = b.mxfp4_kv_pool(PAGES)
        self.table = torch.full((2, WIDTH), -1, dtype=torch.int32, device=DEV)
        self.lens = torch.zeros(2, dtype=torch.int32, device=DEV)
        self.state = (self.pool, self.whole, self.table, self.lens)

    def hidden(self, tokens, row, layers):
        """The tokens, which are new at the end of table row `row`, through the first layers."""
        x = self.embed[tokens.long()]
        n, table, lens = x.shape[0], self.table[row:row + 1], self.lens[row:row + 1]
        for i, w in enumerate(self.layers[:layers]):
            layer = b.mxfp4_kv_layer(self.cache, i)
            qkv = b.mxfp4_woq_gemm(norm(x), *w["qkv"]).view(n, HEADS + 2 * KV_HEADS, DIM)
            q, k, v = qkv.split([HEADS, KV_HEADS, KV_HEADS], dim=1)
            q = b.mxfp4_kv_append(layer, k, v, table, lens, q=q, rope=self.rope)
            seen = b.mxfp4_kv_attention(q, layer, table, lens)
            x = b.mxfp4_woq_gemm_fused(seen.view(n, HEADS * DIM), *w["out"], residual=x)
            x = b.mxfp4_woq_gemm_fused(b.mxfp4_woq_gemm_fused(norm(x), *w["up"], act=b.ACT_SWIGLU), *w["down"], residual=x)
        return norm(x)

    def grow(self, row, count):
        missing = b.mxfp4_kv_extend(*self.state, ints(row), ints(count))
        assert int(missing) == 0, "the cache is full"

    def pick(self, x):
        return b.mxfp4_woq_gemm_argmax(x, *self.head)[0]

    def prompt(self, tokens):
        self.grow(0, len(tokens))
        return self.pick(self.hidden(ints(*tokens), 0, LAYERS)[-1:])

    def step(self, last, drafts):
        """The tokens that follow `last` (int32 [1]), and how many of them the draft had."""
        draft, token = [], last
        if drafts:
            b.mxfp4_kv_fork(*self.state, ints(0), ints(1))
            for _ in range(drafts):
                self.grow(1, 1)
                token = self.pick(self.hidden(token, 1, 1))
                draft.append(token)
            b.mxfp4_kv_release(*self.state, ints(1), ints(0))
        draft = torch.cat([last, *draft])
        self.grow(0, drafts + 1)
        accepted, picks, _ = b.mxfp4_woq_gemm_verify(self.hidden(draft, 0, LAYERS), *self.head, draft[1:] if drafts else None)
        keep = int(accepted[0])
        b.mxfp4_kv_release(*self.state, ints(0), self.lens[:1] - (drafts - keep))
        return picks[: keep + 1], keep


def norm(x):
    return (x.float() * torch.rsqrt(x.float().square().mean(-1, keepdim=True) + 1e-6)).to(torch.bfloat16)


def generate(prompt, tokens, drafts, seed=0):
    """(tokens that follow the prompt, steps, accepted draft tokens, pages in use at the end)"""
    model = Decoder(seed)
    out, steps, taken = [model.prompt(prompt)], 0, 0
    while sum(x.numel() for x in out) < tokens:
        got, keep = model.step(out[-1][-1:], drafts)
        out.append(got)
        steps, taken = steps + 1, taken + keep
    return torch.cat(out).tolist()[:tokens], steps, taken, int((model.pool.refs > 0).sum())


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--tokens", type=int, default=64)
    ap.add_argument("--drafts", type=int, default=4)
    a = ap.parse_args()
    prompt = torch.randint(VOCAB, (100,), generator=torch.Generator().manual_seed(1)).tolist()
    one, steps, _, _ = generate(prompt, a.tokens, 0)
    got, fewer, taken, pages = generate(prompt, a.tokens, a.drafts)
    same = next((i for i, (x, y) in enumerate(zip(one, got)) if x != y), len(got))
    print("%d tokens: %d steps one by one, %d with %d drafted tokens each (%.2f accepted a step), %d pages in use" % (
        a.tokens, steps, fewer, a.drafts, taken / max(1, fewer), pages))
    print("the first %d of %d tokens are the same" % (same, len(got)))


if __name__ == "__main__":
    main()
