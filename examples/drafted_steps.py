"""Serving with drafted tokens behind one common prompt: a small model with random weights and rotary positions decodes a
batch whose sequences all begin with the same prompt, several drafted tokens a step.

    python examples/drafted_steps.py [--sequences 8] [--prompt 512] [--tokens 48] [--drafts 4] [--dtype bf16]

A step of a layer is three calls: ``rotary_and_cache`` turns the new tokens' queries and keys by their
positions and appends keys and values to the paged caches, ``paged_attention_common`` attends to the prompt's blocks once for the
whole batch and to each sequence's own ones; the step ends with ``verify_drafts``.  The drafts are what the model without its layers
would say next.  Sampling is greedy (probabilities of one entry), so that drafted steps have to give the very
tokens of steps of one token: --check decodes once more without drafts and compares.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2505_02351_amd as G  # noqa: E402


class Model:
    """Embedding, layers of attention, and the embedding again as the output."""

    def __init__(self, dtype, vocab=1000, layers=2, heads=8, kv_heads=2, dim=64, seed=0):
        gen = torch.Generator().manual_seed(seed)
        width = heads * dim
        self.heads, self.kv_heads, self.dim, self.vocab, self.dtype = heads, kv_heads, dim, vocab, dtype

        def weights(*shape, scale):
            return (scale * torch.randn(*shape, generator=gen)).to(dtype).cuda()

        self.embed = weights(vocab, width, scale=1.0)
        self.out = weights(width, vocab, scale=1.0 / math.sqrt(width))
        self.qkv = [weights(width, (heads + 2 * kv_heads) * dim, scale=1.0 / math.sqrt(width)) for _ in range(layers)]
        self.proj = [weights(width, width, scale=0.7 / math.sqrt(width)) for _ in range(layers)]
        freqs, self.magnitude = G.rotary_frequencies(dim, 10000.0, G.ROTARY_YARN, 4.0, 4096.0)
        self.freqs = freqs.cuda()

    def logits(self, x):
        return (x @ self.out).float()

    def rows(self, layer, x):
        """q, k and v of tokens' activations: slices of one projection's rows."""
        T, D = x.shape[0], self.dim
        return [r.unflatten(1, (-1, D)) for r in (x @ self.qkv[layer]).split([self.heads * D, self.kv_heads * D, self.kv_heads * D], dim=1)]


class Server:
    """Paged caches of a batch behind one prompt, and its steps."""

    def __init__(self, model, prompt, sequences, max_tokens, drafts, block=16):
        self.m, self.drafts, self.block, self.B = model, drafts, block, sequences
        assert prompt.shape[0] % block == 0, "the common prompt fills whole blocks"
        self.prefix_len = prompt.shape[0]
        NP, own = self.prefix_len // block, -(-(max_tokens + drafts + 1) // block)
        blocks = torch.randperm(NP + sequences * own, dtype=torch.int32).cuda()
        self.prefix = blocks[:NP].contiguous()
        self.tables = torch.cat([self.prefix.expand(sequences, -1), blocks[NP:].view(sequences, own)], dim=1).contiguous()
        shape = (blocks.shape[0], model.kv_heads, block, model.dim)
        self.caches = [[torch.zeros(shape, dtype=model.dtype, device="cuda") for _ in "kv"] for _ in model.qkv]
        self.max_len, self.scale = self.prefix_len + max_tokens + drafts + 1, 1.0 / math.sqrt(model.dim)
        # (drafts are the most that a step has: steps of one token fit, too)
        self.ws = torch.empty(G.common_prefix_workspace_bytes(sequences * (drafts + 1), sequences, model.heads, model.kv_heads, model.dim, block, NP,
                                                              self.max_len, drafts + 1), dtype=torch.uint8, device="cuda")
        self.verify_ws = torch.empty(G.verify_drafts_workspace_bytes(sequences, model.vocab), dtype=torch.uint8, device="cuda")
        self._prefill(prompt)

    def _layers(self, tokens, positions, slots, attend):
        x = self.m.embed[tokens]
        for layer, (k_cache, v_cache) in enumerate(self.caches):
            q, k, v = self.m.rows(layer, x)
            turned, out = torch.empty(q.shape, dtype=q.dtype, device="cuda"), torch.empty(q.shape, dtype=q.dtype, device="cuda")
            G.rotary_and_cache(turned, q, k, v, k_cache, v_cache, slots, positions, self.m.freqs, magnitude=self.m.magnitude)
            attend(out, turned, k_cache, v_cache)
            x = x + out.flatten(1) @ self.m.proj[layer]
        return x

    def _prefill(self, prompt):
        n = self.prefix_len
        at = torch.arange(n, device="cuda")
        lens, cu = torch.tensor([n], dtype=torch.int32).cuda(), torch.tensor([0, n], dtype=torch.int32).cuda()
        table = self.prefix[None]
        x = self._layers(prompt, at.int(), self.prefix[at // self.block].long() * self.block + at % self.block,
                         lambda out, q, k, v: G.paged_prefill(out, q, k, v, table, lens, cu, None, self.scale, n))
        self.first = self.m.logits(x[-1:]).argmax(dim=1)

    def step(self, lens, last, drafts):
        """One step: the sequences' last tokens and `drafts` [B, n] behind them, verified -> (tokens [B, n + 1], kept drafts [B])."""
        B, n = drafts.shape
        i = torch.arange(n + 1, device="cuda")
        positions = lens[:, None] + i
        slots = self.tables.long().gather(1, positions // self.block) * self.block + positions % self.block
        new_lens, cu = (lens + n + 1).int(), (torch.arange(B + 1, device="cuda") * (n + 1)).int()
        tokens = torch.cat([last[:, None], drafts], dim=1).flatten()
        x = self._layers(tokens, positions.flatten().int(), slots.flatten(),
                         lambda out, q, k, v: G.paged_attention_common(out, q, k, v, self.prefix, self.tables, new_lens, cu, None, self.scale,
                                                                       self.max_len, n + 1, self.ws))
        # greedy: the target's probabilities are one entry, the drafts were certain
        probs = torch.nn.functional.one_hot(self.m.logits(x).argmax(dim=1), self.m.vocab).float()
        got, kept = torch.empty(B, n + 1, dtype=torch.int64, device="cuda"), torch.empty(B, dtype=torch.int32, device="cuda")
        u = torch.rand(B * n, device="cuda"), torch.rand(B, device="cuda")
        G.verify_drafts(got, kept, probs, None, drafts.flatten().contiguous(), (torch.arange(B + 1, device="cuda") * n).int(), *u, self.verify_ws)
        return got, kept

    def decode(self, starts, count, drafts):
        """`count` tokens of each sequence behind its first own token; drafts: a step's -> (tokens [B, count], steps)."""
        lens = torch.full((self.B,), self.prefix_len, device="cuda")
        last, said, steps = starts, [[] for _ in range(self.B)], 0
        while min(len(s) for s in said) < count:
            guess = torch.zeros(self.B, 0, dtype=torch.int64, device="cuda")
            token = last
            for _ in range(drafts):                          # what the model without its layers says next
                token = self.m.logits(self.m.embed[token]).argmax(dim=1)
                guess = torch.cat([guess, token[:, None]], dim=1)
            got, kept = self.step(lens, last, guess)
            steps += 1
            for b, (row, n) in enumerate(zip(got.tolist(), kept.tolist())):
                room = count - len(said[b])
                said[b] += row[:n + 1][:room]
            # (a sequence that is done goes on from where it stands, its tokens unused)
            done = torch.tensor([len(s) >= count for s in said], device="cuda")
            lens = torch.where(done, lens, lens + kept + 1)
            last = torch.where(done, last, got.gather(1, kept.long()[:, None])[:, 0])
        return torch.tensor(said), steps


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--sequences", type=int, default=8)
    ap.add_argument("--prompt", type=int, default=512)
    ap.add_argument("--tokens", type=int, default=48)
    ap.add_argument("--drafts", type=int, default=4)
    ap.add_argument("--dtype", choices=("f16", "bf16"), default="bf16")
    ap.add_argument("--check", action="store_true")
    a = ap.parse_args(argv)
    torch.manual_seed(1)
    model = Model(torch.float16 if a.dtype == "f16" else torch.bfloat16)
    prompt, starts = torch.randint(0, model.vocab, (a.prompt,)).cuda(), torch.randint(0, model.vocab, (a.sequences,)).cuda()
    tokens, steps = Server(model, prompt, a.sequences, a.tokens, a.drafts).decode(starts, a.tokens, a.drafts)
    print(f"{a.tokens} tokens of {a.sequences} sequences in {steps} steps with {a.drafts} drafts each")
    if a.check:
        plain, single = Server(model, prompt, a.sequences, a.tokens, 0).decode(starts, a.tokens, 0)
        same = int((tokens == plain).all(dim=1).sum())
        print(f"without drafts: {single} steps; {same} of {a.sequences} sequences the same")
        return tokens, plain
    return tokens, None


if __name__ == "__main__":
    main()
