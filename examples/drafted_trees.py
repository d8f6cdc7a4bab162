"""Serving several continuations of one prompt with trees of drafted tokens: a small model with random weights and rotary positions
reads a prompt once, forks it into a batch, and decodes each sequence with a tree of guesses a step.

    python examples/drafted_trees.py [--sequences 6] [--prompt 300] [--tokens 48] [--width 3] [--depth 3] [--dtype bf16]

The pages are kept on the GPU: ``resize_sequences`` makes room for a step's tree (a block that is shared with other sequences and
about to be written gets a copy, ``copy_blocks``), ``rotary_and_cache`` and ``paged_attention_tree`` are a layer,
``keep_tokens`` moves the accepted branch's rows to the front, and a second ``resize_sequences`` gives the rest back.  ``fork_sequences``
starts the batch and lets sequences go on from others; ``compact_blocks`` packs the pool.  The drafts are what the model without its
layers would say next.  Sampling is greedy, so that trees have to give the very tokens of steps of one token: --check decodes
once more without them and compares.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2505_02351_amd as G  # noqa: E402
from drafted_steps import Model  # noqa: E402


class Tree:
    """`width` guesses behind the last token, each followed by a line of `depth` - 1 more.  Node 0 is the last token itself."""

    def __init__(self, width, depth):
        self.width, self.depth, n = width, depth if width else 0, 1 + width * depth
        self.parents = [-1] + [0 if i <= width else i - width for i in range(1, n)]
        self.nodes = n
        masks, depths = G.tree_masks(self.parents)
        self.masks, self.depths = masks.cuda(), depths.cuda().long()


class Server:
    """A pool of pages, the caches of all layers in them, and the sequences that hold them."""

    def __init__(self, model, prompt, sequences, max_tokens, tree, block=16):
        self.m, self.tree, self.block, self.B = model, tree, block, sequences
        rows = prompt.shape[0] + max_tokens + tree.nodes + tree.depth + 1
        self.max_len, self.width = rows, -(-rows // block)
        self.pool = sequences * self.width                   # (room for sequences that share nothing any more)
        shape = (self.pool, model.kv_heads, block, model.dim)
        self.layers = [[torch.zeros(shape, dtype=model.dtype, device="cuda") for _ in "kv"] for _ in model.qkv]
        self.caches = G.CacheSet([c for pair in self.layers for c in pair])
        self.scale = 1.0 / math.sqrt(model.dim)

        def whole(*shape):
            return torch.zeros(shape, dtype=torch.int32, device="cuda")

        self.tables, self.lens, self.refs = whole(sequences, self.width), whole(sequences), whole(self.pool)
        self.other_tables, self.other_lens = whole(sequences, self.width), whole(sequences)
        self.copies, self.pairs, self.counts, self.no_prefix = whole(sequences, 2), whole(self.pool, 2), whole(2), whole(0)
        n = sequences * tree.nodes
        size = max(G.resize_workspace_bytes(sequences, self.width, self.pool), G.compact_workspace_bytes(self.pool),
                   G.tree_workspace_bytes(n, sequences, model.heads, model.kv_heads, model.dim, block, 0, rows, tree.nodes))
        self.ws = torch.empty(size, dtype=torch.uint8, device="cuda")
        self.cu = (torch.arange(sequences + 1, device="cuda") * tree.nodes).int()
        self.slots = torch.empty(n, dtype=torch.int64, device="cuda")
        self.masks = tree.masks.repeat(sequences, 1)
        self._prefill(prompt)

    def resize(self, lens, slots=None, cu=None, most=None):
        """most: tokens by which a sequence's length changes at most (a tree's, unless given)."""
        most = self.tree.nodes if most is None else most
        G.resize_sequences(self.tables, self.lens, self.refs, lens, slots, cu, self.copies, self.counts, self.block, most, self.ws)
        if slots is not None:
            G.copy_blocks(self.caches, self.copies, self.counts)

    def fork(self, parents):
        """Row b goes on from row parents[b] (negative: it ends)."""
        G.fork_sequences(self.other_tables, self.other_lens, self.tables, self.lens, self.refs, parents.int(), self.block)
        self.tables, self.other_tables, self.lens, self.other_lens = self.other_tables, self.tables, self.other_lens, self.lens

    def tidy(self):
        """Blocks in use to the front of the pool -> how many there are."""
        G.compact_blocks(self.tables, self.lens, self.refs, self.pairs, self.counts, self.block, self.ws)
        G.copy_blocks(self.caches, self.pairs, self.counts)
        return int(self.counts[1])

    def _layers(self, tokens, positions, slots, attend):
        x = self.m.embed[tokens]
        for layer, (k_cache, v_cache) in enumerate(self.layers):
            q, k, v = self.m.rows(layer, x)
            turned, out = torch.empty(q.shape, dtype=q.dtype, device="cuda"), torch.empty(q.shape, dtype=q.dtype, device="cuda")
            G.rotary_and_cache(turned, q, k, v, k_cache, v_cache, slots, positions, self.m.freqs, magnitude=self.m.magnitude)
            attend(out, turned, k_cache, v_cache)
            x = x + out.flatten(1) @ self.m.proj[layer]
        return x

    def _prefill(self, prompt):
        n = prompt.shape[0]
        lens = torch.zeros(self.B, dtype=torch.int32, device="cuda")
        lens[0] = n
        cu = torch.full((self.B + 1,), n, dtype=torch.int32, device="cuda")
        cu[0] = 0
        slots = torch.empty(n, dtype=torch.int64, device="cuda")
        self.resize(lens, slots, cu, n)
        first, table, starts = lens[:1].clone(), self.tables[:1], cu[:2].clone()
        self._layers(prompt, torch.arange(n, device="cuda").int(), slots,
                     lambda out, q, k, v: G.paged_prefill(out, q, k, v, table, first, starts, None, self.scale, n))
        self.fork(torch.zeros(self.B, device="cuda"))

    def guess(self, last):
        """Each sequence's tree: its last token, the likeliest ones behind it, and behind each what is likeliest then."""
        levels = [last[:, None]]
        for level in range(self.tree.depth):
            logits = self.m.logits(self.m.embed[levels[-1]])
            levels.append(logits[:, 0].topk(self.tree.width, dim=1).indices if level == 0 else logits.argmax(dim=2))
        return torch.cat(levels, dim=1)

    def step(self, last):
        """One step -> (tokens [B, depth + 1], how many of them are there [B], the next step's last token)."""
        tree, start = self.tree, self.lens.clone()
        tokens = self.guess(last)
        self.resize(start + tree.nodes, self.slots, self.cu)
        positions = (start.long()[:, None] + tree.depths).flatten().int()
        x = self._layers(tokens.flatten(), positions, self.slots,
                         lambda out, q, k, v: G.paged_attention_tree(out, q, k, v, self.no_prefix, self.tables, self.lens, self.cu, self.masks, positions,
                                                                     None, self.scale, self.max_len, tree.nodes, self.ws))
        said = self.m.logits(x).argmax(dim=1).view(self.B, tree.nodes)
        # from the root on to the child that is what the model says, as long as there is one
        b, at = torch.arange(self.B, device="cuda"), torch.zeros(self.B, dtype=torch.int64, device="cuda")
        path, out = [at], [said[:, 0]]
        count, going = torch.ones_like(at), torch.ones_like(at, dtype=torch.bool)
        parents = torch.tensor(tree.parents, device="cuda")
        for _ in range(tree.depth):
            fits = (parents[None] == at[:, None]) & (tokens == said[b, at][:, None])
            going = going & fits.any(dim=1)
            at = torch.where(going, fits.int().argmax(dim=1), at)
            path.append(at)
            out.append(said[b, at])
            count += going
        paths, kept = torch.stack(path, dim=1).int(), count.int()
        G.keep_tokens(self.caches, self.tables, start, paths, kept)
        self.resize(start + kept)
        return torch.stack(out, dim=1), kept, said[b, at]

    def decode(self, starts, count):
        """`count` tokens of each sequence behind its first own one -> (tokens [B, count], steps)."""
        last, said, steps = starts, [[] for _ in range(self.B)], 0
        while min(len(s) for s in said) < count:
            done = torch.tensor([len(s) >= count for s in said], device="cuda")
            before = self.lens.clone()
            got, kept, following = self.step(last)
            steps += 1
            for b, (row, n) in enumerate(zip(got.tolist(), kept.tolist())):
                said[b] += row[:n][:count - len(said[b])]
            # (a sequence that is done goes on from where it stands, its tokens unused)
            if bool(done.any()):
                self.resize(torch.where(done, before, self.lens))
            last = torch.where(done, last, following)
        return torch.tensor(said), steps


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--sequences", type=int, default=6)
    ap.add_argument("--prompt", type=int, default=300)
    ap.add_argument("--tokens", type=int, default=48)
    ap.add_argument("--width", type=int, default=3)
    ap.add_argument("--depth", type=int, default=3)
    ap.add_argument("--dtype", choices=("f16", "bf16"), default="bf16")
    ap.add_argument("--check", action="store_true")
    a = ap.parse_args(argv)
    torch.manual_seed(1)
    model = Model(torch.float16 if a.dtype == "f16" else torch.bfloat16)
    prompt, starts = torch.randint(0, model.vocab, (a.prompt,)).cuda(), torch.randint(0, model.vocab, (a.sequences,)).cuda()
    server = Server(model, prompt, a.sequences, a.tokens, Tree(a.width, a.depth))
    tokens, steps = server.decode(starts, a.tokens)
    print(f"{a.tokens} tokens of {a.sequences} sequences in {steps} steps with trees of {server.tree.nodes}; {server.tidy()} of {server.pool} blocks in use")
    if a.check:
        plain, single = Server(model, prompt, a.sequences, a.tokens, Tree(0, 0)).decode(starts, a.tokens)
        same = int((tokens == plain).all(dim=1).sum())
        print(f"without drafts: {single} steps; {same} of {a.sequences} sequences the same")
        return tokens, plain
    return tokens, None


if __name__ == "__main__":
    main()
