"""Prompts and drafted trees through GPT-2 blocks with quantised projections: what a serving loop does with several new tokens.

    python -m paper_2604_04701_amd.draft_step --width 768 --heads 12 --blocks 4 --batch 8 --prompt 300 --nodes 16

A prompt of every sequence goes through the blocks of decode_block.py in one packed batch, attending causally.  Then rounds
follow: a draft proposes a tree of tokens behind each sequence's last one, the blocks see all nodes at once (each node the tokens
before the tree and the nodes above it), the head gives the target's probabilities after every node, the verification says which
nodes stand and what comes after them, and their keys and values move to the front in every block's cache.  The nodes of a tree
have no window; a prompt may have one (Model.prompt), but as soon as sequences are longer than that the two are different models.
Weights are random; the draft is a bigram model of the embedding, as undecided as the target is, so that many of its tokens stand.
"""
import argparse
import copy
import time
import warnings

import torch

from . import binding as B
from .decode_block import Block, run_step

DEV = "cuda"


class SeveralBlock(Block):
    """A block whose rows are several new tokens of each sequence."""

    def rows(self, M, max_tokens, S, most_new, window, sinks):
        """The same weights and cache with room for M rows, at most most_new of a sequence."""
        other = copy.copy(self)
        other.alloc_room(M, max_tokens)
        other.ws_window = B.alloc_window_attention_workspace(S, self.heads, self.heads, self.d, most_new, max_tokens, window, sinks, DEV)
        other.ws_tree = B.alloc_tree_attention_workspace(S, self.heads, self.heads, self.d, min(most_new, 64), max_tokens, DEV)
        return other

    def attend(self, q, batch):
        k, v, ks, vs = self.cache
        if batch.parents is None:
            return B.muxq_window_attention(q, k, v, batch.table, batch.starts, batch.lengths, batch.most_new, batch.max_tokens,
                                           window=batch.window, sinks=batch.sinks, k_scale=ks, v_scale=vs, workspace=self.ws_window)
        return B.muxq_tree_attention(q, k, v, batch.table, batch.starts, batch.lengths, batch.parents, batch.most_new, batch.max_tokens,
                                     k_scale=ks, v_scale=vs, workspace=self.ws_tree)


class Rows:
    """What a step needs to know of its rows."""

    def __init__(self, model, starts, parents=None, most_new=1, window=0, sinks=0):
        self.table, self.max_tokens, self.cos_sin, self.adapters = model.table, model.max_tokens, model.cos_sin, model.adapters
        self.starts, self.parents, self.most_new, self.window, self.sinks = starts, parents, most_new, window, sinks
        self.lengths = self.positions = self.slots = None


def tree(nodes, branch):
    """Parents and depths of a tree in the order of its levels."""
    parents = [(i - 1) // branch if i else -1 for i in range(nodes)]
    depth = []
    for p in parents:
        depth.append(0 if p < 0 else depth[p] + 1)
    return parents, depth


def reach(longest, nodes, branch, rounds):
    """The tokens that a sequence may come to: its prompt, the deepest path of every round, and one more tree."""
    return longest + rounds * (max(tree(nodes, branch)[1]) + 1) + nodes


class Model:
    def __init__(self, width, heads, blocks, prompts, nodes, branch, rounds, vocab, page, kv_dtype, adapters, rank, rotated, seed):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        self.S, self.nodes, self.page, self.vocab = len(prompts), nodes, page, vocab
        self.tree, self.depth = tree(nodes, branch)
        self.deepest = max(self.depth) + 1
        self.longest = max(prompts)                       # of the lengths, known on the host
        self.window = 0                                   # of the prompts
        self.max_tokens = reach(self.longest, nodes, branch, rounds)
        per = -(-self.max_tokens // page)
        self.table = torch.randperm(self.S * per, generator=g, device=DEV).int().view(self.S, per)
        self.lengths = torch.zeros(self.S, dtype=torch.int32, device=DEV)          # tokens that stand in the cache
        self.adapters = torch.tensor([i % (adapters + 1) - 1 for i in range(self.S)], dtype=torch.int32, device=DEV)
        self.cos_sin = None
        if rotated:
            half = width // heads // 2
            angle = torch.arange(self.max_tokens, device=DEV)[:, None] * 10000.0 ** (-torch.arange(half, device=DEV) / half)
            self.cos_sin = torch.cat([angle.cos(), angle.sin()], 1).float().contiguous()
        self.embedding = torch.randn(vocab, width, generator=g, device=DEV).half()
        self.final = (torch.ones(width, dtype=torch.float16, device=DEV), torch.zeros(width, dtype=torch.float16, device=DEV))
        padded = -(-vocab // 8) * 8
        head = torch.zeros(width, padded, dtype=torch.float16, device=DEV)
        head[:, :vocab] = (0.02 * torch.randn(width, vocab, generator=g, device=DEV)).half()
        self.head, self.padded = B.muxq_quantize_weight(head, "channel"), padded
        self.blocks = [SeveralBlock(g, width, heads, 1, self.S * per, page, self.max_tokens, kv_dtype, adapters, rank) for _ in range(blocks)]
        n = nodes
        self.at_round = Rows(self, torch.arange(0, self.S * n + 1, n, dtype=torch.int32, device=DEV),
                             torch.tensor(self.tree * self.S, dtype=torch.int32, device=DEV), n)
        self.for_round = [b.rows(self.S * n, self.max_tokens, self.S, n, 0, 0) for b in self.blocks]
        self.depths = torch.tensor(self.depth, dtype=torch.int32, device=DEV)

    def _slots(self, sequence, token):
        return (self.table[sequence, (token // self.page)].long() * self.page + token % self.page).int()

    def prompt(self, tokens, starts, window=0, sinks=0):
        """Packed prompts, tokens [M] and starts (a list of S + 1): the stream behind the blocks."""
        new = [b - a for a, b in zip(starts, starts[1:])]
        if len(new) != self.S or starts[0] != 0 or min(new) < 0 or not tokens.numel() == starts[-1] > 0:
            raise ValueError(f"starts {starts} do not divide {tokens.numel()} tokens into {self.S} prompts")
        M, most = starts[-1], max(new)
        if most > self.max_tokens:
            raise ValueError(f"a prompt of {most} tokens, where the tables and angles hold {self.max_tokens}")
        rows = Rows(self, torch.tensor(starts, dtype=torch.int32, device=DEV), None, most, window, sinks)
        sequence = torch.repeat_interleave(torch.arange(self.S, device=DEV), torch.tensor(new, device=DEV))
        rows.positions = torch.cat([torch.arange(n, device=DEV) for n in new]).int()
        rows.slots = self._slots(sequence, rows.positions.long())
        rows.lengths = torch.tensor(new, dtype=torch.int32, device=DEV)
        stack = [b.rows(M, self.max_tokens, self.S, most, window, sinks) for b in self.blocks]
        out, seen = run_step(stack, rows, self.embedding[tokens.long()])
        self.lengths.copy_(rows.lengths)
        self.longest, self.window = most, window
        return out, seen, rows

    def draft(self, last, generator=None):
        """Trees behind the last tokens [S]: (tokens [S * nodes], probabilities [S * nodes, vocab])."""
        tokens = torch.zeros(self.S, self.nodes, dtype=torch.int64, device=DEV)
        tokens[:, 0] = last.long()
        emb = self.embedding.float()
        said = torch.empty(self.S, self.nodes, self.vocab, device=DEV)
        for i in range(self.nodes):
            if i:
                tokens[:, i] = torch.multinomial(said[:, self.tree[i]], 1, generator=generator)[:, 0]
            said[:, i] = torch.softmax(emb[tokens[:, i]] @ emb.t() / emb.shape[1], 1)
        return tokens.int().view(-1), said.view(-1, self.vocab)

    def place(self):
        """Where the next trees stand."""
        if self.longest + self.nodes > self.max_tokens:
            raise ValueError(f"trees up to token {self.longest + self.nodes}, where the tables and angles hold {self.max_tokens}")
        if 0 < self.window < self.longest + self.nodes:
            warnings.warn(f"the prompts had a window of {self.window} tokens, the nodes of a tree see all tokens: another model")
        r, n = self.at_round, torch.arange(self.nodes, device=DEV)
        at = self.lengths[:, None] + n
        positions = (self.lengths[:, None] + self.depths).view(-1).int()
        slots = self._slots(torch.arange(self.S, device=DEV)[:, None], at.long()).view(-1)
        lengths = self.lengths + self.nodes
        if r.lengths is None:
            r.positions, r.slots, r.lengths = positions, slots, lengths
        else:                                             # in place: a captured round reads them there
            r.positions.copy_(positions), r.slots.copy_(slots), r.lengths.copy_(lengths)

    def round(self, tokens, said, uniforms):
        """The trees through the blocks, verified, and what stands of them moved to the front: (path, counts, next tokens), and what the
        blocks saw."""
        r = self.at_round
        stream, seen = run_step(self.for_round, r, self.embedding[tokens.long()])
        h, _ = B.muxq_norm(stream, *self.final)
        logits = B.muxq_linear(h, *self.head, self.padded, "channel")
        target = torch.softmax(logits[:, :self.vocab].float(), 1)
        path, counts, token = B.muxq_verify_tree(target, tokens, r.starts, r.parents, self.nodes, draft=said, uniforms=uniforms)
        for b in self.for_round:
            k, v, ks, vs = b.cache
            B.muxq_kv_compact(path, counts, r.starts, r.lengths, self.table, k, v, self.nodes, k_scale=ks, v_scale=vs)
        return (path, counts, token), seen, target

    def keep(self, counts):
        """The accepted nodes are part of their sequences."""
        self.lengths += counts
        self.longest += self.deepest

    def fork(self, source, target):
        """Sequence `target` becomes a copy of sequence `source`, with pages of its own."""
        for b in self.blocks:
            k, v, ks, vs = b.cache
            B.muxq_kv_copy(self.table[source], self.table[target], k, v, k_scale=ks, v_scale=vs)
        self.lengths[target] = self.lengths[source]


def make(width=256, heads=4, blocks=2, prompts=(40, 17, 1), nodes=13, branch=3, rounds=3, vocab=1000, page=16, kv_dtype=torch.int8,
         adapters=2, rank=8, rotated=True, seed=0):
    return Model(width, heads, blocks, list(prompts), nodes, branch, rounds, vocab, page, kv_dtype, adapters, rank, rotated, seed)


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--width", type=int, default=768)
    ap.add_argument("--heads", type=int, default=12)
    ap.add_argument("--blocks", type=int, default=4)
    ap.add_argument("--batch", type=int, default=8)
    ap.add_argument("--prompt", type=int, default=300)
    ap.add_argument("--window", type=int, default=0, help="of the prompts, at least what a sequence comes to: trees have none")
    ap.add_argument("--nodes", type=int, default=16)
    ap.add_argument("--branch", type=int, default=2)
    ap.add_argument("--rounds", type=int, default=8)
    ap.add_argument("--vocab", type=int, default=50257)
    ap.add_argument("--fp16-cache", action="store_true")
    args = ap.parse_args()
    most = reach(max(1, args.prompt), args.nodes, args.branch, args.rounds + 1)
    if 0 < args.window < most:
        ap.error(f"a window of {args.window} tokens: the nodes of a tree see all of up to {most}, which is another model")
    B.muxq_init()
    prompts = [max(1, args.prompt - 11 * i) for i in range(args.batch)]
    model = make(args.width, args.heads, args.blocks, prompts, args.nodes, args.branch, args.rounds + 1, args.vocab,
                 kv_dtype=torch.float16 if args.fp16_cache else torch.int8)
    starts = [0]
    for n in prompts:
        starts.append(starts[-1] + n)
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    tokens = torch.randint(0, args.vocab, (starts[-1],), generator=g, device=DEV)
    model.prompt(tokens, starts, args.window, 4)
    last, kept, spent = torch.zeros(args.batch, dtype=torch.int32, device=DEV), 0, []
    for i in range(args.rounds + 1):
        trees, said = model.draft(last, g)
        uniforms = torch.rand(trees.numel(), generator=g, device=DEV)
        model.place()
        torch.cuda.synchronize()
        t = time.perf_counter()
        (_, counts, last), _, _ = model.round(trees, said, uniforms)
        torch.cuda.synchronize()
        if i:                                             # (the first one loads kernels)
            spent.append(time.perf_counter() - t)
        model.keep(counts)
        kept += int(counts.sum())
    print(f"{args.blocks} blocks of {args.width}, {args.batch} prompts to {args.prompt} tokens, trees of {args.nodes}: "
          f"{sorted(spent)[len(spent) // 2] * 1e6:.0f} us a round, {kept / (args.rounds + 1) / args.batch:.2f} tokens a sequence and round stand")


if __name__ == "__main__":
    main()
