"""A decode step of GPT-2 blocks with quantised projections: what stands between them, run together.

    python -m paper_2604_04701_amd.decode_block --width 1280 --heads 20 --blocks 4 --batch 24 --context 512

Each block is  norm -> c_attn (+ the request's adapter) -> keys and values to the paged cache, queries and keys
rotated if asked -> attention over the cache -> c_proj -> norm with the residual stream -> MLP,  all of it through
`binding`, with the channel maxima going from the first norm to c_attn (the MLP takes its own).  Weights are random, of GPT-2's
shapes; every sequence starts with a random cached context of its own length.  The step is captured in a HIP graph once and
replayed per token, the way a serving loop runs it; positions, lengths and slots are counted on up the device.
"""
import argparse
import time

import torch

from . import binding as B

DEV = "cuda"


def _weights(g, K, N):
    w = (0.02 * torch.randn(K, N, generator=g, device=DEV)).half()
    return *B.muxq_quantize_weight(w, "channel"), (0.02 * torch.randn(N, generator=g, device=DEV)).half()


class Block:
    """Weights, adapters, cache and workspaces of one block for a batch of S sequences."""

    def __init__(self, g, width, heads, S, n_pages, page, max_tokens, kv_dtype, adapters, rank):
        K = width
        self.K, self.heads, self.d, self.S = K, heads, width // heads, S
        self.c_attn, self.c_proj = _weights(g, K, 3 * K), _weights(g, K, K)
        self.c_fc, self.c_out = _weights(g, K, 4 * K), _weights(g, 4 * K, K)
        self.ln = [(torch.ones(K, dtype=torch.float16, device=DEV), torch.zeros(K, dtype=torch.float16, device=DEV)) for _ in range(2)]
        self.A = (torch.randn(adapters, rank, K, generator=g, device=DEV) / K ** 0.5).half()
        self.B = (0.1 * torch.randn(adapters, 3 * K, rank, generator=g, device=DEV)).half()
        self.scales = torch.ones(adapters, device=DEV)
        self.cache = B.alloc_kv_cache(n_pages, page, heads, self.d, kv_dtype)
        k, v, ks, vs = self.cache
        for x in (k, v):
            x.copy_(torch.randn(x.shape, generator=g, device=DEV) * (1 if kv_dtype == torch.float16 else 40))
        for x in (ks, vs):
            if x is not None:
                x.fill_(0.025)
        self.alloc_room(S, max_tokens)

    def alloc_room(self, S, max_tokens):
        """Workspaces for S rows."""
        K, heads = self.K, self.heads
        self.S = S
        self.ws_attn, self.lay = B.alloc_workspace(S, K, 3 * K, 64), B.workspace_layout(S, K, 3 * K, 64)
        self.ws_proj = B.alloc_workspace(S, K, K, 64)
        self.ws_mlp = torch.empty(B.lib().muxq_mlp_workspace_bytes(S, K, 4 * K, K, 64), dtype=torch.uint8, device=DEV)
        self.ws_kv = B.alloc_attention_workspace(S, heads, heads, self.d, max_tokens)

    def attend(self, q, batch):
        k, v, ks, vs = self.cache
        return B.muxq_paged_attention(q, k, v, batch.table, batch.lengths, batch.max_tokens, k_scale=ks, v_scale=vs, workspace=self.ws_kv)

    def step(self, x, stream, batch):
        """x: what the block before adds to the residual stream (or, with stream None, the stream itself).  Returns the
        same of this block, and everything in between by name."""
        K, S = self.K, self.S
        k, v, ks, vs = self.cache
        h, kept = B.muxq_norm(x, *self.ln[0], residual=stream, slabs=self.ws_attn[self.lay.absmax_partial:])
        stream = x if kept is None else kept
        w, s, b = self.c_attn
        qkv = B.muxq_linear(h, w, s, 3 * K, "channel", bias=b, workspace=self.ws_attn, absmax_ready=True,
                            absmax_slabs=B.norm_slabs(S, K))
        tuned = B.muxq_lora(h, self.A, self.B, self.scales, batch.starts, batch.adapters, qkv)
        q, kk, vv = tuned.view(S, 3 * self.heads, self.d).split(self.heads, 1)
        q = B.muxq_kv_append(kk, vv, batch.slots, k, v, k_scale=ks, v_scale=vs, q=q, positions=batch.positions, cos_sin=batch.cos_sin)
        o = self.attend(q, batch)
        w, s, b = self.c_proj
        a = B.muxq_linear(o.view(S, K), w, s, K, "channel", bias=b, workspace=self.ws_proj)
        h2, stream2 = B.muxq_norm(a, *self.ln[1], residual=stream)
        (w1, s1, b1), (w2, s2, b2) = self.c_fc, self.c_out
        _, y, _ = B.muxq_mlp(h2, w1, s1, 4 * K, w2, s2, K, "channel", bias1=b1, bias2=b2, workspace=self.ws_mlp)
        return y, stream2, {"stream": stream, "h": h, "qkv": qkv, "tuned": tuned, "q": q, "o": o, "a": a, "h2": h2, "stream2": stream2}


class Batch:
    """What the scheduler of a serving program keeps on the device for S sequences."""

    def __init__(self, g, S, lengths, max_tokens, page, d, adapters, rotated):
        per = -(-max_tokens // page)
        self.max_tokens, self.page, self.n_pages = max_tokens, page, S * per
        self.longest = 0                                 # of the lengths, known on the host
        self._grow(max(lengths) + 1)
        self.table = torch.randperm(self.n_pages, generator=g, device=DEV).int().view(S, per)
        self.positions = torch.tensor(lengths, dtype=torch.int32, device=DEV)       # of the new tokens
        self.lengths, self.slots = self.positions + 1, torch.empty_like(self.positions)
        self.starts = torch.arange(S + 1, dtype=torch.int32, device=DEV)
        self.adapters = torch.tensor([i % (adapters + 1) - 1 for i in range(S)], dtype=torch.int32, device=DEV)
        self.cos_sin = None
        if rotated:
            angle = torch.arange(max_tokens, device=DEV)[:, None] * 10000.0 ** (-torch.arange(d // 2, device=DEV) * 2.0 / d)
            self.cos_sin = torch.cat([angle.cos(), angle.sin()], 1).float().contiguous()
        self._place()

    def _grow(self, longest):
        if longest > self.max_tokens:
            raise ValueError(f"a sequence of {longest} tokens, where the tables and angles hold {self.max_tokens}")
        self.longest = longest

    def _place(self):
        at = self.positions.long()
        self.slots.copy_(self.table.gather(1, (at // self.page)[:, None])[:, 0] * self.page + at % self.page)

    def next_token(self):
        self._grow(self.longest + 1)
        self.positions += 1
        self.lengths += 1
        self._place()


def make(width=768, heads=12, blocks=2, S=5, context=100, new_tokens=8, page=16, kv_dtype=torch.int8, adapters=3, rank=8,
         rotated=False, seed=0):
    """Blocks, batch and the embedding of the first new tokens, all from the seed."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    lengths = [max(0, context - 7 * i * i % max(context, 1)) for i in range(S)]
    batch = Batch(g, S, lengths, context + new_tokens + 1, page, width // heads, adapters, rotated)
    stack = [Block(g, width, heads, S, batch.n_pages, page, batch.max_tokens, kv_dtype, adapters, rank) for _ in range(blocks)]
    return stack, batch, torch.randn(S, width, generator=g, device=DEV).half()


def run_step(stack, batch, x):
    """One token of every sequence through all blocks: the stream behind them, and what each block did."""
    stream, seen = None, []
    for block in stack:
        x, stream, inside = block.step(x, stream, batch)
        seen.append(inside)
    return stream + x, seen


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--width", type=int, default=1280)
    ap.add_argument("--heads", type=int, default=20)
    ap.add_argument("--blocks", type=int, default=4)
    ap.add_argument("--batch", type=int, default=24)
    ap.add_argument("--context", type=int, default=512)
    ap.add_argument("--tokens", type=int, default=32, help="half of them eager, half replayed")
    ap.add_argument("--fp16-cache", action="store_true")
    ap.add_argument("--rotated", action="store_true")
    args = ap.parse_args()
    if args.tokens < 2:
        ap.error("--tokens is 2 at least")
    B.muxq_init()
    stack, batch, x = make(args.width, args.heads, args.blocks, args.batch, args.context, args.tokens + 2,
                           kv_dtype=torch.float16 if args.fp16_cache else torch.int8, rotated=args.rotated)
    out, _ = run_step(stack, batch, x)
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        out, _ = run_step(stack, batch, x)
    torch.cuda.synchronize()
    times = {}
    for name, step in (("eager", lambda: run_step(stack, batch, x)), ("graph", graph.replay)):
        t0 = time.perf_counter()
        for _ in range(args.tokens // 2):
            batch.next_token()
            step()
        torch.cuda.synchronize()
        times[name] = (time.perf_counter() - t0) / (args.tokens // 2) * 1e6
    print(f"{args.blocks} blocks of {args.width}, {args.batch} sequences around {args.context} tokens, "
          f"{'fp16' if args.fp16_cache else '8-bit'} cache: {times['eager']:.0f} us a token eager, {times['graph']:.0f} us replayed; "
          f"finite: {bool(torch.isfinite(out).all())}")


if __name__ == "__main__":
    main()
