"""Prompts and drafted trees through blocks: each operator against 64 bits on the step's own values, and a captured round against the
eager one."""
import pytest
import torch

from block_common import *
from paper_2604_04701_amd import draft_step as D
from several_common import below, causal, rows64, verify64

pytestmark = pytest.mark.gpu


def start(kv_dtype, window=0, sinks=0, **kw):
    prompts = [40, 17, 1, 66]
    model = D.make(prompts=prompts, kv_dtype=kv_dtype, **kw)
    starts = [0]
    for n in prompts:
        starts.append(starts[-1] + n)
    tokens = torch.randint(0, model.vocab, (starts[-1],), generator=gen(2), device=DEV)
    return model, starts, model.prompt(tokens, starts, window, sinks)


@pytest.mark.parametrize("kv_dtype", [torch.float16, torch.int8])
def test_prompts_and_rounds_against_64_bits(kv_dtype):
    say(f"[draft] 2 blocks of 256, {kv_dtype}")
    model, starts, (out, seen, rows) = start(kv_dtype, 20, 3)
    assert torch.isfinite(out).all()
    for block, s in zip(model.blocks, seen):
        want, tol = rows64(s["q"], *block.cache, model.table, starts, model.lengths.tolist(), lambda _, n, length: causal(n, length, 20, 3), 0.125)
        check(s["o"], want, tol, "prompt")
    g, last, n, deepest = gen(3), torch.zeros(model.S, dtype=torch.int32, device=DEV), model.nodes, 0
    for _ in range(3):
        trees, said = model.draft(last, g)
        uniforms = torch.rand(trees.numel(), generator=g, device=DEV)
        model.place()
        r = model.at_round
        held = []
        # the caches as the attention sees them, before the accepted nodes move
        for b in model.for_round:
            b.attend = lambda q, batch, b=b: (held.append([None if x is None else x.clone() for x in b.cache]), D.SeveralBlock.attend(b, q, batch))[1]
        (path, counts, last), seen, target = model.round(trees, said, uniforms)
        torch.cuda.synchronize()
        edges = r.starts.tolist()
        for cache, s in zip(held, seen):
            want, tol = rows64(s["q"], *cache, model.table, edges, r.lengths.tolist(), lambda _, n, length: below(model.tree, length), 0.125)
            check(s["o"], want, tol, "tree")
        p, c, t = verify64(target, said, trees.tolist(), model.tree * model.S, uniforms.tolist(), edges)
        assert path.tolist() == p and counts.tolist() == c and last.tolist() == t
        deepest = max(deepest, *c)
        for cache, b in zip(held, model.for_round):
            for old, new in zip(cache, b.cache):
                if old is None:
                    continue
                for s in range(model.S):
                    for j in range(c[s]):
                        at, to = (int(model.lengths[s]) + x for x in (p[s * n + j], j))
                        at, to = ((int(model.table[s, x // 16]), x % 16) for x in (at, to))
                        assert torch.equal(new[to[0], :, to[1]], old[at[0], :, at[1]])
        model.keep(counts)
    assert deepest > 1                    # (nodes moved)
    with pytest.raises(ValueError):
        model.longest = model.max_tokens
        model.place()


def test_captured_rounds():
    say("[draft] captured round")
    B.muxq_init()
    model, _, _ = start(torch.int8)
    g, last = gen(4), torch.zeros(model.S, dtype=torch.int32, device=DEV)
    trees, said = model.draft(last, g)
    uniforms = torch.rand(trees.numel(), generator=g, device=DEV)
    model.place()
    caches = [x for b in model.blocks for x in b.cache if x is not None]

    def eager():
        kept = [x.clone() for x in caches]
        (path, counts, token), _, _ = model.round(trees, said, uniforms)
        after = [x.clone() for x in caches]
        for x, y in zip(caches, kept):
            x.copy_(y)
        return path, counts, token, after
    eager()
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    kept = [x.clone() for x in caches]
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        (path, counts, token), _, _ = model.round(trees, said, uniforms)
    torch.cuda.synchronize()
    for x, y in zip(caches, kept):
        x.copy_(y)
    for _ in range(3):
        want = eager()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(path, want[0]) and torch.equal(counts, want[1]) and torch.equal(token, want[2])
        for x, y in zip(caches, want[3]):
            assert torch.equal(x, y)
        model.keep(counts)
        a, b = model.draft(token, g)
        trees.copy_(a), said.copy_(b), uniforms.copy_(torch.rand(trees.numel(), generator=g, device=DEV))
        if model.longest + model.nodes <= model.max_tokens:
            model.place()


def test_fork():
    model, _, _ = start(torch.float16)
    model.fork(3, 0)
    torch.cuda.synchronize()
    assert model.lengths.tolist() == [66, 17, 1, 66]
    for b in model.blocks:
        for x in b.cache[:2]:
            assert torch.equal(x[model.table[0].long()], x[model.table[3].long()])
