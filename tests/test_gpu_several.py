"""Attention of several new tokens, verification of drafted tokens, and pages moved within the cache: against 64 bits."""
import math

import pytest
import torch

from block_common import check, say
from paper_2604_04701_amd import binding as B
from several_common import *          # noqa: F401,F403
from several_common import Case, below, causal, random_tree, verify64

pytestmark = pytest.mark.gpu


def window(c, win=0, sinks=0, scale=None, max_new=None, max_length=None, **kw):
    starts, lengths = c.device()
    out = torch.full_like(c.q.contiguous(), math.nan)
    B.muxq_window_attention(c.q, c.k, c.v, c.table, starts, lengths, max_new or max(max(c.new), 1), max_length or max(max(c.lengths), 1),
                            window=win, sinks=sinks, scale=scale, out=out, **c.scales(), **kw)
    return out


def check_window(c, win=0, sinks=0, scale=None, what="window"):
    want, tol = c.exact(lambda s, n, length: causal(n, length, win, sinks) if length >= n else causal(n, n, win, sinks)[:, :0].new_zeros(n, length) | torch.cat(
        [torch.zeros(n - length, length, dtype=torch.bool), causal(length, length, win, sinks)]), scale)
    check(window(c, win, sinks, scale), want, tol, what)


# new tokens and lengths of each sequence, heads, and the page
BATCHES = {
    "one": ([1], [1], 4, 4, 64, 16),
    "one_behind": ([1], [513], 4, 2, 64, 16),
    "decode": ([1] * 7, [1, 0, 17, 300, 64, 33, 128], 8, 2, 64, 16),
    "decode_group7": ([1] * 3, [70, 1000, 5], 14, 2, 128, 32),
    "prompt": ([77], [77], 4, 4, 64, 16),
    "prompt_128": ([128], [128], 3, 3, 128, 8),
    "prompt_behind": ([65, 3, 200], [129, 3, 771], 6, 2, 128, 64),
    "ragged": ([1, 33, 0, 300, 7, 64], [900, 33, 50, 301, 2000, 64], 4, 1, 64, 16),
    "more_rows_than_tokens": ([9, 5], [4, 0], 4, 2, 64, 16),
    "long": ([700], [700], 2, 1, 64, 256),
    "many_rows": ([300, 290], [1300, 290], 8, 1, 128, 32),
}


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("win,sinks", [(0, 0), (64, 4), (1, 0), (37, 70)])
@pytest.mark.parametrize("name", BATCHES)
def test_windows(name, win, sinks, bits):
    new, lengths, H, heads, d, page = BATCHES[name]
    say(f"[case] window {name} window={win} sinks={sinks} bits={bits}")
    check_window(Case(11, new, lengths, H, heads, d, page, bits), win, sinks, what=name)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("win,sinks", [(0, 0), (700, 45), (1, 33), (33, 1), (128, 0), (100, 1000), (2000, 64), (5000, 3)])
@pytest.mark.parametrize("H,heads,d,page", [(8, 4, 64, 8), (5, 1, 128, 16), (40, 2, 80, 64), (6, 6, 32, 256)])
def test_single_rows(H, heads, d, page, win, sinks, bits):
    """At most a row of each sequence: rows and sequences do not go by the same numbers."""
    say(f"[case] single rows {H} of {heads} d={d} page={page} window={win} sinks={sinks} bits={bits}")
    check_window(Case(17, [1, 0, 1, 1, 1, 0, 1, 1], [2300, 5, 1000, 9, 1, 0, 0, 131], H, heads, d, page, bits), win, sinks, what="single rows")


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("layout", ["heads", "tokens"])
@pytest.mark.parametrize("d", [16, 48, 80, 96, 144, 256])
def test_head_sizes(d, layout, bits):
    say(f"[case] window d={d} {layout} bits={bits}")
    check_window(Case(d, [40, 1, 130], [100, 300, 130], 6, 2, d, 16, bits, layout, columns=True), 90, 3, what=f"d={d}")


# batches that fill the chip with tiles of 64 and of 128 rows
FULL = {"rows128": ([150] * 9 + [131, 140, 150], [150 + 31 * i for i in range(12)], 32, 16, 128), "rows128_d80": ([150] * 12, [400] * 11 + [150], 32, 16, 80),
        "rows128_d64": ([100] * 12, [100 + 50 * i for i in range(12)], 48, 24, 64), "rows64": ([60, 33] * 20, [60, 333] * 20, 16, 16, 64),
        "rows64_d128": ([60, 64] * 20, [160, 64] * 20, 16, 16, 128), "heads256": ([100] * 4, [100, 130, 333, 1000], 12, 6, 256),
        "rows128_of_64": ([200] * 9 + [131], [200 + 31 * i for i in range(10)], 104, 52, 64), "rows64_of_64": ([60, 33] * 26, [60, 133] * 26, 16, 16, 64),
        "rows128_in_pieces": ([260, 1, 200], [900, 2000, 260], 32, 8, 128), "rows64_in_pieces": ([64, 3], [1500, 64], 16, 4, 80)}


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("win,sinks", [(0, 0), (70, 5)])
@pytest.mark.parametrize("layout", ["heads", "tokens"])
@pytest.mark.parametrize("name", FULL)
def test_full_batches(name, layout, win, sinks, bits):
    new, lengths, H, heads, d = FULL[name]
    say(f"[case] full {name} {layout} window={win} sinks={sinks} bits={bits}")
    check_window(Case(13, new, lengths, H, heads, d, 32, bits, layout), win, sinks, what=name)


@pytest.mark.parametrize("H,heads", [(1, 1), (5, 1), (32, 1), (40, 1), (12, 4), (130, 2)])
def test_groups(H, heads):
    say(f"[case] window {H} of {heads}")
    check_window(Case(H, [3, 50, 1], [30, 50, 400], H, heads, 64, 16), 0, 0, what=f"{H} of {heads}")


@pytest.mark.parametrize("scale", [0.0, -0.3, 3.0, 1e-6])
def test_scales(scale):
    say(f"[case] window scale={scale}")
    check_window(Case(3, [40, 1], [100, 300], 4, 2, 64, 16), 50, 2, scale=scale, what=f"scale={scale}")


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("kind", ["tree", "chain", "star", "forest"])
@pytest.mark.parametrize("new,lengths,H,heads,d", [
    ([1], [1], 4, 4, 64), ([8], [45], 12, 12, 64), ([64, 64], [64, 1000], 8, 2, 128), ([31, 1, 0, 64, 17], [31, 200, 30, 77, 900], 4, 1, 64),
    ([33, 20], [300, 25], 6, 6, 256), ([5], [2000], 32, 8, 128),
    ([64, 50, 64] * 3, [64, 700, 300] * 3, 16, 8, 128), ([40, 37] * 4, [100, 340] * 4, 64, 32, 64), ([30, 40], [800, 40], 12, 12, 80),
    ([9, 5, 64], [4, 0, 63], 4, 2, 64)])
def test_trees(new, lengths, H, heads, d, kind, bits):
    say(f"[case] tree {new} {lengths} {H} of {heads} d={d} {kind} bits={bits}")
    c = Case(5, new, lengths, H, heads, d, 16, bits)
    trees = [random_tree(n, 7 + i, kind) for i, n in enumerate(new)]
    starts, lens = c.device()
    out = torch.full_like(c.q, math.nan)
    B.muxq_tree_attention(c.q, c.k, c.v, c.table, starts, lens, ints([p for t in trees for p in t]), max(new), max(lengths), out=out, **c.scales())
    want, tol = c.exact(lambda s, n, length: below(trees[s], length))
    check(out, want, tol, kind)


@pytest.mark.parametrize("V", [1, 5, 1000, 1024, 1025, 50257, 131073])
@pytest.mark.parametrize("how", ["sampled", "given", "greedy"])
def test_verification(V, how):
    say(f"[case] verify V={V} {how}")
    g = gen(V)
    new = [9, 1, 0, 64, 30, 2, 17]
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    M = starts[-1]
    parents = [p for i, n in enumerate(new) for p in random_tree(n, i, ["tree", "chain", "star", "forest"][i % 4])]
    logits = 2.0 * torch.randn(M, V, generator=g, device=DEV)
    target = torch.softmax(logits, 1)
    draft = torch.softmax(logits + 0.5 * torch.randn(M, V, generator=g, device=DEV), 1)
    at = 0
    tokens = torch.zeros(M, dtype=torch.int64, device=DEV)
    for n in new:
        for i in range(1, n):
            up = at + max(parents[at + i], 0)
            tokens[at + i] = target[up].argmax() if how == "greedy" and i % 2 else torch.multinomial(draft[up], 1, generator=g)[0]
        at += n
    uniforms = None if how == "greedy" else torch.rand(M, generator=g, device=DEV)
    if how != "sampled":
        draft = None
    got = B.muxq_verify_tree(target, tokens.int(), ints(starts), ints(parents), 64, draft=draft, uniforms=uniforms)
    want = verify64(target, draft, tokens.tolist(), parents, None if uniforms is None else uniforms.tolist(), starts)
    for x, y in zip(got, want):
        assert x.tolist() == y


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("heads,d,page,layout", [(4, 64, 16, "heads"), (4, 64, 16, "tokens"), (1, 16, 8, "heads"), (3, 80, 256, "tokens"),
                                                 (8, 128, 32, "heads"), (1, 256, 64, "tokens")])
def test_copies(heads, d, page, layout, bits):
    say(f"[case] copy {heads} heads of {d}, pages of {page}, {layout}, bits={bits}")
    g = gen(d)
    k, v, ks, vs = make_cache(g, 40, heads, page, d, bits, layout)
    order = torch.randperm(40, generator=g, device=DEV)
    src, dst = order[:15].int(), order[15:30].int()
    src[3], dst[5], dst[7] = -1, 40, src[7]
    want = [None if x is None else x.clone() for x in (k, v, ks, vs)]
    for i, (a, b) in enumerate(zip(src.tolist(), dst.tolist())):
        if i not in (3, 5):
            for x in want:
                if x is not None:
                    x[b] = x[a]
    B.muxq_kv_copy(src, dst, k, v, k_scale=ks, v_scale=vs)
    for x, y in zip((k, v, ks, vs), want):
        assert x is None or torch.equal(x, y)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("heads,d,page,layout", [(4, 64, 16, "heads"), (4, 64, 16, "tokens"), (1, 16, 8, "heads"), (3, 256, 32, "tokens")])
def test_compaction(heads, d, page, layout, bits):
    say(f"[case] compact {heads} heads of {d}, pages of {page}, {layout}, bits={bits}")
    new, lengths = [8, 64, 1, 0, 30, 5], [20, 100, 7, 9, 30, 4]
    c = Case(2, new, lengths, heads, heads, d, page, bits, layout)
    paths = [[0, 1, 2, 5], sorted(range(0, 64, 3)) + [63], [0], [], [0, 29, 3, 4, 2, 1, -1, 30, 7], [0, 1]]
    flat, counts = [], [len(p) for p in paths]
    for n, p in zip(new, paths):
        flat += (p + [-1] * n)[:n]
    want = [None if x is None else x.clone() for x in (c.k, c.v, c.ks, c.vs)]

    def place(s, t):
        return int(c.table[s, t // page]), t % page
    for s, (n, p) in enumerate(zip(new, paths)):
        first = lengths[s] - n
        for j, x in enumerate(p):
            if 0 <= x < n and first >= 0:
                (a, i), (b, y) = place(s, first + x), place(s, first + j)
                for w, old in zip(want, (c.k, c.v, c.ks, c.vs)):
                    if w is not None:
                        w[b, :, y] = old[a, :, i]
    starts, lens = c.device()
    B.muxq_kv_compact(ints(flat), ints(counts), starts, lens, c.table, c.k, c.v, 64, **c.scales())
    for x, y in zip((c.k, c.v, c.ks, c.vs), want):
        assert x is None or torch.equal(x.nan_to_num(7.0) if x.is_floating_point() else x, y.nan_to_num(7.0) if y.is_floating_point() else y)
