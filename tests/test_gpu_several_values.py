"""Several new tokens where it can go wrong: infinities, NaN, pages that are missing, workspaces, streams, graphs, offsets beyond 32 bits."""
import math

import pytest
import torch

from block_common import check, say
from paper_2604_04701_amd import binding as B
from several_common import *          # noqa: F401,F403
from several_common import Case, below, causal, random_tree, verify64

pytestmark = pytest.mark.gpu


def window(c, win=0, sinks=0, **kw):
    starts, lengths = c.device()
    return B.muxq_window_attention(c.q, c.k, c.v, c.table, starts, lengths, max(max(c.new), 1), max(max(c.lengths), 1), window=win, sinks=sinks,
                                   **c.scales(), **kw)


def place(c, s, t):
    return int(c.table[s, t // c.page]), t % c.page


SHAPES = {"few": ([5, 1], [70, 300], 4, 4, 64), "wide": ([1, 7], [200, 77], 8, 4, 128), "rows64": ([60, 60, 61], [60, 200, 61], 4, 4, 64),
          "rows128": ([130, 128], [130, 300], 4, 2, 128), "full128": ([130] * 12, [130] * 11 + [200], 32, 16, 128), "full80": ([130] * 12, [130] * 11 + [200], 32, 16, 80), "many": ([300] * 12, [300] * 12, 24, 12, 64), "heads256": ([40, 3], [40, 90], 2, 1, 256),
          "full64": ([130] * 12, [130] * 11 + [200], 60, 30, 64), "split128": ([130] * 3, [130, 150, 900], 32, 16, 128),
          "single": ([1, 1, 1], [70, 5, 300], 8, 2, 64), "single80": ([1, 0, 1], [40, 3, 900], 4, 4, 80)}


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("name", SHAPES)
def test_infinite_values(name, bits):
    """An infinite value makes the sums of the rows that see it infinite, and no others; two of different signs, or NaN, make NaN."""
    say(f"[case] infinite values {name} bits={bits}")
    new, lengths, H, heads, d = SHAPES[name]
    c = Case(4, new, lengths, H, heads, d, 16, bits)
    s, n, length = len(new) - 1, new[-1], lengths[-1]
    t, late = length - max(1, n // 2), length - 1
    (p0, i0), (p1, i1) = place(c, s, t), place(c, s, late)
    if bits == 16:
        c.v[p0, 0, i0, 3] = math.inf
        c.v[p0, 0, i0, d - 1] = math.nan
        if late != t:
            c.v[p1, 0, i1, 3] = -math.inf
        infinite = {3: math.inf, d - 1: math.nan}
    else:
        c.v[p0, 0, i0] = torch.arange(d, device=DEV).sub(5).clamp(-127, 127).to(torch.int8)         # negative, 0, positive
        c.vs[p0, 0, i0] = math.inf
        infinite = {e: (e - 5) * math.inf for e in range(d)}
    got = window(c).float()
    clean = Case(4, new, lengths, H, heads, d, 16, bits)
    plain, group = window(clean).float(), H // heads
    seen = causal(n, length, 0, 0)
    for m in range(c.starts[-1]):
        i = m - c.starts[s]
        for h in range(H):
            for e in range(d):
                if i >= 0 and h < group and e in infinite and seen[i, t]:
                    want = infinite[e]
                    if bits == 16 and e == 3 and late != t and seen[i, late]:
                        want = math.nan
                    x = got[m, h, e].item()
                    assert (math.isnan(x) and math.isnan(want)) or x == want, (m, h, e, x, want)
                    plain[m, h, e] = got[m, h, e] = 0.0
    if bits == 8:                         # (the codes of that token are others: rows that see it differ)
        for i in range(n):
            if seen[i, t]:
                got[c.starts[s] + i, :group] = plain[c.starts[s] + i, :group] = 0.0
    assert torch.isfinite(got).all() and (got - plain).abs().max() <= 2.0 ** -10 * plain.abs().max()


@pytest.mark.parametrize("kind", ["causal", "window", "tree"])
@pytest.mark.parametrize("name", SHAPES)
def test_large_scales_in_places_that_a_row_does_not_see(name, kind):
    """Weights are cut by the largest scale of a value; one that other rows of the batch see, or none, changes no bit of a row."""
    say(f"[case] large scales {name} {kind}")
    new, lengths, H, heads, d = SHAPES[name]
    if kind == "tree":
        new = [min(n, 64) for n in new]
    s, n, length, group = len(new) - 1, new[-1], lengths[-1], H // heads
    win = 9 if kind == "window" else 0
    parents = sum((random_tree(n, i) for i, n in enumerate(new)), [])
    seen = below(parents[-n:], length) if kind == "tree" else causal(n, length, win, 0)
    places = [max(0, length - max(1, n // 2))] if kind != "window" else [length - 1, max(0, length - n - 20), max(0, length - n // 2 - 12)]
    found = []
    for large in (False, True):
        c = Case(6, new, lengths, H, heads, d, 16, 8)
        starts, at = c.device()
        for t in places if large else []:
            page, i = place(c, s, t)
            c.vs[page, :, i] = 1e30
        if kind == "tree":
            found.append(B.muxq_tree_attention(c.q, c.k, c.v, c.table, starts, at, ints(parents), max(new), max(lengths), **c.scales()))
        else:
            found.append(window(c, win))
    clear = ~seen[:, places].any(1)
    assert clear.any() or n == 1 or kind == "window"
    plain, got = (x[c.starts[s]:][clear] for x in found)
    assert torch.equal(plain, got), (plain.float() - got.float()).abs().max()
    assert torch.equal(found[0][:c.starts[s]], found[1][:c.starts[s]])


def test_more_infinite_tiles_than_are_remembered():
    say("[case] infinite values in 60 tiles")
    c = Case(9, [40], [64 * 70], 2, 2, 128, 16)
    for t in range(10, 64 * 60, 64):
        p, i = place(c, 0, t)
        c.v[p, 1, i, 7] = math.inf if t < 64 * 59 else -math.inf
    got = window(c)
    assert torch.isnan(got[:, 1, 7]).all() and torch.isfinite(got[:, 0]).all() and torch.isfinite(got[:, 1, :7]).all()
    assert torch.isfinite(window(c, 64, 4)).all()              # behind the window
    assert torch.isinf(window(c, 64, 20)[:, 1, 7]).all()


def test_scores_of_minus_infinity():
    say("[case] scores of -infinity")
    c = Case(6, [3, 2], [3, 50], 2, 1, 64, 16)
    c.q[:, :, 0] = 1.0
    p, i = place(c, 0, 0)
    c.k[p, 0, i, 0] = -math.inf
    got = window(c)
    assert torch.isnan(got[0]).all()                              # its only token
    assert torch.isfinite(got[1:]).all()
    c.k[p, 0, i + 1, 0] = math.inf
    got = window(c)
    assert torch.isnan(got[:3]).all() and torch.isfinite(got[3:]).all()


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("name", SHAPES)
def test_missing_pages(name, bits):
    """Tokens of pages outside the cache are left out; a row that has no others is zeros."""
    say(f"[case] missing pages {name} bits={bits}")
    new, lengths, H, heads, d = SHAPES[name]
    c = Case(8, new, lengths, H, heads, d, 8, bits)
    c.table[0, 0] = -1
    c.table[1, ::2] = c.n_pages
    c.table[1, 3] = -5
    want, tol = c.exact(lambda s, n, length: causal(n, length, 0, 0))
    got = window(c)
    check(got, want, tol, name)
    assert (got[(want == 0).all(2)] == 0).all()
    c.table[:] = -1
    assert (window(c) == 0).all()


def test_rows_of_no_sequence_stay_as_they_were():
    say("[case] rows of no sequence")
    c = Case(2, [4, 9, 2], [40, 300, 2], 4, 2, 64)
    starts, lengths = c.device()
    q = torch.cat([c.q, c.q])
    out = torch.full_like(q, 7.0)
    for most in (9, 8):                   # the second sequence has more rows than 8: it counts as one without
        out.fill_(7.0)
        B.muxq_window_attention(q, c.k, c.v, c.table, starts, lengths, most, 300, out=out)
        touched = [*range(4), *(range(4, 13) if most == 9 else ()), 13, 14]
        left = [m for m in range(30) if m not in touched]
        assert (out[left] == 7.0).all() and not (out[touched] == 7.0).all(2).any()
    starts = ints([3, 3, 5, 1 << 30])     # clamped to the rows there are
    out.fill_(7.0)
    B.muxq_window_attention(q, c.k, c.v, c.table, starts, lengths, 30, 300, out=out)
    assert (out[:3] == 7.0).all() and not (out[3:] == 7.0).all(2).any()


def test_lengths_beyond_the_bound():
    say("[case] lengths beyond max_length")
    c = Case(2, [4], [200], 4, 2, 64)
    starts, _ = c.device()
    a = B.muxq_window_attention(c.q, c.k, c.v, c.table, starts, ints([150]), 4, 150)
    b = B.muxq_window_attention(c.q, c.k, c.v, c.table, starts, ints([2000]), 4, 150)
    assert torch.equal(a, b)
    assert (B.muxq_window_attention(c.q, c.k, c.v, c.table, starts, ints([-3]), 4, 150) == 0).all()


@pytest.mark.parametrize("tree", [False, True])
def test_one_workspace_for_calls_of_all_sizes(tree):
    """The workspace of the largest call serves smaller ones, which are cut into other pieces, one behind the other on a stream."""
    say(f"[case] one workspace, tree={tree}")
    H, heads, d = 8, 2, 128
    if tree:
        ws = B.alloc_tree_attention_workspace(9, H, heads, d, 64, 5000)
    else:
        ws = B.alloc_window_attention_workspace(9, H, heads, d, 70, 5000)
    ws.fill_(255)                         # NaN everywhere
    cases = [Case(i, new, lengths, H, heads, d, 16, 16 if i % 2 else 8) for i, (new, lengths) in enumerate(
        [([1], [5000]), ([3, 1], [4000, 1]), ([64], [3000]), ([20] * 9, [500] * 9), ([9], [1200]), ([1] * 9, [4999] * 9), ([33, 64], [64, 5000])])]
    outs = []
    for c in cases:
        starts, lengths = c.device()
        if tree:
            trees = [random_tree(n, n) for n in c.new]
            outs.append(B.muxq_tree_attention(c.q, c.k, c.v, c.table, starts, lengths, ints([p for t in trees for p in t]), max(c.new), max(c.lengths),
                                              workspace=ws, **c.scales()))
        else:
            outs.append(window(c, workspace=ws))
    for c, out in zip(cases, outs):
        want, tol = c.exact((lambda s, n, length: below(random_tree(n, n), length)) if tree else (lambda s, n, length: causal(n, length, 0, 0)))
        check(out, want, tol, f"{c.new} of {c.lengths}")


def test_the_same_call_gives_the_same_bits():
    say("[case] same bits")
    c = Case(1, [1, 40, 7], [4000, 900, 2500], 8, 2, 64)
    first = window(c)
    for _ in range(3):
        assert torch.equal(window(c), first)


def test_other_streams():
    say("[case] other streams")
    c = Case(1, [3, 40], [2000, 900], 8, 2, 64)
    want = window(c)
    torch.cuda.synchronize()
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    outs = []
    for s in (a, b, a):                   # two at once, each with a workspace of its own
        with torch.cuda.stream(s):
            outs.append(window(c))
    torch.cuda.synchronize()
    for out in outs:
        assert torch.equal(out, want)


def test_captured_calls():
    """All entry points in one graph, replayed on new inputs, the program's own work between the replays."""
    say("[case] captured calls")
    B.muxq_init()
    c = Case(1, [8, 8, 8], [2000, 900, 40], 8, 2, 64, 16, 8)
    starts, lengths = c.device()
    parents = ints(random_tree(8, 1) * 3)
    g, V, M = gen(5), 777, 24
    target = torch.softmax(2 * torch.randn(M, V, generator=g, device=DEV), 1)
    tokens = torch.randint(0, V, (M,), generator=g, device=DEV).int()
    uniforms = torch.rand(M, generator=g, device=DEV)
    src = ints([int(c.table[0, 0]), int(c.table[1, 1])])
    dst = ints([int(x) for x in c.unused[:2]])
    rows, ws = c.q.clone(), (B.alloc_window_attention_workspace(3, 8, 2, 64, 8, 2000), B.alloc_tree_attention_workspace(3, 8, 2, 64, 8, 2000))
    caches = [c.k, c.v, c.ks, c.vs]
    kept = [x.clone() for x in caches]

    def run():
        a = B.muxq_window_attention(rows, c.k, c.v, c.table, starts, lengths, 8, 2000, window=500, sinks=4, workspace=ws[0], **c.scales())
        b = B.muxq_tree_attention(rows, c.k, c.v, c.table, starts, lengths, parents, 8, 2000, workspace=ws[1], **c.scales())
        v = B.muxq_verify_tree(target, tokens, starts, parents, 8, uniforms=uniforms)
        w = B.muxq_verify_tree(target, tokens, starts, parents, 8)
        B.muxq_kv_compact(v[0], v[1], starts, lengths, c.table, c.k, c.v, 8, **c.scales())
        B.muxq_kv_copy(src, dst, c.k, c.v, **c.scales())
        return [a, b, *v, *w]

    def back():
        for x, y in zip(caches, kept):
            x.copy_(y)
    run()
    torch.cuda.synchronize()
    back()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        outs = run()
    for i in range(4):
        rows.copy_(torch.randn(rows.shape, generator=g, device=DEV).half())
        uniforms.copy_(torch.rand(M, generator=g, device=DEV) * (0.01 if i % 2 else 1.0))
        back()
        want = [x.clone() for x in run()]
        after = [x.nan_to_num(7.0) if x.is_floating_point() else x.clone() for x in caches]
        back()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(outs, want):
            assert torch.equal(x, y)
        for x, y in zip(caches, after):
            assert torch.equal(x.nan_to_num(7.0) if x.is_floating_point() else x, y)


def test_offsets_beyond_32_bits():
    """Pages far apart: 3 pages of a cache that spans 6 GB, its strides given by a view."""
    say("[case] offsets beyond 32 bits")
    heads, page, d, far = 2, 16, 64, 1 << 30
    flat = torch.empty(2 * far + 2 * heads * page * d, dtype=torch.float16, device=DEV)
    views = [flat.as_strided((3, heads, page, d), (far, page * d, d, 1), o) for o in (0, heads * page * d)]
    g = gen(3)
    for v in views:
        v.copy_(normal(g, 3, heads, page, d))
    k, v = views
    q = normal(g, 40, 4, d)
    table = ints([[2, 0, 1]])
    got = B.muxq_window_attention(q, k, v, table, ints([0, 40]), ints([45]), 40, 48)
    want = B.muxq_window_attention(q, k.contiguous(), v.contiguous(), table, ints([0, 40]), ints([45]), 40, 48)
    assert torch.equal(got, want)
    before = [x[2].clone() for x in views]
    B.muxq_kv_copy(ints([2]), ints([1]), k, v)
    assert torch.equal(k[1], before[0]) and torch.equal(v[1], before[1])
    B.muxq_kv_compact(ints([0, 39] + [-1] * 38), ints([2]), ints([0, 40]), ints([45]), table, k, v, 64)
    assert torch.equal(k[2, :, 6], k[1, :, 12]) and torch.equal(v[2, :, 6], v[1, :, 12])
    # rows of the probabilities beyond 2^32 bytes
    V, M = 1 << 20, 1100
    target = torch.zeros(M, V, device=DEV)
    target[:, 5] = 1.0
    target[M - 1, 5], target[M - 1, V - 1] = 0.0, 1.0
    starts, parents = ints([0, M - 2, M]), ints([-1] * (M - 2) + [-1, 0])
    for u in (torch.full((M,), 0.5, device=DEV), None):
        path, counts, said = B.muxq_verify_tree(target, ints([5] * M), starts, parents, 64, uniforms=u)
        assert counts.tolist() == [0, 2] and said.tolist() == [-1, V - 1] and path[M - 2:].tolist() == [0, 1]


def test_verification_at_its_edges():
    say("[case] verification at its edges")
    V = 2000
    one = torch.zeros(V, device=DEV)
    one[3], one[7] = 0.25, 0.75

    def ask(rows, tokens, parents, uniforms, draft=None, starts=None):
        M = len(tokens)
        got = B.muxq_verify_tree(torch.stack(rows), ints(tokens), ints(starts or [0, M]), ints(parents), 64, draft=draft,
                                 uniforms=None if uniforms is None else torch.tensor(uniforms, device=DEV))
        return [x.tolist() for x in got]
    top = 1.0 - 2.0 ** -24
    # borders of the running sum: u * sum < 0.25 is token 3, 0.25 itself is not
    assert ask([one], [0], [-1], [0.25])[2] == [7] and ask([one], [0], [-1], [0.25 - 2.0 ** -26])[2] == [3]
    assert ask([one], [0], [-1], [0.0])[2] == [3] and ask([one], [0], [-1], [top])[2] == [7]
    assert ask([one], [0], [-1], [1.5])[2] == [7]                                # u beyond its range: the last one
    # a token outside the vocabulary, or with no probability, does not stand; parents that are not in front mark roots of nothing
    assert ask([one] * 4, [0, -1, V, 9], [-1, 0, 0, 0], [0.0] * 4) == [[0, -1, -1, -1], [1], [3]]
    assert ask([one] * 3, [0, 7, 7], [-1, 5, 2], [0.0] * 3)[1] == [1]
    # given tokens that are rejected are not what comes next
    assert ask([one] * 2, [0, 7], [-1, 0], [0.9, 0.8])[2] == [3]
    assert ask([one] * 3, [0, 7, 3], [-1, 0, 0], [0.9, 0.8, top]) == [[0, 2, -1], [2], [7]]
    # nothing left: the target itself
    draft = one.repeat(3, 1)
    assert ask([one * 0.5] * 3, [0, 7, 3], [-1, 0, 0], [0.1, 0.9, 0.9], draft) == [[0, -1, -1], [1], [3]]
    # no probabilities at all; NaN stays in its bounds
    assert ask([one * 0], [0], [-1], [0.5])[2] == [-1]
    assert -1 <= ask([one * math.nan], [0], [-1], [0.5])[2][0] < V
    # greedy: the lowest of equal ones, NaN below everything
    tie = torch.full((V,), -math.inf, device=DEV)
    assert ask([tie], [0], [-1], None)[2] == [0]
    tie[11] = tie[1500] = 2.0
    tie[3] = math.nan
    assert ask([tie] * 3, [0, 1500, 11], [-1, 0, 0], None) == [[0, 2, -1], [2], [11]]
    # more rows than the bound, and an empty sequence
    got = B.muxq_verify_tree(one.repeat(6, 1), ints([7] * 6), ints([0, 0, 4, 6]), ints([-1, 0, 1, 2, -1, 0]), 3, uniforms=torch.zeros(6, device=DEV))
    assert [x.tolist() for x in got] == [[-1, -1, -1, -1, 0, 1], [0, 0, 2], [-1, -1, 3]]


def test_strided_probabilities():
    say("[case] strided probabilities")
    g, V = gen(1), 1003
    wide = torch.softmax(torch.randn(9, 1100, generator=g, device=DEV), 1)
    target, draft = wide[:, 2:2 + V], torch.softmax(torch.randn(9, V + 1, generator=g, device=DEV), 1)[:, :V]
    tokens = torch.randint(0, V, (9,), generator=g, device=DEV).int()
    parents, u = random_tree(9, 3, "star"), torch.rand(9, generator=g, device=DEV)
    got = B.muxq_verify_tree(target, tokens, ints([0, 9]), ints(parents), 9, draft=draft, uniforms=u)
    assert [x.tolist() for x in got] == list(verify64(target, draft, tokens.tolist(), parents, u.tolist(), [0, 9]))
