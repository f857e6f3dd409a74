"""Rows of several new tokens whose scores are no numbers, beside infinite values: NaN, however the call is divided."""
import math

import pytest
import torch

from block_common import check, say
from paper_2604_04701_amd import binding as B
from several_common import *          # noqa: F401,F403
from several_common import Case, below, causal, random_tree, rows64

pytestmark = pytest.mark.gpu

# every tile of rows, whole and in pieces, and single rows: new tokens and lengths of each sequence, heads
SHAPES = {"rows32_of_64": ([5, 1], [70, 300], 4, 4, 64), "rows32_of_128": ([1, 7], [200, 77], 8, 4, 128), "rows64": ([60, 61], [60, 200], 4, 4, 128),
          "rows128": ([130, 128], [130, 300], 4, 2, 128), "rows128_of_80": ([130] * 12, [130] * 11 + [200], 32, 16, 80),
          "rows64_of_64": ([60, 33] * 26, [60, 133] * 26, 16, 16, 64), "rows128_of_64": ([300] * 12, [300] * 12, 24, 12, 64),
          "heads256": ([40, 3, 40], [40, 90, 90], 2, 1, 256), "pieces32_of_64": ([5, 1, 7], [2000, 300, 3000], 4, 4, 64),
          "pieces32_of_128": ([5, 1, 7], [2000, 300, 3000], 4, 4, 128), "pieces64": ([64, 3, 64], [1500, 64, 1500], 4, 4, 128),
          "pieces128": ([130] * 3, [130, 150, 900], 32, 16, 128), "pieces256": ([40, 40], [1500, 1300], 2, 1, 256),
          "single": ([1, 1, 1], [70, 5, 300], 8, 2, 64), "single80": ([1, 0, 1], [40, 3, 900], 4, 4, 80)}


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("kind,early", [("query", False), ("query", True), ("key", True), ("same", False)])
@pytest.mark.parametrize("name", SHAPES)
def test_scores_that_are_no_numbers_beside_infinite_values(name, early, kind, bits):
    """A row with a NaN in its query, or with a token whose score is NaN or infinite, is NaN, also where it sees an infinite value; the rows
    before it are infinite there, or as they were."""
    new, lengths, H, heads, d = SHAPES[name]
    tree = name in ("rows32_of_128", "rows64", "pieces64")
    say(f"[case] no numbers {name} early={early} {kind} bits={bits} tree={tree}")
    c = Case(12, new, lengths, H, heads, d, 16, bits)
    s, n, length, group = len(new) - 1, new[-1], lengths[-1], H // heads
    a, trees = c.starts[s], [random_tree(m, 3 + m) for m in new]
    starts, at = c.device()

    def seen_of(i, m, most):
        return below(trees[i], most) if tree else causal(m, most, 0, 0)

    def place(t):
        return int(c.table[s, t // c.page]), t % c.page

    def run():
        if tree:
            return B.muxq_tree_attention(c.q, c.k, c.v, c.table, starts, at, ints(sum(trees, [])), max(new), max(lengths), **c.scales())
        return B.muxq_window_attention(c.q, c.k, c.v, c.table, starts, at, max(new), max(lengths), **c.scales())
    # without any of it: what the other rows are
    late, inf_at = length - max(1, n // 4), 0 if early else length - max(1, n // 2)
    if kind == "same":
        late = inf_at
    (p0, i0), (p1, i1) = place(inf_at), place(late)
    c.v[p0, 0, i0] = 0
    c.k[p1, 0, i1] = 0
    want, tol = c.exact(seen_of)
    # (that token's scale counts for the bound where there are codes; its score is 0 in the formula above and in the call)
    sign = torch.where(torch.arange(d, device=DEV) % 3 == 0, 1, -1)
    if bits == 16:
        c.v[p0, 0, i0] = sign * math.inf
    else:
        c.v[p0, 0, i0] = (sign * 5).to(torch.int8)
        c.vs[p0, 0, i0] = math.inf
    broken = torch.zeros(n, dtype=torch.bool)
    seen = seen_of(s, n, length)
    if kind == "query":
        broken[n // 2:] = True
        c.q[a + n // 2:, :group, 1] = math.nan
    elif bits == 16:
        c.q[:, :, 2] = 1.0          # (a score of +infinity where the key is)
        want, tol = rows64(c.q, c.k, torch.where(torch.isinf(c.v), 0.0, c.v), c.ks, c.vs, c.table, c.starts, lengths, seen_of, d ** -0.5)
        c.k[p1, 0, i1, 2] = math.inf if kind == "same" else math.nan
        broken = seen[:, late]
    else:
        c.ks[p1, 0, i1] = math.nan
        broken = seen[:, late]
    got = run().double()
    infinite = seen[:, inf_at] & ~broken
    assert broken.any()
    mine = got[a:, :group]
    assert torch.isnan(mine[broken]).all(), f"{name}: {int((~torch.isnan(mine[broken])).sum())} numbers in rows that are NaN"
    assert (mine[infinite] == sign * math.inf).all(), f"{name}: rows that see an infinite value"
    got[a:, :group][broken | infinite] = want[a:, :group][broken | infinite]
    check(got, want, tol, name)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("what", ["key", "query"])
@pytest.mark.parametrize("name", SHAPES)
def test_infinite_values_with_weights_of_0(name, what, bits):
    """A score of -infinity is a weight of 0, and 0 times an infinite value is NaN; a row that has no other scores is 0 / 0."""
    new, lengths, H, heads, d = SHAPES[name]
    say(f"[case] weights of 0 {name} {what} bits={bits}")
    c = Case(14, new, lengths, H, heads, d, 16, bits)
    s, n, length, group = len(new) - 1, new[-1], lengths[-1], H // heads
    a, t = c.starts[s], length - max(1, n // 2)
    p, i = int(c.table[s, t // c.page]), t % c.page
    c.q[:, :, 2] = 1.0
    spoilt = torch.arange(d, device=DEV) % 3 == 0

    def seen_of(x, m, most):
        seen = causal(m, most, 0, 0)
        if x == s:
            seen[:, t] = False
        return seen
    want, tol = c.exact(lambda x, m, most: causal(m, most, 0, 0))
    without = c.exact(seen_of)
    want[:, :group], tol[:, :group] = without[0][:, :group], without[1][:, :group]         # (only these heads' scores are infinite)
    sees = causal(n, length, 0, 0)[:, t]
    assert sees.any() and length > 1
    c.k[p, 0, i] = 0
    if bits == 16:
        c.k[p, 0, i, 2] = -math.inf
        c.v[p, 0, i] = torch.where(spoilt, math.inf, 1.0).half()
    else:
        c.k[p, 0, i, 2] = -1
        c.ks[p, 0, i] = c.vs[p, 0, i] = math.inf
        spoilt[:] = True
    if what == "query":           # the same of all tokens, for one row
        m = a + int(sees.nonzero()[0])
        used = c.table[s, :-(-length // c.page)].long()
        c.k[used, 0, :, 3] = -1
        c.q[m, :group, 3] = math.inf
    starts, at = c.device()
    got = B.muxq_window_attention(c.q, c.k, c.v, c.table, starts, at, max(new), max(lengths), **c.scales()).double()
    if what == "query":
        assert torch.isnan(got[m, :group]).all()
        return
    mine = got[a:, :group]
    assert torch.isnan(mine[sees][..., spoilt]).all()
    hit = sees.to(DEV)[:, None, None] & spoilt
    got[a:, :group] = torch.where(hit, want[a:, :group], mine)
    check(got, want, tol, name)
