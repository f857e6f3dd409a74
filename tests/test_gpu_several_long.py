"""Attention of several new tokens where a workgroup goes through more tiles of tokens than it has pages at hand for, or remembers infinite values
of; and batches of very unequal numbers of new tokens."""
import math

import pytest
import torch

from block_common import check, say
from paper_2604_04701_amd import binding as B
from several_common import *          # noqa: F401,F403
from several_common import Case, below, causal, random_tree, rows64

pytestmark = pytest.mark.gpu

LONG = 4480          # tokens of the last sequence: 35 tiles of 128, the widest there are

# new tokens and lengths of each sequence, heads: so many workgroups that none of them is cut along the tokens
FORMS = {"rows32_of_64": ([2] * 65, [5] * 64 + [LONG], 8, 8, 64), "rows64_of_64": ([40] * 49, [40] * 48 + [LONG], 16, 16, 64),
         "rows128_of_64": ([70] * 64, [70] * 63 + [LONG], 16, 16, 64), "rows32_of_128": ([2] * 64, [9] * 63 + [LONG], 16, 16, 128),
         "rows64_of_128": ([40] * 33, [40] * 32 + [LONG], 16, 16, 128), "rows128_of_128": ([130] * 40, [130] * 39 + [LONG], 32, 16, 128),
         "rows128_of_80": ([130] * 40, [130] * 39 + [LONG], 32, 16, 80), "rows128_of_256": ([40] * 64, [40] * 63 + [LONG], 8, 8, 256),
         "trees64_of_64": ([40] * 33, [40] * 32 + [LONG], 16, 16, 64), "trees128_of_128": ([64] * 33, [64] * 32 + [LONG], 32, 16, 128)}


def call(c, tree):
    starts, lengths = c.device()
    if tree:
        parents = ints(sum((random_tree(n, n) for n in c.new), []))
        return B.muxq_tree_attention(c.q, c.k, c.v, c.table, starts, lengths, parents, max(c.new), max(c.lengths), **c.scales())
    return B.muxq_window_attention(c.q, c.k, c.v, c.table, starts, lengths, max(c.new), max(c.lengths), **c.scales())


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("kind", ["plain", "missing", "infinite"])
@pytest.mark.parametrize("name", FORMS)
def test_many_tiles_of_one_workgroup(monkeypatch, name, kind, bits):
    new, lengths, H, heads, d = FORMS[name]
    tree = name.startswith("trees")
    say(f"[case] many tiles {name} {kind} bits={bits}")
    c = Case(21, new, lengths, H, heads, d, 16, bits)
    s, n, group = len(new) - 1, new[-1], H // heads
    if kind == "missing":                # in every 32 tiles of 32, 64 or 128 tokens
        for t in (500, 1030, 2100, 3000, 4100, 4200):
            c.table[s, t // c.page] = [-1, c.n_pages][t % 2]
    if kind == "infinite":
        tokens = list(range(10, LONG - n, 64))
        pages, at = c.table[s, torch.tensor(tokens, device=DEV) // c.page].long(), torch.tensor(tokens, device=DEV) % c.page
        # (values are finite for the formula; the kernel sees them infinite)
        if bits == 16:
            c.v[pages, 1, at, 7] = 0
            c.v[pages, 1, at, 9] = 0
        else:
            c.v[pages, 1, at] = 0
    # (a workspace that is asked for would say that the work is cut into pieces)
    for form in ("window", "tree"):
        monkeypatch.setattr(B, f"alloc_{form}_attention_workspace", lambda *_: pytest.fail("in pieces: fewer than 33 tiles a workgroup"))
    want, tol = rows64(c.q, c.k, c.v, c.ks, c.vs, c.table, c.starts, lengths,
                       lambda i, m, length: below(random_tree(m, m), length) if tree else causal(m, length, 0, 0), d ** -0.5)
    if kind != "infinite":
        check(call(c, tree), want, tol, name)
        return
    if bits == 16:
        c.v[pages, 1, at, 7] = math.inf
        c.v[pages, 1, at, 9] = math.inf
        c.v[pages[-1], 1, at[-1], 9] = -math.inf
    else:
        c.v[pages, 1, at] = 3
        c.vs[pages, 1, at] = math.inf
    got = call(c, tree).double()
    a = c.starts[s]
    mine = got[a:, group:2 * group]
    for e in (7, 9) if bits == 16 else range(d):
        assert (torch.isnan(mine[..., e]) if e == 9 and bits == 16 else mine[..., e] == math.inf).all(), e
        mine[..., e] = want[a:, group:2 * group, e]
    check(got, want, tol, name)


# a chunk of a prompt beside single tokens, as a server's step has them
MIXED = {"12x64": (12, 12, 64), "32of8x128": (32, 8, 128), "4of1x256": (4, 1, 256)}


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("win,sinks", [(0, 0), (300, 4)])
@pytest.mark.parametrize("name", MIXED)
def test_a_chunk_beside_single_tokens(name, win, sinks, bits):
    H, heads, d = MIXED[name]
    say(f"[case] mixed batch {name} window={win} sinks={sinks} bits={bits}")
    singles = [1 + 37 * i * i % 4001 for i in range(40)]
    c = Case(22, [1] * 11 + [512] + [1] * 29 + [3], singles[:11] + [1300] + singles[11:] + [700], H, heads, d, 16, bits)
    starts, lengths = c.device()
    got = B.muxq_window_attention(c.q, c.k, c.v, c.table, starts, lengths, 512, max(c.lengths), window=win, sinks=sinks, **c.scales())
    want, tol = c.exact(lambda i, m, length: causal(m, length, win, sinks))
    check(got, want, tol, name)


@pytest.mark.parametrize("bits", [16, 8])
def test_a_dimension_that_is_infinite_everywhere(bits):
    """As a model has it that passes fp16 in a channel: right, and in milliseconds (each row's look at each token from memory took 600)."""
    say(f"[case] a dimension of infinite values, bits={bits}")
    n = 4096
    c = Case(23, [n], [n], 32, 8, 128, 16, bits)
    if bits == 16:
        c.v[..., 3] = 0
        want = call(c, False)
        c.v[..., 3] = math.inf
        c.v[c.table[0, 100].long(), 2, 5, 3] = -math.inf          # token 1605: NaN from there on, in its heads
        want[..., 3] = math.inf
        want[1605:, 8:12, 3] = math.nan
    else:
        want = torch.full_like(c.q, math.inf)
        want[..., ::2] = -math.inf
        c.v[..., ::2], c.v[..., 1::2] = -1, 1
        c.vs[:] = math.inf
    best = math.inf
    for _ in range(3):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        got = call(c, False)
        b.record()
        torch.cuda.synchronize()
        best = min(best, a.elapsed_time(b))
    assert torch.equal(got.nan_to_num(7.0, 8.0, 9.0), want.nan_to_num(7.0, 8.0, 9.0))
    assert best < 150.0, f"{best:.0f} ms"


def test_verification_of_more_rows_than_a_grid_holds():
    """Greedy, where the rows of all nodes are looked at at once as long as a launch holds them."""
    M = (1 << 22) + 5
    say(f"[case] verify {M} rows")
    target = torch.rand(M, 2, generator=gen(1), device=DEV)
    tokens, parents = torch.zeros(M, dtype=torch.int32, device=DEV), torch.full((M,), -1, dtype=torch.int32, device=DEV)
    parents[M - 2:] = ints([0, 1])
    for V in (1, 2):
        rows = target[:, :V]
        tokens[M - 2:] = rows[M - 3:M - 1].argmax(1).int()          # what the target says after the node above
        left = torch.full((M,), 7, dtype=torch.int32, device=DEV)
        path, counts, said = B.muxq_verify_tree(rows, tokens, ints([3, 4, M - 3, M]), parents, 64, path=left)
        assert counts.tolist() == [1, 0, 3] and said.tolist() == [int(rows[3].argmax()), -1, int(rows[M - 1].argmax())]
        assert path[3] == 0 and (path[:3] == 7).all() and (path[4:M - 3] == -1).all() and path[M - 3:].tolist() == [0, 1, 2]


def test_copies_of_more_pairs_than_a_launch_takes():
    n = (1 << 22) + 9                     # 2^22 pairs of pages of two parts each are one launch
    say(f"[case] copy {n} pairs")
    k, v = (normal(gen(i), 12, 1, 8, 16) for i in (1, 2))
    src, dst = (torch.full((n,), -1, dtype=torch.int32, device=DEV) for _ in range(2))
    at = torch.tensor([0, (1 << 22) - 1, 1 << 22, n - 1], device=DEV)
    src[at], dst[at] = ints([1, 2, 3, 4]), ints([5, 6, 7, 8])
    want = [x.clone() for x in (k, v)]
    for x in want:
        x[5:9] = x[1:5]
    B.muxq_kv_copy(src, dst, k, v)
    assert torch.equal(k, want[0]) and torch.equal(v, want[1])


@pytest.mark.parametrize("new", [1, 2])
def test_as_many_sequences_as_there_may_be(new):
    """65535 of them, a page each: attention, verification and compaction."""
    S, d, page = 65535, 16, 8
    say(f"[case] {S} sequences of {new} rows")
    g = gen(new)
    k, v = (normal(g, S, 1, page, d) for _ in "kv")
    table = torch.randperm(S, generator=g, device=DEV).int().view(S, 1)
    lengths = torch.randint(new, page + 1, (S,), generator=g, device=DEV).int()
    starts = torch.arange(0, S * new + 1, new, device=DEV).int()
    q = normal(g, S * new, 1, d)
    parents = torch.arange(new, device=DEV).int().sub(1).repeat(S)
    for tree in (False, True):
        if tree:
            got = B.muxq_tree_attention(q, k, v, table, starts, lengths, parents, new, page)
        else:
            got = B.muxq_window_attention(q, k, v, table, starts, lengths, new, page)
        kk, vv = (x[table[:, 0].long(), 0].double() for x in (k, v))
        score = (q.double().view(S, new, 1, d) * kk[:, None]).sum(3) / 4
        last = lengths[:, None] - new + torch.arange(new, device=DEV)
        score = score.masked_fill(torch.arange(page, device=DEV) > last[..., None], -math.inf)
        p = torch.softmax(score, 2)
        want, mass = ((p[..., None] * x[:, None]).sum(2) for x in (vv, vv.abs()))
        # one rounding of the output, one of the weights, and of sums of 16 products of some 20 in all
        tol = TINY16 + 2.0 ** -11 * (want.abs() + 1.01 * mass) + 3 * 2.0 ** -16 * mass
        check(got.view(S, new, d), want, tol, "attention")
    V = 5
    target = torch.softmax(torch.randn(S * new, V, generator=g, device=DEV), 1)
    tokens = torch.randint(0, V, (S * new,), generator=g, device=DEV).int()
    path, counts, said = B.muxq_verify_tree(target, tokens, starts, parents, new)
    best = target.argmax(1).view(S, new)
    stands = (tokens.view(S, new)[:, -1] == best[:, 0]) & (new == 2)
    assert torch.equal(counts, 1 + stands.int())
    assert torch.equal(said, torch.where(stands, best[:, -1], best[:, 0]).int())
    assert (path.view(S, new)[:, 0] == 0).all()
    # the last node to the front
    at = torch.full((S * new,), new - 1, dtype=torch.int32, device=DEV)
    kept = [x[table[:, 0].long(), 0, lengths.long() - 1] for x in (k, v)]
    B.muxq_kv_compact(at, torch.ones(S, dtype=torch.int32, device=DEV), starts, lengths, table, k, v, new)
    for x, y in zip((k, v), kept):
        assert torch.equal(x[table[:, 0].long(), 0, lengths.long() - new], y)
