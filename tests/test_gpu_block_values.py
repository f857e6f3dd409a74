"""Infinities and NaN in the operators between the projections: what the formulas give in 64 bits, on the CPU, place by place."""
import math

import pytest
import torch

from block_common import *

pytestmark = pytest.mark.gpu

INF = math.inf


def check_places(got, want, tol, what):
    """Infinities and NaN where they belong, the rest within its bound."""
    got = got.double().cpu()
    for kind, g, w in (("NaN", got.isnan(), want.isnan()), ("infinity", got == INF, want == INF), ("-infinity", got == -INF, want == -INF)):
        wrong = (g != w).nonzero().tolist()
        assert not wrong, f"{what}: {kind} at {(g & ~w).sum().item()} places where there is none, none at {(w & ~g).sum().item()}, first {wrong[0]}"
    there = want.isfinite()
    check(got[there], want[there], tol[there], what)


# ---- adapters --------------------------------------------------------------------------------------


@pytest.mark.parametrize("M,K,N,r,starts", [
    (9, 64, 40, 8, [0, 1, 2, 3, 4, 9]),                 # single tokens
    (70, 264, 200, 40, [0, 30, 33, 50, 64, 70]),        # tiles of 16 rows
    (40, 1024, 136, 64, [0, 8, 16, 24, 32, 40]),        # two launches
    (2000, 800, 72, 16, [0, 1000, 1500, 1501, 1502, 2000]),          # tiles of 32 rows
    (700, 2304, 136, 32, [0, 300, 301, 302, 400, 700])])             # the same in two launches
def test_lora_infinities(M, K, N, r, starts):
    g = torch.Generator()
    g.manual_seed(M)
    X, Y = torch.randn(M, K, generator=g).half(), torch.randn(M, N, generator=g).half()
    A = (torch.randn(3, r, K, generator=g) / math.sqrt(K)).half()
    Bm = (torch.randn(3, N, r, generator=g) / math.sqrt(r)).half()
    scales = torch.tensor([0.75, -1.5, 1.0])
    adapters = [0, 1, -1, 2, 0]
    # a channel of A of one sign, and of B columns of one sign, of the other, and mixed ones
    A[0, :, 3] = A[0, :, 3].abs() + 0.1
    A[1, :, 3] = A[1, :, 3].abs() + 0.1
    for i in (0, 1):
        Bm[i, 0::3], Bm[i, 1::3] = Bm[i, 0::3].abs() + 1e-3, -Bm[i, 1::3].abs() - 1e-3
    Bm[0, 6, r - 1] = 0.0                        # infinity times zero
    X[starts[0], 3], X[starts[1], 3], X[starts[2], 3] = INF, -INF, INF
    X[starts[5] - 1, 3], X[starts[5] - 2, 3] = -INF, math.nan
    X[starts[3]] = 0.0
    A[2, 1, 7] = INF                             # times zero in that row
    Bm[1, 9, 2], Bm[1, 10, 3] = INF, -INF        # in columns of their own: H decides the sign
    Y[starts[4], 5], Y[starts[4], 6] = INF, math.nan
    want, slack = Y.double(), torch.zeros(M, N, dtype=torch.float64)
    for a, b, i in zip(starts, starts[1:], adapters):
        if i < 0:
            continue
        x, aa, bb = X[a:b].double(), A[i].double(), Bm[i].double()
        h = x @ aa.t()
        want[a:b] += scales[i].double() * (h @ bb.t())
        # the bound of lora64: K and r products summed in binary32, H in parts of 22 bits of the row's largest
        off = (K + 8) * U32 * (x.abs() @ aa.abs().t()) + 2.0 ** -19 * h.abs().amax(1, keepdim=True)
        slack[a:b] = 2 * scales[i].double().abs() * (off @ bb.abs().t())
    assert want.isnan().any() and (want == INF).any() and (want == -INF).any() and want.isfinite().any()
    tol = U16 * want.abs() + TINY16 + 2 * U32 * Y.double().abs() + slack
    say(f"[lora] infinities, M={M} K={K} N={N} r={r}")
    got = B.muxq_lora(*(t.to(DEV) for t in (X, A, Bm, scales)), ints(starts), ints(adapters), Y.to(DEV))
    torch.cuda.synchronize()
    check_places(got, want, tol, "adapters")


# ---- attention of one new token ----------------------------------------------------------------


def _exact_places(q, k, v, ks, vs, table, lengths, scale):
    """attend64 on the CPU, with a bound that leaves out what is not finite."""
    S, H, d = q.shape
    heads, page = k.shape[1], k.shape[2]
    want, tol = torch.zeros(S, H, d, dtype=torch.float64), torch.zeros(S, H, d, dtype=torch.float64)
    for s, n in enumerate(lengths):
        pages = table[s, :-(-n // page)].long()
        for h in range(heads if n else 0):
            kk, vv = (x[pages, h].double().reshape(-1, d)[:n] for x in (k, v))
            if ks is not None:
                kk, vv = kk * ks[pages, h].double().reshape(-1)[:n, None], vv * vs[pages, h].double().reshape(-1)[:n, None]
            at = slice(h * (H // heads), (h + 1) * (H // heads))
            qq = q[s, at].double()
            p = torch.softmax(qq @ kk.t() * scale, 1)
            want[s, at] = p @ vv
            size_k, size_v = (torch.where(x.isfinite(), x.abs(), 0.0) for x in (kk, vv))
            off = scale * (d + 8) * U32 * (qq.abs() @ size_k.t()).amax(1, keepdim=True) + 2.0 ** -16
            tol[s, at] = U16 * want[s, at].abs() + TINY16 + 3 * off * (torch.nan_to_num(p) @ size_v)
    return want, tol


def _loose_cache(seed, lengths, H, heads, d, bits):
    """A cache on the CPU, a table, queries, and set(s, t, ...): changes token t of sequence s in all heads."""
    g = torch.Generator()
    g.manual_seed(seed)
    page = 16
    need = [-(-n // page) for n in lengths]
    order = torch.randperm(sum(need) + 1, generator=g).tolist()
    table = torch.zeros(len(lengths), max(need), dtype=torch.int32)
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
        at += n
    shape = (len(order), heads, page, d)
    k, v = (torch.randn(shape, generator=g).half() if bits == 16 else torch.randint(-127, 128, shape, generator=g).to(torch.int8) for _ in "kv")
    ks, vs = (0.005 + 0.01 * torch.rand(shape[:3], generator=g) for _ in "kv") if bits == 8 else (None, None)
    q = torch.randn(len(lengths), H, d, generator=g).half()
    q[:, :, 0] = q[:, :, 0].abs() + 0.5
    q[:, 1::2, 0] *= -1                          # what is -infinity to one query is infinity to its neighbour

    def place(s, t):
        return int(table[s, t // page]), slice(None), t % page
    return q, k, v, ks, vs, table, place


def _loose_check(q, k, v, ks, vs, table, lengths, what):
    scale = q.shape[2] ** -0.5
    want, tol = _exact_places(q, k, v, ks, vs, table, lengths, scale)
    say(f"[attend] {what}, S={len(lengths)} H={q.shape[1]}/{k.shape[1]} d={q.shape[2]} {k.dtype} longest={max(lengths)}")
    on = [None if x is None else x.to(DEV) for x in (q, k, v, table, ks, vs)]
    got = B.muxq_paged_attention(*on[:4], ints(lengths), max(lengths), scale=scale, k_scale=on[4], v_scale=on[5])
    torch.cuda.synchronize()
    check_places(got, want, tol, what)
    B.muxq_paged_attention(*on[:4], ints(lengths), max(lengths), scale=scale, k_scale=on[4], v_scale=on[5], out=on[0])
    torch.cuda.synchronize()
    assert torch.equal(on[0].view(torch.int16), got.view(torch.int16)), "in place"
    return want


ROUTES = [[37, 20, 9, 64, 100, 128], [300, 257, 64, 700, 33, 512], [5000, 2700, 2600, 4000, 4097, 2900]]       # 4 waves, 8 waves, shares


@pytest.mark.parametrize("lengths", ROUTES)
@pytest.mark.parametrize("H,heads,d", [(4, 2, 64), (8, 1, 80), (3, 3, 128), (4, 2, 256)])
def test_attention_infinities_of_fp16(lengths, H, heads, d):
    q, k, v, ks, vs, table, place = _loose_cache(d, lengths, H, heads, d, 16)

    def far(s, t):                               # a score of about -60: a weight that is 0 in 16 bits
        group = q[s].view(heads, H // heads, d).float().mean(1)
        k[place(s, t)] = (-60.0 * d ** 0.5 * group / group.square().sum(1, keepdim=True)).half()
    n = lengths[0]
    for t, x in ((1, INF), (n // 2, -INF)):                       # in full weight, alone, together, and NaN
        v[place(0, t)][..., 3 if t == 1 else 4] = x
        v[place(0, t)][..., 5] = x
    v[place(0, n - 1)][..., 6] = math.nan
    v[place(0, n - 2)][..., 7] = INF
    for t, e in ((0, 2), (lengths[1] - 1, 9)):                    # beside tokens that outweigh them by far, before and behind
        far(1, t)
        v[place(1, t)][..., e] = -INF
    k[place(2, 5)][..., 0] = -INF                                 # a score of -infinity (or infinity): what stands there counts nothing, unless
    v[place(2, 5)][..., 8] = INF                                  # it is infinite
    k[place(3, lengths[3] - 1)][..., 0] = math.nan
    far(5, 0)
    v[place(5, 0)][..., 1] = INF
    v[place(5, lengths[5] // 2)][..., d - 1] = INF
    want = _loose_check(q, k, v, ks, vs, table, lengths, "infinities")
    assert want.isnan().any() and (want == INF).any() and (want == -INF).any() and want.isfinite().any()


@pytest.mark.parametrize("lengths", ROUTES)
@pytest.mark.parametrize("H,heads,d", [(4, 2, 64), (8, 1, 80), (3, 3, 128), (4, 2, 256)])
def test_attention_infinite_scales(lengths, H, heads, d):
    q, k, v, ks, vs, table, place = _loose_cache(d, lengths, H, heads, d, 8)

    def far(s, t):
        group = q[s].view(heads, H // heads, d).float().mean(1)
        k[place(s, t)] = (-group / group.abs().amax(1, keepdim=True) * 127).round().to(torch.int8)
        ks[place(s, t)] = 60.0 * d ** 0.5 * group.abs().amax(1) / 127 / group.square().sum(1)
    v[place(0, 1)][..., 3:5] = 0                                  # infinity times a code of zero
    vs[place(0, 1)] = INF
    far(1, 0)
    far(1, lengths[1] - 1)
    vs[place(1, 0)] = INF
    ks[place(3, lengths[3] - 1)] = math.nan
    vs[place(4, lengths[4] // 2)] = math.nan
    far(5, lengths[5] // 2)
    vs[place(5, lengths[5] // 2)] = INF
    want = _loose_check(q, k, v, ks, vs, table, lengths, "infinite scales")
    assert want.isnan().any() and (want == INF).any() and (want == -INF).any() and want.isfinite().any()


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("lengths", ROUTES)
@pytest.mark.parametrize("H,heads,d", [(4, 2, 64), (8, 1, 80), (3, 3, 128), (4, 2, 256)])
def test_attention_scores_of_minus_infinity(lengths, H, heads, d, bits):
    q, k, v, ks, vs, table, place = _loose_cache(d, lengths, H, heads, d, bits)
    q[:] = q.abs() + 0.01
    page = k.shape[2]

    def shut(s, tokens):                         # a score of -infinity to every query
        for t in tokens:
            if bits == 16:
                k[place(s, t)][..., 0] = -INF
            else:
                k[place(s, t)] = -(k[place(s, t)].int().abs().clamp_min(1)).to(torch.int8)
                ks[place(s, t)] = INF
    shut(0, range(lengths[0]))                   # all: 0 / 0
    shut(1, range(lengths[1] // 2))              # a half, either one: no weight
    shut(2, range(lengths[2] // 2, lengths[2]))
    shut(3, [t for t in range(lengths[3]) if t != lengths[3] - 3])           # all but one
    shut(4, range(0, lengths[4], 2))
    shut(5, range(lengths[5]))
    last = lengths[5] - 1
    if bits == 16:
        k[place(5, last)][..., 0] = 0.5          # one is left at the very end
    else:
        ks[place(5, last)] = 0.01
    want = _loose_check(q, k, v, ks, vs, table, lengths, "scores of -infinity")
    assert want[0].isnan().all() and want[1:].isfinite().all()
    # pages outside the cache leave their tokens out: of the first sequence all of them, zeros; of the second all but shut ones, 0 / 0
    table = table.clone()
    table[0] = -1
    table[1, -(-(lengths[1] // 2) // page):] = k.shape[0]
    shut(1, range(-(-(lengths[1] // 2) // page) * page))
    on = [None if x is None else x.to(DEV) for x in (q, k, v, table, ks, vs)]
    got = B.muxq_paged_attention(*on[:4], ints(lengths), max(lengths), k_scale=on[4], v_scale=on[5])
    torch.cuda.synchronize()
    assert (got[0] == 0).all() and got[1].isnan().all() and got[2:].isfinite().all()


# ---- one workspace for many calls --------------------------------------------------------------


def test_adapters_share_the_workspace_of_the_largest_batch():
    g = gen(21)
    K, N, r, n = 4096, 264, 32, 3
    M, requests = 1600, 40
    X, Y = normal(g, M, K), normal(g, M, N)
    A, Bm = (normal(g, n, r, K, dtype=torch.float32) / 64).half(), normal(g, n, N, r)
    scales = torch.rand(n, generator=g, device=DEV)
    size = B.alloc_lora_workspace(M, K, N, r, requests).numel()
    room = torch.full((size + 4096,), 0x7f, dtype=torch.uint8, device=DEV)
    for m, q in ((M, requests), (M - 5, 1), (1300, 1), (900, 3), (511, 40), (200, 7), (33, 1), (16, 16), (1, 1)):
        starts = [m * i // q for i in range(q + 1)]
        adapters = [i % n for i in range(q)]
        say(f"[lora] workspace of {M} rows for {m} of {q} requests")
        got = B.muxq_lora(X[:m], A, Bm, scales, ints(starts), ints(adapters), Y[:m], workspace=room[:size])
        torch.cuda.synchronize()
        want, tol = lora64(X[:m], A, Bm, scales, starts, adapters, Y[:m])
        check(got, want, tol, "adapters")
        assert (room[size:] == 0x7f).all()


def test_attention_shares_the_workspace_of_the_largest_batch():
    # with shares, with fewer sequences and longer ones, and calls that need none
    g = gen(22)
    H, heads, d, page, most = 8, 4, 64, 16, 6000
    k, v, ks, vs = make_cache(g, 2000, heads, page, d, 16)
    size = B.attention_workspace_bytes(64, H, heads, d, most)
    assert size > 0
    room = torch.full((size + 4096,), 0x7f, dtype=torch.uint8, device=DEV)
    for lengths in ([500] * 63 + [most], [most, 1, 3000], [1300], [2600, 2400], [100] * 64, [700, 0], [0], [most]):
        table = torch.randint(0, 2000, (len(lengths), max(1, -(-max(lengths) // page))), generator=g, device=DEV).int()     # pages in common
        q = normal(g, len(lengths), H, d)
        say(f"[attend] workspace of 64 x {most} for {len(lengths)} to {max(lengths)}")
        got = B.muxq_paged_attention(q, k, v, table, ints(lengths), max(max(lengths), 1), workspace=room[:size])
        torch.cuda.synchronize()
        want, tol = attend64(q, k, v, None, None, table, lengths, d ** -0.5)
        check(got, want, tol, "attention")
        assert (room[size:] == 0x7f).all()
