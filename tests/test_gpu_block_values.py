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
