"""Shared by the tests of the operators between the projections: paged caches and the same operators in 64 bits."""
import math

import torch

from paper_2604_04701_amd import binding as B

DEV = "cuda"
U16 = 2.0 ** -11          # fp16: half a unit in the last place, relative
TINY16 = 2.0 ** -25       # ... and where values are subnormal, absolute
U32 = 2.0 ** -24          # binary32


def say(msg):
    print(msg, flush=True)


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def normal(g, *shape, dtype=torch.float16):
    return torch.randn(*shape, generator=g, device=DEV, dtype=torch.float32).to(dtype)


def make_cache(g, n_pages, heads, page, d, bits, layout="heads"):
    """k, v [pages, heads, page, d] and scales, all filled."""
    shape = (n_pages, page, heads, d) if layout == "tokens" else (n_pages, heads, page, d)
    out = []
    for _ in "kv":
        c = normal(g, *shape) if bits == 16 else torch.randint(-127, 128, shape, generator=g, device=DEV, dtype=torch.int32).to(torch.int8)
        out.append(c.transpose(1, 2) if layout == "tokens" else c)
    if bits == 16:
        return *out, None, None
    return *out, *(0.002 + 0.03 * torch.rand(n_pages, heads, page, generator=g, device=DEV) for _ in "kv")


def make_table(g, lengths, page, n_pages, width=None, unused=0):
    """A block table of pages drawn without repeats; entries past a sequence's pages are `unused`."""
    need = [-(-max(n, 0) // page) for n in lengths]
    assert sum(need) <= n_pages
    order = torch.randperm(n_pages, generator=g, device=DEV).tolist()
    table = torch.full((len(lengths), width or max(max(need), 1)), unused, dtype=torch.int32)
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
        at += n
    return table.to(DEV), order[at:]


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def attend64(q, k, v, ks, vs, table, lengths, scale):
    """The attention in 64 bits, and the bound of what binary32 sums and one rounding to fp16 may be off."""
    S, H, d = q.shape
    n_pages, heads, page, _ = k.shape
    out = torch.zeros(S, H, d, dtype=torch.float64, device=DEV)
    tol = torch.zeros_like(out)
    for s, n in enumerate(lengths):
        n = max(0, min(n, table.shape[1] * page))
        if n == 0:
            continue
        pages = table[s, :-(-n // page)].long()
        kept = ((pages >= 0) & (pages < n_pages)).repeat_interleave(page)[:n]
        pages = pages.clamp(0, n_pages - 1)
        if not kept.any():
            continue
        for h in range(heads):
            kk, vv = (x[pages, h].double().reshape(-1, d)[:n][kept] for x in (k, v))
            if ks is not None:
                kk = kk * ks[pages, h].double().reshape(-1)[:n][kept, None]
                vv = vv * vs[pages, h].double().reshape(-1)[:n][kept, None]
            qq = q[s, h * (H // heads):(h + 1) * (H // heads)].double()
            p = torch.softmax(qq @ kk.t() * scale, 1)
            o = p @ vv
            # a score is d products summed in binary32; exp's argument and value add a few units each
            off = abs(scale) * (d + 8) * U32 * (qq.abs() @ kk.abs().t()).amax(1, keepdim=True) + 2.0 ** -16
            hh = slice(h * (H // heads), (h + 1) * (H // heads))
            out[s, hh] = o
            tol[s, hh] = U16 * o.abs() + TINY16 + 3 * off * (p @ vv.abs())
    return out, tol


def check(got, want, tol, what):
    assert torch.isfinite(got.double()).all(), f"{what}: not finite"
    over = ((got.double() - want).abs() - tol)
    worst = over.max().item() if over.numel() else 0.0
    assert worst <= 0.0, f"{what}: {worst:.3g} beyond its bound, largest difference {(got.double() - want).abs().max().item():.3g}"


def rotate64(x, cos_sin, positions, interleaved):
    """x [M, heads, d] float64 with its first rot dimensions turned; positions within the table."""
    rot = cos_sin.shape[1]
    c, s = (t.double()[:, None] for t in cos_sin[positions.long()].split(rot // 2, 1))
    y = x.clone()
    i, j = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    y[..., i] = x[..., i] * c - x[..., j] * s
    y[..., j] = x[..., j] * c + x[..., i] * s
    return y


def lora64(X, A, Bm, scales, starts, adapters, Y):
    """Adapters in 64 bits, and the bound: K products and r products summed in binary32, one rounding to fp16."""
    out, slack = Y.double(), torch.zeros_like(Y, dtype=torch.float64)
    K, n = X.shape[1], A.shape[0]
    for a, b, i in zip(starts, starts[1:], adapters):
        if 0 <= i < n and b > a:
            x, aa, bb, sc = X[a:b].double(), A[i].double(), Bm[i].double(), abs(scales[i].double())
            h = x @ aa.t()
            out[a:b] += scales[i].double() * (h @ bb.t())
            off = (K + 8) * U32 * (x.abs() @ aa.abs().t()) + 2.0 ** -19 * h.abs().amax(1, keepdim=True)
            slack[a:b] = 2 * sc * (off @ bb.abs().t())
    return out, U16 * out.abs() + TINY16 + 2 * U32 * Y.double().abs() + slack


def norm64(x, w, b, kind, eps):
    """The norm of rows in 64 bits, and how much a relative change of the row's largest element moves it."""
    mean = x.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(x[:, :1])
    z = x - mean
    inv = 1.0 / torch.sqrt((z * z).mean(1, keepdim=True) + eps)
    y = z * inv * w.double() + (0.0 if b is None else b.double())
    return y, inv * x.abs().amax(1, keepdim=True) * w.double().abs()


def slots_of(table_row, positions, page):
    return [int(table_row[p // page]) * page + p % page for p in positions]


__all__ = [n for n in dir() if not n.startswith("__")]
