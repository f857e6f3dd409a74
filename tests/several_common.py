"""Shared by the tests of the operators for several new tokens of a sequence: the same operators in 64 bits."""
import math

import torch

from block_common import DEV, TINY16, U16, U32, gen, ints, make_cache, make_table, normal


def causal(n, length, window, sinks):
    """[n, length]: which tokens the last n of a sequence see."""
    p = torch.arange(length - n, length)[:, None]
    t = torch.arange(length)[None]
    seen = t <= p
    if window:
        seen &= (t > p - window) | (t < sinks)
    return seen


def below(parents, length):
    """[n, length]: which tokens the nodes of a tree see, n of them being the last of the sequence."""
    n = len(parents)
    seen = torch.zeros(n, max(length, n), dtype=torch.bool)
    seen[:, :max(length - n, 0)] = True
    for i in range(n):
        x = i
        while x >= 0:
            seen[i, max(length, n) - n + x] = True
            x = parents[x] if parents[x] < x else -1
    return seen[:, max(length, n) - length:] if length < n else seen


def rows64(q, k, v, ks, vs, table, starts, lengths, seen_of, scale):
    """Attention of the rows starts[s]..starts[s + 1] of q over the first lengths[s] tokens of each sequence, seen_of(s, n, length) giving
    which of them each row sees; and the bound of what the arithmetic may be off:
      scores  d products summed in binary32, an argument and a value of the exponential: as for one new token;
      weights one rounding to fp16 (U16 of each), cut to multiples of 2^-32 of the largest (codes: 2^-31 of that and the largest scale);
      the output's rounding."""
    M, H, d = q.shape
    n_pages, heads, page, _ = k.shape
    out = torch.zeros(M, H, d, dtype=torch.float64, device=DEV)
    tol = torch.full_like(out, TINY16)
    group = H // heads
    for s, length in enumerate(lengths):
        a, b = starts[s], starts[s + 1]
        length = max(0, min(length, table.shape[1] * page))
        if a >= b or length == 0:
            continue
        pages = table[s, :-(-length // page)].long()
        kept = ((pages >= 0) & (pages < n_pages)).repeat_interleave(page)[:length]
        pages = pages.clamp(0, n_pages - 1)
        seen = seen_of(s, b - a, length).to(DEV) & kept
        for h in range(heads):
            kk, vv = (x[pages, h].double().reshape(-1, d)[:length] for x in (k, v))
            cut = 2.0 ** -32
            if ks is not None:
                kk = kk * ks[pages, h].double().reshape(-1)[:length, None]
                scales = vs[pages, h].double().reshape(-1)[:length, None]
                vv = vv * scales
            # what no row sees may be anything
            some = seen.any(0)[:, None]
            kk, vv = torch.where(some, kk, 0.0), torch.where(some, vv, 0.0)
            most = vv.abs().amax() if ks is None else 2 * 127 * torch.where(some, scales, 0.0).amax()
            for x in range(h * group, (h + 1) * group):
                qq = q[a:b, x].double()
                score = (qq @ kk.t() * scale).masked_fill(~seen, -math.inf)
                top = score.amax(1, keepdim=True)
                p = torch.exp(score - torch.where(top == -math.inf, 0.0, top))
                total = p.sum(1, keepdim=True).clamp_min(1e-300)
                o = p @ vv / total
                mass = p @ vv.abs() / total
                off = abs(scale) * (d + 8) * U32 * (qq.abs() @ kk.abs().t()).amax(1, keepdim=True) + 2.0 ** -16
                out[a:b, x] = o
                tol[a:b, x] += U16 * o.abs() + U16 * mass + cut * length * most / total + 3 * off * mass
    return out, tol


class Case:
    """A batch: `new` and `lengths` of each sequence, caches and tables that hold garbage where nothing may read."""

    def __init__(self, seed, new, lengths, H, heads, d, page=16, bits=16, layout="heads", spare=4, columns=False):
        g = gen(seed)
        need = sum(-(-max(n, 0) // page) for n in lengths)
        self.n_pages = need + spare
        self.k, self.v, self.ks, self.vs = make_cache(g, self.n_pages, heads, page, d, bits, layout)
        self.table, self.unused = make_table(g, lengths, page, self.n_pages, unused=1 << 30)
        self.new, self.lengths, self.page, self.H, self.heads, self.d = new, lengths, page, H, heads, d
        self.starts = [0]
        for n in new:
            self.starts.append(self.starts[-1] + n)
        M = max(self.starts[-1], 1)
        if columns:                     # a range of the columns of a wider tensor, as a projection gives it
            self.q = normal(g, M, (H + 2 * heads) * d)[:, :H * d].view(M, H, d)
        else:
            self.q = normal(g, M, H, d)
        self.g = g
        # the unused pages, and what stands behind each sequence in its last page, are NaN
        bad = math.nan
        for x in (self.k, self.v):
            if bits == 16:
                x[self.unused] = bad
        for x in (self.ks, self.vs):
            if x is not None:
                x[self.unused] = bad
        for s, n in enumerate(lengths):
            if n > 0 and n % page:
                p = int(self.table[s, n // page])
                for x in (self.k, self.v):
                    if bits == 16:
                        x[p, :, n % page:] = bad
                for x in (self.ks, self.vs):
                    if x is not None:
                        x[p, :, n % page:] = bad

    def scales(self):
        return dict(k_scale=self.ks, v_scale=self.vs)

    def exact(self, seen_of, scale=None):
        return rows64(self.q, self.k, self.v, self.ks, self.vs, self.table, self.starts, self.lengths, seen_of,
                      self.d ** -0.5 if scale is None else scale)

    def device(self):
        return ints(self.starts), ints(self.lengths)


def random_tree(n, seed, kind="tree"):
    import random
    r = random.Random(seed)
    if n == 0:
        return []
    if kind == "chain":
        return [i - 1 for i in range(n)]
    if kind == "star":
        return [-1] + [0] * (n - 1)
    if kind == "forest":
        return [r.randint(-1, i - 1) for i in range(n)]
    return [-1] + [r.randint(max(0, i - 9), i - 1) for i in range(1, n)]


def verify64(target, draft, tokens, parents, uniforms, starts):
    """The verification from its definition, on the host: target, draft float32 tensors on the host or the device."""
    path, counts, said = [], [], []
    V = target.shape[1]
    for a, b in zip(starts, starts[1:]):
        n = b - a
        if n == 0:
            counts.append(0)
            said.append(-1)
            continue
        v, way, answer = 0, [0], None
        while answer is None:
            p = target[a + v].double()
            children = [c for c in range(v + 1, n) if parents[a + c] == v]
            taken = None
            if uniforms is None:
                best = int((p == p.max()).nonzero()[0])
                taken = next((c for c in children if tokens[a + c] == best), None)
                if taken is None:
                    answer = best
            else:
                r, Z = p, 1.0
                for c in children:
                    x = tokens[a + c]
                    if not 0 <= x < V:
                        continue
                    if draft is not None:
                        q = draft[a + v].double()
                    else:
                        q = torch.zeros_like(p)
                        q[x] = 1.0
                    if float(uniforms[a + c]) * float(q[x]) * Z < float(r[x]):
                        taken = c
                        break
                    r = (r / Z - q).clamp_min(0.0)
                    Z = float(r.sum())
                    if Z == 0.0:
                        r = p
                        break
                if taken is None:
                    up = r.cumsum(0)
                    total = float(up[-1])
                    if total > 0:
                        past = (up > float(uniforms[a]) * total).nonzero()
                        answer = int(past[0]) if len(past) else int(r.nonzero()[-1])
                    else:
                        answer = -1
            if taken is not None:
                v = taken
                way.append(v)
        path += (way + [-1] * n)[:n]
        counts.append(len(way))
        said.append(answer)
    return path, counts, said


__all__ = [n for n in dir() if not n.startswith("__")]
