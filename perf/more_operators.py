"""What a block needs when a sequence has several new tokens, as measurable cases: prompts, and trees of drafted tokens.

Five kinds, each one pass through one operator:

  window   the new tokens of every sequence attend to its paged key-value cache, causally, within a sliding
           window and to the first few tokens, which stay visible
  tree     the nodes of a drafted tree attend to the cache, to the nodes above them and to themselves
  verify   drafted trees (chains among them) against the target's probabilities, from given random numbers
  copy     pages of the cache to other pages: a forked sequence, a pool that closes its gaps
  compact  the accepted nodes of every tree move to the front of its new tokens in the cache

Head counts and widths are those of the GPT-2 models that `synth.config_cases` takes its projections from
(12 and 20 heads of 64, 50257 tokens), beside generic ones with shared key-value heads and heads of 128.
Everything is drawn from the seed.

With `own` false `run` computes the operators from elementary torch operations, attention in 32 bits and
probabilities in 64, where sums decide which token is next.
"""
import math

import torch

own = False

DEV = "cuda"


def _window(name, S, M, H, Hkv, d, prefix_from, prefix_to, *, window=0, sinks=0, page=16, bits=16, idle=False, layout="heads"):
    """M new tokens in S sequences, behind cached prefixes spread evenly; `idle`: the first sequence has a length of none."""
    return _named({"kind": "window", "S": S, "M": M, "H": H, "Hkv": Hkv, "d": d, "prefix_from": prefix_from,
                   "prefix_to": prefix_to, "window": window, "sinks": sinks, "page": page, "bits": bits, "idle": idle,
                   "layout": layout}, name)


def _tree(name, S, nodes, H, Hkv, d, prefix_from, prefix_to, *, branch=2, page=16, bits=16, layout="heads"):
    """S trees of half of `nodes` to `nodes` nodes, `branch` children to a node; 1: chains."""
    return _named({"kind": "tree", "S": S, "nodes": nodes, "H": H, "Hkv": Hkv, "d": d, "prefix_from": prefix_from,
                   "prefix_to": prefix_to, "branch": branch, "page": page, "bits": bits, "layout": layout}, name)


def _verify(name, S, nodes, V, *, branch=2, draw="sampled"):
    """`draw`: how the drafted tokens were found: "sampled" from the draft's probabilities, "given" without any, "greedy"."""
    return _named({"kind": "verify", "S": S, "nodes": nodes, "V": V, "branch": branch, "draw": draw}, name)


def _copy(name, copies, pages, Hkv, d, *, page=16, bits=16, layout="heads"):
    return _named({"kind": "copy", "copies": copies, "pages": pages, "Hkv": Hkv, "d": d, "page": page, "bits": bits,
                   "layout": layout}, name)


def _compact(name, S, nodes, accepted, Hkv, d, prefix, *, page=16, bits=16, layout="heads"):
    return _named({"kind": "compact", "S": S, "nodes": nodes, "accepted": accepted, "Hkv": Hkv, "d": d, "prefix": prefix,
                   "page": page, "bits": bits, "layout": layout}, name)


def _named(case, name):
    return case if name is None else {"name": name, **case}


def listed():
    return [
        # a decode step of 24 sequences of GPT-2 large, up to a full context, with a window over 8-bit codes; one
        # place of the batch is idle
        _window("window_24x20x64_1024_int8", 24, 24, 20, 20, 64, 0, 1023, window=256, sinks=4, bits=8, idle=True),
        # a prompt of GPT-2 small that fills its context, no window; the cache's tokens stand before its heads
        _window("window_1024x12x64", 1, 1024, 12, 12, 64, 0, 0, layout="tokens"),
        # packed prompts of odd lengths, some behind a cached prefix, over 8-bit codes
        _window("window_8192x32of8x128_int8", 13, 8192, 32, 8, 128, 0, 1500, window=1024, sinks=4, page=32, bits=8),
        # one long document, read in one pass with a window: the largest
        _window("window_16384x32of8x128", 1, 16384, 32, 8, 128, 0, 0, window=4096, sinks=4, page=32),
        # eight drafted nodes of GPT-2 small a few words into its answer: all latency
        _tree("tree_1x8x12x64_37", 1, 8, 12, 12, 64, 37, 37),
        # a drafting step of 64 sequences of a generic model, ragged lengths and trees
        _tree("tree_64x32x32of8x128_8192", 64, 32, 32, 8, 128, 100, 8150, branch=3),
        # one user, a chain of four drafted tokens, greedy
        _verify("verify_1x5x50257_greedy", 1, 5, 50257, branch=1, draw="greedy"),
        # 64 users with drafted trees, sampled
        _verify("verify_64x32x50257", 64, 32, 50257, branch=3),
        # a sequence of GPT-2 small forks: its last, half-filled page
        _copy("copy_1x12x64", 1, 80, 12, 64),
        # a pool closes its gaps: 4096 pages move to its lower end
        _copy("copy_4096x8x128", 4096, 8192, 8, 128, page=32),
        # one user's accepted nodes
        _compact("compact_1x8x12x64", 1, 8, 3, 12, 64, 37),
        # the accepted nodes of 64 trees, in 8-bit codes
        _compact("compact_64x32x8x128_int8", 64, 32, 7, 8, 128, 1000, page=32, bits=8),
    ]


def _log_int(rng, lo, hi, step=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(lo, min(hi, int(round(v / step)) * step))


def draw(rng):
    kind = rng.choices(["window", "tree", "verify", "copy", "compact"], [4, 3, 3, 1, 1])[0]
    d = rng.choice([64, 64, 80, 96, 128])
    Hkv = rng.choice([1, 2, 4, 8, 12, 16, 20])
    H = Hkv * rng.choice([1, 1, 2, 4, 7, 8])
    shape = {"page": rng.choice([16, 16, 32, 64]), "bits": rng.choice([16, 16, 8]), "layout": rng.choice(["heads", "heads", "tokens"])}
    if kind == "verify":
        how = rng.choice(["sampled", "sampled", "given", "greedy"])
        case = _verify(None, _log_int(rng, 1, 64), _log_int(rng, 2, 64), _log_int(rng, 1000, 131072), branch=rng.choice([1, 2, 3, 4]), draw=how)
        while case["S"] * case["nodes"] * case["V"] > 64 * 32 * 50257:
            case["S"] = (case["S"] + 1) // 2
            case["V"] = case["V"] * 3 // 4
        return case
    if kind == "copy":
        copies = _log_int(rng, 1, 4096)
        while copies * Hkv * d * shape["page"] > 4096 * 8 * 128 * 32:
            copies = (copies + 1) // 2
        return _copy(None, copies, 2 * copies + rng.randint(0, 50), Hkv, d, **shape)
    if kind == "compact":
        nodes = _log_int(rng, 3, 64)
        return _compact(None, _log_int(rng, 1, 128), nodes, rng.randint(1, (nodes + 1) // 2), Hkv, d, _log_int(rng, 1, 2000), **shape)
    prefix = _log_int(rng, 1, 16384) - 1
    start = int(prefix * rng.random())
    if kind == "tree":
        case = _tree(None, _log_int(rng, 1, 64), _log_int(rng, 2, 64), H, Hkv, d, start, prefix, branch=rng.choice([1, 2, 3, 4]), **shape)
        most = work(listed()[5])
    else:
        M = _log_int(rng, 1, 8192)
        S = M if M <= 64 and rng.random() < 0.4 else min(M, _log_int(rng, 1, 64))
        window = rng.choice([0, 0, _log_int(rng, 1, 4096)])
        case = _window(None, S, M, H, Hkv, d, start, prefix, window=window, sinks=rng.choice([0, 1, 4, 4, 64]) if window else 0,
                       idle=S > 1 and rng.random() < 0.3, **shape)
        most = {"flops": work(listed()[3])["flops"], "bytes": work(listed()[5])["bytes"]}
    # a case's work, and what its sequences hold, at most the largest's
    while (any(work(case)[x] > most[x] for x in most) or
           sum(_lengths(case)) * case["Hkv"] * case["d"] > 64 * 4160 * 8 * 128 or
           (kind == "window" and case["M"] * max(_lengths(case)) * case["H"] > 16384 * 16384 * 32)):
        case["S"] = (case["S"] + 1) // 2
        if kind == "window":
            case["M"] = max(case["S"], case["M"] * 3 // 4)
            case["idle"] = case["idle"] and case["S"] > 1
        case["prefix_to"] = case["prefix_to"] * 3 // 4
        case["prefix_from"] = min(case["prefix_from"], case["prefix_to"])
    return case


# ---- inputs --------------------------------------------------------------------------------


def _shares(total, parts):
    """`total` tokens in `parts` requests, each a little longer than the one before."""
    edges = [total * (i * (i + parts)) // (parts * 2 * parts) for i in range(parts + 1)]
    edges = [max(e, i) for i, e in enumerate(edges)]
    edges[-1] = total
    for i in range(parts - 1, 0, -1):
        edges[i] = min(edges[i], edges[i + 1] - 1)
    return edges


def _new(case):
    """The new tokens of each sequence."""
    S = case["S"]
    if case["kind"] == "window":
        edges = _shares(case["M"], S)
        return [b - a for a, b in zip(edges, edges[1:])]
    n = case["nodes"]
    if case["kind"] == "tree":
        return [n if S == 1 else n - (n // 2) * (i * 7 % S) // S for i in range(S)]
    return [n] * S


def _prefixes(case):
    S, lo, hi = case["S"], case["prefix_from"], case["prefix_to"]
    return [hi if S == 1 else lo + (hi - lo) * (i * 5 % S) // (S - 1) for i in range(S)]


def _lengths(case):
    """The tokens of each sequence in the cache, the new ones among them."""
    if case["kind"] == "compact":
        return [case["prefix"] + i * 13 % 50 + case["nodes"] for i in range(case["S"])]
    lens = [p + n for p, n in zip(_prefixes(case), _new(case))]
    return [0] + lens[1:] if case.get("idle") else lens


def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _half(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV, dtype=torch.float16)


def _int(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _order(n, g):
    return torch.randperm(n, generator=g, device=DEV).tolist()


def _cache(g, case, n_pages):
    """Keys and values of a running program: [pages, heads, tokens of a page, d], in the case's order in memory."""
    Hkv, page, d = case["Hkv"], case["page"], case["d"]
    tokens_first = case["layout"] == "tokens"
    shape = (n_pages, page, Hkv, d) if tokens_first else (n_pages, Hkv, page, d)
    out = {}
    for name in ("k", "v"):
        if case["bits"] == 16:
            c = _half(g, *shape)
        else:
            c = (_half(g, *shape) * 40).clamp_(-127, 127).round_().to(torch.int8)
            out[name + "_scale"] = 0.01 + 0.03 * torch.rand(n_pages, Hkv, page, generator=g, device=DEV)
        out[name] = c.transpose(1, 2) if tokens_first else c
    return out


def _parents(nodes, branch):
    """A tree in the order of its levels; the root's parent is -1."""
    return [(i - 1) // branch if i else -1 for i in range(nodes)]


def _sequences(g, case, s):
    lens, new, page = _lengths(case), _new(case), case["page"]
    need = [-(-n // page) for n in lens]
    pages = _order(sum(need) + 5, g)
    table = torch.zeros(len(lens), max(max(need), 1), dtype=torch.int32)
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = torch.tensor(pages[at:at + n], dtype=torch.int32)
        at += n
    s.update(_cache(g, case, len(pages)))
    edges = [0]
    for n in new:
        edges.append(edges[-1] + n)
    s["table"], s["lengths"], s["starts"] = table.to(DEV), _int(lens), _int(edges)
    s["longest"], s["most_new"], s["M"] = max(max(lens), 1), max(new), edges[-1]


def _prepare_verify(g, case, s):
    S, n, V, branch, how = case["S"], case["nodes"], case["V"], case["branch"], case["draw"]
    parents = _parents(n, branch)
    # the draft is the target's opinion, blurred
    logits = 2.5 * torch.randn(S, n, V, generator=g, device=DEV)
    target = torch.softmax(logits, 2)
    blurred = torch.softmax(logits + 0.7 * torch.randn(S, n, V, generator=g, device=DEV), 2)
    del logits
    above = torch.tensor([0] + parents[1:], device=DEV)
    if how == "greedy":
        tokens = target.argmax(2)[:, above]             # what the target would say after the parent ...
        wrong = torch.randint(0, V, (S, n), generator=g, device=DEV)
        node = torch.arange(n, device=DEV)
        # ... in the first half of the nodes, and for its last child only
        right = (node <= n // 2) & ((node % branch == 0) | (node == n // 2))
        tokens = torch.where(right, tokens, wrong)
    else:
        tokens = torch.multinomial(blurred.view(S * n, V), branch, replacement=True, generator=g).view(S, n, branch)
        nth = torch.tensor([(i - 1) % branch if i else 0 for i in range(n)], device=DEV)
        tokens = tokens[:, above, nth]
    s["tokens"] = tokens.int().reshape(-1).contiguous()
    s["target"] = target.view(S * n, V)
    s["draft"] = blurred.view(S * n, V) if how == "sampled" else None
    s["uniforms"] = None if how == "greedy" else torch.rand(S * n, generator=g, device=DEV)
    s["parents"], s["starts"] = _int(parents * S), _int([i * n for i in range(S + 1)])


def prepare(case, seed):
    g = _generator(seed)
    kind = case["kind"]
    s = {"case": case}
    if kind in ("window", "tree"):
        _sequences(g, case, s)
        s["q"] = _half(g, s["M"], case["H"], case["d"])
        s["out"] = torch.empty_like(s["q"])
        if kind == "tree":
            s["parents"] = _int([p for n in _new(case) for p in _parents(n, case["branch"])])
    elif kind == "verify":
        _prepare_verify(g, case, s)
    elif kind == "copy":
        n, order = case["copies"], _order(case["pages"], g)
        s.update(_cache(g, case, case["pages"]))
        s["src"], s["dst"] = _int(order[:n]), _int(order[n:2 * n])
    else:
        _sequences(g, case, s)
        n, path, counts = case["nodes"], [], []
        for i in range(case["S"]):
            kept = 1 + (case["accepted"] - 1) * (3 - i % 3) // 3
            # behind the places they go to, so that a pass can be made again
            behind = sorted(x + kept for x in _order(n - kept, g)[:kept - 1])
            path += ([0] + behind + [-1] * n)[:n]
            counts.append(1 + len(behind))
        s["path"], s["counts"] = _int(path), _int(counts)
    return s


# ---- one pass ------------------------------------------------------------------------------


def run(state):
    return _run_own(state) if own else _PLAIN[state["case"]["kind"]](state)


def _run_own(s):
    from paper_2604_04701_amd import binding as B
    c = s["case"]
    kind = c["kind"]
    scales = {"k_scale": s.get("k_scale"), "v_scale": s.get("v_scale")}
    if kind == "window":
        if "workspace" not in s:        # a serving program keeps it
            s["workspace"] = B.alloc_window_attention_workspace(c["S"], c["H"], c["Hkv"], c["d"], s["most_new"], s["longest"],
                                                                c["window"], c["sinks"])
        return B.muxq_window_attention(s["q"], s["k"], s["v"], s["table"], s["starts"], s["lengths"], s["most_new"], s["longest"],
                                       window=c["window"], sinks=c["sinks"], out=s["out"], workspace=s["workspace"], **scales)
    if kind == "tree":
        if "workspace" not in s:
            s["workspace"] = B.alloc_tree_attention_workspace(c["S"], c["H"], c["Hkv"], c["d"], s["most_new"], s["longest"])
        return B.muxq_tree_attention(s["q"], s["k"], s["v"], s["table"], s["starts"], s["lengths"], s["parents"], s["most_new"],
                                     s["longest"], out=s["out"], workspace=s["workspace"], **scales)
    if kind == "verify":
        return B.muxq_verify_tree(s["target"], s["tokens"], s["starts"], s["parents"], c["nodes"], draft=s["draft"],
                                  uniforms=s["uniforms"])
    if kind == "copy":
        B.muxq_kv_copy(s["src"], s["dst"], s["k"], s["v"], **scales)
    else:
        B.muxq_kv_compact(s["path"], s["counts"], s["starts"], s["lengths"], s["table"], s["k"], s["v"], c["nodes"], **scales)
    return [s[x] for x in ("k", "v", "k_scale", "v_scale") if x in s]


def _plain_attention(s):
    c = s["case"]
    H, Hkv, d, page = c["H"], c["Hkv"], c["d"], c["page"]
    new, lens = _new(c), _lengths(c)
    out = torch.zeros(s["M"], H, d, dtype=torch.float16, device=DEV)

    def rows(name, pages, n):           # [Hkv, tokens, d] in 32 bits
        x = s[name][pages].float()
        if c["bits"] == 8:
            x = x * s[name + "_scale"][pages].unsqueeze(-1)
        return x.transpose(0, 1).reshape(Hkv, -1, d)[:, :n]

    at = 0
    for i, (n, length) in enumerate(zip(new, lens)):
        if length == 0:
            at += n
            continue
        pages = s["table"][i, :-(-length // page)].long()
        k, v = rows("k", pages, length), rows("v", pages, length)
        t = torch.arange(length, device=DEV)
        first = length - n
        if c["kind"] == "tree":
            seen = _visible_nodes(s["parents"][at:at + n].long(), n)
        step = max(1, 2 ** 30 // (H * length))
        for a in range(0, n, step):
            b = min(n, a + step)
            p = first + torch.arange(a, b, device=DEV)[:, None]
            if c["kind"] == "tree":
                there = torch.cat([torch.ones(b - a, first, dtype=torch.bool, device=DEV), seen[a:b]], 1)
            else:
                there = t <= p
                if c["window"]:
                    there &= (t > p - c["window"]) | (t < c["sinks"])
            q = s["q"][at + a:at + b].float().view(b - a, Hkv, H // Hkv, d).permute(1, 2, 0, 3).reshape(Hkv, -1, d)
            score = torch.matmul(q, k.transpose(1, 2).contiguous()) / math.sqrt(d)
            score = score.view(H, b - a, length).masked_fill_(~there, -math.inf)
            score = torch.exp(score - score.amax(2, keepdim=True))
            total = score.sum(2, keepdim=True)
            o = torch.matmul(score.view(Hkv, -1, length), v).view(H, b - a, d) / total
            out[at + a:at + b] = o.transpose(0, 1).half()
        at += n
    return out


def _visible_nodes(parents, n):
    """[n, n]: a node sees itself and what its parent sees."""
    seen = torch.eye(n, dtype=torch.bool, device=DEV)
    up = parents
    for _ in range(n - 1):
        there = up >= 0
        seen |= there[:, None] & (torch.arange(n, device=DEV) == up[:, None])
        up = torch.where(there, parents[up.clamp_min(0)], up)
    return seen


def _plain_verify(s):
    c = s["case"]
    S, n, V = c["S"], c["nodes"], c["V"]
    target = s["target"].view(S, n, V)
    tokens, parents = s["tokens"].view(S, n).long(), s["parents"].view(S, n)
    every = torch.arange(S, device=DEV)
    at = torch.zeros(S, dtype=torch.int64, device=DEV)         # the last accepted node
    count = torch.ones_like(at)
    path = torch.full((S, n), -1, dtype=torch.int32, device=DEV)
    path[:, 0] = 0
    greedy = c["draw"] == "greedy"
    if greedy:
        best = target.argmax(2)
    else:
        u = s["uniforms"].view(S, n).double()
        rest = target[:, 0].double()
        total = torch.ones(S, dtype=torch.float64, device=DEV)
    for i in range(1, n):
        mine, token = parents[:, i] == at, tokens[:, i]
        if greedy:
            yes = mine & (best[every, at] == token)
        else:
            if c["draw"] == "sampled":
                q = s["draft"].view(S, n, V)[every, at].double()
            else:
                q = (torch.arange(V, device=DEV) == token[:, None]).double()
            yes = mine & (u[:, i] * q[every, token] * total < rest[every, token])
            less = (rest / total[:, None] - q).clamp_min(0.0)
            sum_less = less.sum(1)
            no = mine & ~yes
            rest = torch.where(no[:, None], less, rest)
            total = torch.where(no, sum_less, total)
            rest = torch.where(yes[:, None], target[:, i].double(), rest)
            total = torch.where(yes, 1.0, total)
        at = torch.where(yes, i, at)
        path[every, torch.where(yes, count, 0)] = torch.where(yes, i, 0).int()
        count = count + yes
    if greedy:
        token = best[every, at]
    else:
        rest = torch.where((rest.sum(1) > 0)[:, None], rest, target[every, at].double())
        up = rest.cumsum(1)
        token = (up <= u[:, :1] * up[:, -1:]).sum(1)
        last = V - 1 - (rest > 0).flip(1).int().argmax(1)
        token = torch.minimum(token, last)
    return path.view(-1), count.int(), token.int()


def _all_of(s):
    return [s[x] for x in ("k", "v", "k_scale", "v_scale") if x in s]


def _plain_copy(s):
    src, dst = s["src"].long(), s["dst"].long()
    for x in _all_of(s):
        x[dst] = x[src]
    return _all_of(s)


def _plain_compact(s):
    c = s["case"]
    S, n, page = c["S"], c["nodes"], c["page"]
    j = torch.arange(n, device=DEV)
    first = s["lengths"].long()[:, None] - n
    kept = j < s["counts"][:, None]
    table = s["table"].long()
    path = s["path"].view(S, n).long()

    def place(token):
        return table.gather(1, token // page)[kept], (token % page)[kept]

    (from_page, from_at), (to_page, to_at) = place(first + path.clamp_min(0)), place(first + j.expand(S, n))
    for x in _all_of(s):
        x[to_page, :, to_at] = x[from_page, :, from_at]
    return _all_of(s)


_PLAIN = {"window": _plain_attention, "tree": _plain_attention, "verify": _plain_verify, "copy": _plain_copy, "compact": _plain_compact}


# ---- what a pass cannot do without -----------------------------------------------------------


def _clamped_sum(first, n, most):
    """The sum of min(most, first + i) over i < n."""
    full = max(0, min(n, first + n - most))          # terms that are `most`
    m = n - full
    return m * first + m * (m - 1) // 2 + full * most


def _row_bytes(case):
    return 2 * case["Hkv"] * (case["d"] * case["bits"] // 8 + (4 if case["bits"] == 8 else 0))


def work(case):
    kind = case["kind"]
    if kind == "verify":
        # the row that a sequence's walk ends at, of both models where the draft's counts
        rows = case["S"] * (2 if case["draw"] == "sampled" else 1)
        return {"bytes": 4 * rows * case["V"] + 16 * case["S"] * case["nodes"], "flops": 2 * rows * case["V"]}
    if kind == "copy":
        return {"bytes": 2 * case["copies"] * case["page"] * _row_bytes(case) + 8 * case["copies"], "flops": 1}
    if kind == "compact":
        moved = sum((case["accepted"] - 1) * (3 - i % 3) // 3 for i in range(case["S"]))
        return {"bytes": 2 * moved * _row_bytes(case) + 20 * case["S"], "flops": 1}
    H, d = case["H"], case["d"]
    read = pairs = pages = 0
    for n, length in zip(_new(case), _lengths(case)):
        if length == 0:
            continue
        first = length - n
        if kind == "tree":
            depth, level, at = [], 0, 0
            while at < n:                                   # nodes of each level of the tree
                width = min(n - at, case["branch"] ** level)
                depth.append(width)
                at, level = at + width, level + 1
            pairs += n * first + sum((i + 1) * w for i, w in enumerate(depth))
            read += length
        elif case["window"]:
            w, k = case["window"], case["sinks"]
            pairs += _clamped_sum(first + 1, n, w + k) if k else _clamped_sum(first + 1, n, w)
            read += min(length, w + n - 1 + k)
        else:
            pairs += n * first + n * (n + 1) // 2
            read += length
        pages += -(-length // case["page"])
    M = sum(_new(case))
    return {"bytes": read * _row_bytes(case) + 4 * M * H * d + 4 * pages + 8 * case["S"], "flops": max(1, 4 * pairs * H * d)}


# ---- the same in 64 bits ---------------------------------------------------------------------


def _exact_attention(s):
    c = s["case"]
    d, page, group = c["d"], c["page"], c["H"] // c["Hkv"]
    out = torch.zeros(s["M"], c["H"], d, dtype=torch.float64, device=DEV)
    starts = s["starts"].tolist()
    for i, length in enumerate(s["lengths"].tolist()):
        a, b = starts[i], starts[i + 1]
        if length == 0 or a == b:
            continue
        used = s["table"][i, :-(-length // page)].long()
        keys = torch.arange(length, device=DEV)
        n = b - a
        hidden = torch.zeros(n, length, dtype=torch.bool, device=DEV)
        if c["kind"] == "tree":
            parents = s["parents"][a:b].tolist()
            hidden[:, length - n:] = True
            for x in range(n):
                y = x
                while y >= 0:
                    hidden[x, length - n + y] = False
                    y = parents[y]
        else:
            # how far behind its query a key stands
            behind = torch.arange(length - n, length, device=DEV)[:, None] - keys
            hidden = behind < 0
            if c["window"]:
                hidden |= (behind >= c["window"]) & (keys >= c["sinks"])
        for h in range(c["Hkv"]):
            k, v = (s[name][used, h].double().reshape(-1, d)[:length] for name in ("k", "v"))
            if c["bits"] == 8:
                k, v = (x * s[name][used, h].double().reshape(-1)[:length, None] for x, name in ((k, "k_scale"), (v, "v_scale")))
            for x in range(h * group, (h + 1) * group):
                score = torch.mm(s["q"][a:b, x].double(), k.t().contiguous()) * d ** -0.5
                out[a:b, x] = torch.mm(torch.softmax(score.masked_fill_(hidden, -math.inf), 1), v)
    return out


def _exact_verify(s):
    c = s["case"]
    n = c["nodes"]
    paths, counts, said = [], [], []
    parents, tokens = s["parents"].tolist(), s["tokens"].tolist()
    u = None if s["uniforms"] is None else s["uniforms"].tolist()
    for base in s["starts"].tolist()[:-1]:
        at, path, answer = 0, [0], None
        while answer is None:
            p = s["target"][base + at].double()
            children = [i for i in range(n) if parents[base + i] == at and i > 0]
            if c["draw"] == "greedy":
                best = int((p == p.max()).nonzero()[0])
                taken = [i for i in children if tokens[base + i] == best][:1]
                answer = None if taken else best
            else:
                taken, left = [], p
                for i in children:
                    x = tokens[base + i]
                    if c["draw"] == "sampled":
                        q = s["draft"][base + at].double()
                    else:
                        q = torch.zeros_like(p)
                        q[x] = 1.0
                    if u[base + i] * float(q[x]) < float(left[x]):
                        taken = [i]
                        break
                    left = torch.relu(left - q)
                    if float(left.sum()) == 0.0:
                        left = p
                        break
                    left = left / left.sum()
                if not taken:
                    up = torch.cumsum(left, 0)
                    answer = int(torch.searchsorted(up, u[base] * up[-1], right=True))
                    answer = min(answer, int(left.nonzero()[-1]))
            if taken:
                at = taken[0]
                path.append(at)
        paths += (path + [-1] * n)[:n]
        counts.append(len(path))
        said.append(answer)
    return _int(paths), _int(counts), _int(said)


def _exact_copy(s):
    to = dict(zip(s["dst"].tolist(), s["src"].tolist()))
    pages = torch.tensor([to.get(i, i) for i in range(s["k"].shape[0])], device=DEV)
    return [x.index_select(0, pages).double() for x in _all_of(s)]


def _exact_compact(s):
    n, page = s["case"]["nodes"], s["case"]["page"]
    outs = [x.transpose(1, 2).double() for x in _all_of(s)]         # [pages, tokens, heads, ...]
    outs = [x.contiguous() for x in outs]
    starts, lengths, table, path = (s[x].tolist() for x in ("starts", "lengths", "table", "path"))
    for i, kept in enumerate(s["counts"].tolist()):
        where = [table[i][t // page] * page + t % page for t in range(lengths[i] - n, lengths[i])]
        for x in outs:
            flat = x.view(-1, *x.shape[2:])
            flat[where[:kept]] = flat[[where[j] for j in path[starts[i]:starts[i] + kept]]]
    return [x.transpose(1, 2) for x in outs]


_EXACT = {"window": _exact_attention, "tree": _exact_attention, "verify": _exact_verify, "copy": _exact_copy, "compact": _exact_compact}


def exact(case, seed):
    return _EXACT[case["kind"]](prepare(case, seed))
