"""The operators between the quantised projections of a block that serves requests, as measurable cases.

Four kinds, each one pass through one operator:

  attend   one new token of every sequence attends to the sequence's paged key-value cache
  append   keys and values of new tokens go to their slots of the paged cache, rotated by their
           position on the way (queries too); a cache of 8-bit codes is read back for comparison
  lora     low-rank adapters of many requests beside a shared projection: Y + s_i (X A_i^T) B_i^T
  norm     the norm after a block, its gate, the residual stream and the norm in front of the next
           block, with the column maxima that the next quantised layer starts from

Head counts and widths are those of the GPT-2 models that `synth.config_cases` takes its
projections from (12 and 20 heads of 64, widths 768 to 1280), beside generic ones with shared
key-value heads and heads of 128.  Activations are normal, with a few loud channels where a
projection reads them; everything is drawn on the GPU from the seed.

With `own` false `run` computes the operators from elementary torch operations in 32 bits.
"""
import math

import torch

own = False

DEV = "cuda"
EPS = 1e-5


def _attend(name, S, H, Hkv, d, shortest, longest, *, page=16, bits=16, idle=False, layout="heads"):
    """S sequences with lengths spread evenly from `shortest` to `longest`; `idle`: the first has none."""
    return _named({"kind": "attend", "S": S, "H": H, "Hkv": Hkv, "d": d, "shortest": shortest, "longest": longest,
                   "page": page, "bits": bits, "idle": idle, "layout": layout}, name)


def _append(name, M, requests, H, Hkv, d, *, rotated=0, interleaved=False, page=16, bits=16, padded=0, layout="heads"):
    """M tokens of `requests` sequences, the last `padded` of them without a slot; `rotated`: dimensions that rotate."""
    return _named({"kind": "append", "M": M, "requests": requests, "H": H, "Hkv": Hkv, "d": d, "rotated": rotated,
                   "interleaved": interleaved, "page": page, "bits": bits, "padded": padded, "layout": layout}, name)


def _lora(name, M, requests, K, N, r, adapters):
    return _named({"kind": "lora", "M": M, "requests": requests, "K": K, "N": N, "r": r, "adapters": adapters}, name)


def _norm(name, M, K, *, root_mean=False, post=False, gate=False, residual_scale=1.0):
    return _named({"kind": "norm", "M": M, "K": K, "root_mean": root_mean, "post": post, "gate": gate,
                   "residual_scale": residual_scale}, name)


def _named(case, name):
    return case if name is None else {"name": name, **case}


def listed():
    return [
        # one sequence of GPT-2 small a few words into its answer: the smallest call, all latency;
        # the cache's tokens stand before its heads
        _attend("attend_1x12x64_37", 1, 12, 12, 64, 37, 37, layout="tokens"),
        # a decode step of 24 sequences of GPT-2 large, up to a full context, in 8-bit codes; one place
        # of the batch is idle
        _attend("attend_24x20x64_1024_int8", 24, 20, 20, 64, 1, 1024, bits=8, idle=True),
        # one long document and nothing else: a single row split over the cache's length
        _attend("attend_1x32of8x128_131072", 1, 32, 8, 128, 131071, 131071, page=32),
        # a full decode step of a generic model with four queries to a key-value head, ragged lengths:
        # the largest
        _attend("attend_64x32of8x128_8192", 64, 32, 8, 128, 131, 8192),
        # one token of GPT-2 small goes to the cache, no rotation
        _append("append_1x12x64", 1, 1, 12, 12, 64),
        # a decode step of 64 sequences in a batch padded by 3, rotated, into 8-bit codes
        _append("append_64x32of8x128_int8", 64, 64, 32, 8, 128, rotated=128, bits=8, padded=3),
        # packed prompts of odd lengths, rotated: the cache's pages are filled from the middle on
        _append("append_8192x32of8x128", 8192, 13, 32, 8, 128, rotated=128, page=32),
        # one token of one request beside c_attn of GPT-2 small
        _lora("lora_1x768x2304_r8", 1, 1, 768, 2304, 8, 4),
        # a decode step of 64 requests with 24 adapters beside c_attn of GPT-2 large
        _lora("lora_64x1280x3840_r16", 64, 64, 1280, 3840, 16, 24),
        # packed prompts of 21 requests beside a generic square projection
        _lora("lora_8192x4096x4096_r32", 8192, 21, 4096, 4096, 32, 8),
        # a decode step of 24 sequences of GPT-2 large: the residual stream and ln_2
        _norm("norm_24x1280", 24, 1280),
        # sixteen contexts of GPT-2 large through a block with norms on both sides and a gate
        _norm("norm_16384x1280_both_gate", 16384, 1280, root_mean=True, post=True, gate=True, residual_scale=0.9),
    ]


def _log_int(rng, lo, hi, step=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(lo, min(hi, int(round(v / step)) * step))


def draw(rng):
    kind = rng.choices(["attend", "append", "lora", "norm"], [4, 2, 3, 2])[0]
    d = rng.choice([64, 64, 80, 96, 128])
    Hkv = rng.choice([1, 2, 4, 8, 12, 16, 20])
    H = Hkv * rng.choice([1, 1, 2, 4, 7, 8])
    page = rng.choice([16, 16, 32, 64])
    bits = rng.choice([16, 16, 8])
    layout = rng.choice(["heads", "heads", "tokens"])
    if kind == "attend":
        S = _log_int(rng, 1, 256)
        longest = _log_int(rng, 1, 131072)
        case = _attend(None, S, H, Hkv, d, max(1, int(longest * rng.random())), longest, page=page, bits=bits,
                       idle=S > 1 and rng.random() < 0.3, layout=layout)
        most = work(listed()[3])["bytes"]
        while work(case)["bytes"] > most:
            case["S"] = (case["S"] + 1) // 2
            case["longest"] = (case["longest"] * 3 + 3) // 4
            case["shortest"] = min(case["shortest"], case["longest"])
        return case
    if kind == "append":
        M = _log_int(rng, 1, 8192)
        rotated = rng.choice([0, d, d, d // 2])
        return _append(None, M, min(M, _log_int(rng, 1, 256)), H, Hkv, d, rotated=rotated,
                       interleaved=rotated > 0 and rng.random() < 0.4, page=page, bits=bits,
                       padded=rng.randint(0, 3) if M > 8 else 0, layout=layout)
    if kind == "lora":
        M, K, N = _log_int(rng, 1, 8192), _log_int(rng, 256, 5120, 8), _log_int(rng, 256, 5120, 8)
        return _lora(None, M, min(M, _log_int(rng, 1, 128)), K, N, rng.choice([8, 16, 16, 24, 32, 64]), _log_int(rng, 1, 32))
    return _norm(None, _log_int(rng, 1, 16384), _log_int(rng, 256, 5120, 8), root_mean=rng.random() < 0.5,
                 post=rng.random() < 0.4, gate=rng.random() < 0.4, residual_scale=rng.choice([1.0, 1.0, 0.5]))


# ---- inputs --------------------------------------------------------------------------------


def _lengths(case):
    S, lo, hi = case["S"], case["shortest"], case["longest"]
    lens = [hi if S == 1 else lo + (hi - lo) * i // (S - 1) for i in range(S)]
    return [0] + lens[1:] if case["idle"] and S > 1 else lens


def _shares(total, parts):
    """`total` tokens in `parts` requests, each a little longer than the one before."""
    edges = [total * (i * (i + parts)) // (parts * 2 * parts) for i in range(parts + 1)]
    edges = [max(e, i) for i, e in enumerate(edges)]
    edges[-1] = total
    for i in range(parts - 1, 0, -1):
        edges[i] = min(edges[i], edges[i + 1] - 1)
    return edges


def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV, dtype=torch.float32)


def _half(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV, dtype=torch.float16)


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


def _loud(g, M, K):
    """Activations with one channel in two hundred 20 to 100 times louder."""
    x = _normal(g, M, K)
    ch = torch.randperm(K, generator=g, device=DEV)[:max(1, K // 200)]
    x[:, ch] *= 20.0 + 80.0 * torch.rand(ch.numel(), generator=g, device=DEV)
    return x.half()


def _int(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _order(n, g):
    return torch.randperm(n, generator=g, device=DEV).tolist()


def prepare(case, seed):
    g = _generator(seed)
    kind = case["kind"]
    s = {"case": case}
    if kind == "attend":
        lens, page = _lengths(case), case["page"]
        lens = [lens[i] for i in _order(len(lens), g)]
        need = [-(-n // page) for n in lens]
        pages = _order(sum(need) + 5, g)
        table = torch.zeros(len(lens), max(max(need), 1), dtype=torch.int32)
        at = 0
        for i, n in enumerate(need):
            table[i, :n] = torch.tensor(pages[at:at + n], dtype=torch.int32)
            at += n
        s.update(_cache(g, case, len(pages)))
        s["table"], s["lengths"], s["longest"] = table.to(DEV), _int(lens), max(lens)
        s["q"] = _half(g, case["S"], case["H"], case["d"])
        s["out"] = torch.empty_like(s["q"])
    elif kind == "append":
        M, page, d = case["M"], case["page"], case["d"]
        edges, positions, slots, used = _shares(M, case["requests"]), [], [], 0
        first = torch.randint(0, 1000, (case["requests"],), generator=g, device=DEV).tolist()
        spans = [(p, p + b - a) for p, a, b in zip(first, edges, edges[1:])]
        pages = _order(sum(-(-(e - b) // page) + 1 for b, e in spans), g)
        for b, e in spans:
            positions += range(b, e)
            slots += [pages[used + p // page - b // page] * page + p % page for p in range(b, e)]
            used += -(-e // page) - b // page
        slots[M - case["padded"]:] = [-1] * case["padded"]
        s.update(_cache(g, case, len(pages) + 1))       # the last page belongs to nobody
        s["pages"] = len(pages)
        s["slots"], s["positions"] = _int(slots), _int(positions)
        # what the projection in front gives: queries, keys and values of a token in one row
        s["qkv"] = _half(g, M, (case["H"] + 2 * case["Hkv"]) * d)
        s["q_out"] = torch.empty(M, case["H"], d, dtype=torch.float16, device=DEV)
        if case["rotated"]:
            half = case["rotated"] // 2
            angle = torch.arange(max(positions) + 1, device=DEV)[:, None] * 10000.0 ** (-torch.arange(half, device=DEV) / half)
            s["cos_sin"] = torch.cat([angle.cos(), angle.sin()], 1).float().contiguous()
        if case["bits"] == 8:
            s["k_back"] = torch.empty(M, case["Hkv"], d, dtype=torch.float16, device=DEV)
            s["v_back"] = torch.empty_like(s["k_back"])
    elif kind == "lora":
        M, K, N, r, n = case["M"], case["K"], case["N"], case["r"], case["adapters"]
        s["X"], s["Y"] = _loud(g, M, K), _half(g, M, N)
        s["A"] = (_normal(g, n, r, K) / math.sqrt(K)).half()
        s["B"] = (_normal(g, n, N, r) / math.sqrt(r)).half()
        s["scales"] = 0.5 + 1.5 * torch.rand(n, generator=g, device=DEV)
        s["starts"] = _int(_shares(M, case["requests"]))
        order = _order(n, g)
        s["adapter"] = _int([-1 if i % 8 == 7 else order[i % n] for i in range(case["requests"])])
        s["out"] = torch.empty_like(s["Y"])
    else:
        M, K = case["M"], case["K"]
        s["x"], s["residual"] = _half(g, M, K), _loud(g, M, K)
        s["weight"] = (1.0 + 0.2 * _normal(g, K)).half()
        s["bias"] = None if case["root_mean"] else (0.1 * _normal(g, K)).half()
        if case["post"]:
            s["post_weight"] = (1.0 + 0.2 * _normal(g, K)).half()
            s["post_bias"] = None if case["root_mean"] else (0.1 * _normal(g, K)).half()
        if case["gate"]:
            s["gate"] = (0.3 * _normal(g, K)).half()
        s["y"], s["stream"] = torch.empty_like(s["x"]), torch.empty_like(s["x"])
        s["maxima"] = torch.empty(64, -(-K // 64) * 64, dtype=torch.float16, device=DEV)
    return s


# ---- one pass ------------------------------------------------------------------------------


def run(state):
    return _run_own(state) if own else _PLAIN[state["case"]["kind"]](state)


def _run_own(s):
    from paper_2604_04701_amd import binding as B
    c = s["case"]
    kind = c["kind"]
    if kind == "attend":
        if "workspace" not in s:        # a serving program keeps it
            s["workspace"] = B.alloc_attention_workspace(c["S"], c["H"], c["Hkv"], c["d"], s["longest"])
        return B.muxq_paged_attention(s["q"], s["k"], s["v"], s["table"], s["lengths"], s["longest"],
                                      k_scale=s.get("k_scale"), v_scale=s.get("v_scale"), out=s["out"],
                                      workspace=s["workspace"])
    if kind == "append":
        q, k, v = _split(s)
        n = s["pages"]
        ks, vs = (s["k_scale"][:n], s["v_scale"][:n]) if c["bits"] == 8 else (None, None)
        kc, vc = s["k"][:n], s["v"][:n]
        B.muxq_kv_append(k, v, s["slots"], kc, vc, k_scale=ks, v_scale=vs, q=q, q_out=s["q_out"],
                         positions=s["positions"], cos_sin=s.get("cos_sin"), interleaved=c["interleaved"])
        if c["bits"] == 16:
            return s["q_out"], kc, vc
        return s["q_out"], *B.muxq_kv_gather(s["slots"], kc, vc, k_scale=ks, v_scale=vs, k_out=s["k_back"],
                                             v_out=s["v_back"])
    if kind == "lora":
        return B.muxq_lora(s["X"], s["A"], s["B"], s["scales"], s["starts"], s["adapter"], s["Y"], out=s["out"])
    if "scratch" not in s:
        s["scratch"] = B.alloc_norm_scratch(c["M"], c["K"])
    y, stream = B.muxq_norm(s["x"], s["weight"], s["bias"], residual=s["residual"], residual_scale=c["residual_scale"],
                            post_weight=s.get("post_weight"), post_bias=s.get("post_bias"), gate=s.get("gate"),
                            kind="rms" if c["root_mean"] else "layer", eps=EPS, out=s["y"], residual_out=s["stream"],
                            slabs=s["maxima"], scratch=s["scratch"])
    return y, stream, s["maxima"][:_maxima_rows(c["M"]), :c["K"]]


def _maxima_rows(M):
    """The maxima come as one row over all tokens; up to 64 tokens as the magnitudes of each."""
    return M if M <= 64 else 1


def _split(s):
    c = s["case"]
    M, H, Hkv, d = c["M"], c["H"], c["Hkv"], c["d"]
    q, k, v = s["qkv"].view(M, H + 2 * Hkv, d).split([H, Hkv, Hkv], 1)
    return q, k, v


def _plain_attend(s):
    c = s["case"]
    S, H, Hkv, d, page = c["S"], c["H"], c["Hkv"], c["d"], c["page"]
    table = s["table"].long()
    n = table.shape[1] * page

    def rows(name):             # [S, Hkv, tokens, d] in 32 bits
        x = s[name][table].float()
        if c["bits"] == 8:
            x = x * s[name + "_scale"][table].unsqueeze(-1)
        return x.transpose(1, 2).reshape(S, Hkv, n, d)

    q = s["q"].float().view(S, Hkv, H // Hkv, d)
    score = torch.matmul(q, rows("k").transpose(2, 3)) / math.sqrt(d)
    there = (torch.arange(n, device=DEV) < s["lengths"][:, None])[:, None, None, :]
    score = score.masked_fill(~there, -math.inf)
    top = score.amax(3, keepdim=True)
    p = torch.exp(score - top.masked_fill(top == -math.inf, 0.0))
    p = p / p.sum(3, keepdim=True).clamp_min(1e-37)
    return torch.matmul(p, rows("v")).view(S, H, d).half()


def _rotate(x, s, cos_sin):
    """The pairs of the first `rotated` dimensions turned by their token's angles."""
    c = s["case"]
    r = c["rotated"]
    if not r:
        return x
    cs = cos_sin[s["positions"].long()].unsqueeze(1)
    cos, sin = cs[..., :r // 2], cs[..., r // 2:]
    if c["interleaved"]:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = x[..., :r // 2], x[..., r // 2:r]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turned, x[..., r:]], -1)


def _plain_append(s):
    c = s["case"]
    q, k, v = _split(s)
    turned = [_rotate(x.float(), s, s.get("cos_sin")) for x in (q, k)] + [v.float()]
    slots = s["slots"].long()
    there = slots >= 0
    pages = torch.where(there, slots // c["page"], s["pages"])
    at = slots % c["page"]
    back = []
    for name, x in (("k", turned[1]), ("v", turned[2])):
        if c["bits"] == 16:
            s[name][pages, :, at] = x.half()
            back.append(s[name][:s["pages"]])
        else:
            most = x.abs().amax(2)
            code = torch.round(x * torch.where(most > 0, 127.0 / most, 0.0).unsqueeze(2)).clamp(-127, 127)
            scale = most / 127.0
            s[name][pages, :, at] = code.to(torch.int8)
            s[name + "_scale"][pages, :, at] = scale
            back.append(torch.where(there[:, None, None], code * scale.unsqueeze(2), 0.0).half())
    return turned[0].half(), *back


def _plain_lora(s):
    M, n, r = s["case"]["M"], s["case"]["adapters"], s["case"]["r"]
    request = torch.bucketize(torch.arange(M, device=DEV), s["starts"][1:-1].long(), right=True)
    mine = s["adapter"][request][:, None] == torch.arange(n, device=DEV)
    factor = mine * s["scales"]                                                      # [M, adapters]
    h = torch.matmul(s["X"].float(), s["A"].float().view(n * r, -1).t()).view(M, n, r) * factor.unsqueeze(2)
    b = s["B"].float().transpose(1, 2).reshape(n * r, -1)
    return (s["Y"].float() + torch.matmul(h.view(M, n * r), b)).half()


def _normed(x, weight, bias, root_mean):
    if not root_mean:
        x = x - x.mean(1, keepdim=True)
    y = x / torch.sqrt((x * x).mean(1, keepdim=True) + EPS) * weight.to(x.dtype)
    return y if bias is None else y + bias.to(x.dtype)


def _norm_of(s, as_type):
    c = s["case"]
    x = s["x"].to(as_type)
    if c["post"]:
        x = _normed(x, s["post_weight"], s["post_bias"], c["root_mean"])
    if c["gate"]:
        x = x * s["gate"].to(as_type)
    stream = c["residual_scale"] * s["residual"].to(as_type) + x
    return _normed(stream, s["weight"], s["bias"], c["root_mean"]), stream


def _plain_norm(s):
    y, stream = _norm_of(s, torch.float32)
    y = y.half()
    size = y.abs()
    return y, stream.half(), size if _maxima_rows(s["case"]["M"]) > 1 else size.amax(0, keepdim=True)


_PLAIN = {"attend": _plain_attend, "append": _plain_append, "lora": _plain_lora, "norm": _plain_norm}


# ---- what a pass cannot do without -----------------------------------------------------------


def work(case):
    kind = case["kind"]
    if kind == "attend":
        lens, H, Hkv, d = _lengths(case), case["H"], case["Hkv"], case["d"]
        token = 2 * Hkv * (d * case["bits"] // 8 + (4 if case["bits"] == 8 else 0))
        pages = sum(-(-n // case["page"]) for n in lens)
        return {"bytes": sum(lens) * token + 4 * case["S"] * H * d + 4 * pages + 4 * case["S"], "flops": 4 * sum(lens) * H * d}
    if kind == "append":
        M, H, Hkv, d = case["M"], case["H"], case["Hkv"], case["d"]
        stored = M - case["padded"]
        if case["bits"] == 16:
            cache = stored * 2 * Hkv * d * 2
        else:       # codes and scales written and read again, the values they stand for written
            cache = stored * 2 * Hkv * 2 * (d + 4) + M * 2 * Hkv * d * 2
        return {"bytes": M * (2 * H + 2 * Hkv) * d * 2 + cache + 8 * M + (M * case["rotated"] * 4),
                "flops": M * (H + Hkv) * case["rotated"] * 3 + M * Hkv * d * 2 + 1}
    if kind == "lora":
        M, K, N, r = case["M"], case["K"], case["N"], case["r"]
        edges = _shares(M, case["requests"])
        rows = sum(b - a for i, (a, b) in enumerate(zip(edges, edges[1:])) if i % 8 != 7)
        used = len({i % case["adapters"] for i in range(case["requests"]) if i % 8 != 7})
        return {"bytes": rows * K * 2 + M * N * 4 + used * r * (K + N) * 2, "flops": 2 * rows * r * (K + N) + 2 * M * N}
    M, K = case["M"], case["K"]
    vectors = (1 if case["root_mean"] else 2) * (2 if case["post"] else 1) + (1 if case["gate"] else 0)
    return {"bytes": 8 * M * K + 2 * vectors * K + 2 * _maxima_rows(M) * K, "flops": (16 if case["post"] else 10) * M * K}


# ---- the same in 64 bits ---------------------------------------------------------------------


def _exact_attend(s):
    c = s["case"]
    d, page, group = c["d"], c["page"], c["H"] // c["Hkv"]
    out = torch.zeros(c["S"], c["H"], d, dtype=torch.float64, device=DEV)
    for i, n in enumerate(s["lengths"].tolist()):
        if n == 0:
            continue
        used = s["table"][i, :-(-n // page)].long()
        for h in range(c["Hkv"]):
            k, v = (s[name][used, h].double().reshape(-1, d)[:n] for name in ("k", "v"))
            if c["bits"] == 8:
                k, v = (x * s[name][used, h].double().reshape(-1)[:n, None] for x, name in ((k, "k_scale"), (v, "v_scale")))
            heads = slice(h * group, (h + 1) * group)
            out[i, heads] = torch.softmax(s["q"][i, heads].double() @ k.t() * d ** -0.5, 1) @ v
    return out


def _exact_append(s):
    c = s["case"]
    q, k, v = (x.double() for x in _split(s))
    r, kept = c["rotated"], s["slots"] >= 0
    if r:
        # each pair as a complex number, turned by e^(i angle)
        pair = torch.complex(*(x.double() for x in s["cos_sin"][s["positions"].long()].split(r // 2, 1)))[:, None]
        first, second = (slice(0, r, 2), slice(1, r, 2)) if c["interleaved"] else (slice(0, r // 2), slice(r // 2, r))
        for x in (q, k):
            turned = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * pair
            x[..., first], x[..., second] = turned.real, turned.imag
    if c["bits"] == 8:
        back = []
        for x in (k, v):
            step = x.abs().amax(2, keepdim=True) / 127.0
            code = torch.where(step > 0, x / step.clamp_min(1e-300), 0.0).round()
            back.append(code * step * kept[:, None, None])
        return q, *back
    caches = []
    for name, x in (("k", k), ("v", v)):
        flat = s[name][:s["pages"]].double().transpose(1, 2).contiguous()      # [pages, tokens, heads, d]
        flat.view(-1, c["Hkv"], c["d"])[s["slots"][kept].long()] = x[kept]
        caches.append(flat.transpose(1, 2))
    return q, *caches


def _exact_lora(s):
    out = s["Y"].double()
    edges = s["starts"].tolist()
    for a, b, i in zip(edges, edges[1:], s["adapter"].tolist()):
        if i >= 0:
            out[a:b] += s["scales"][i].double() * ((s["X"][a:b].double() @ s["A"][i].double().t()) @ s["B"][i].double().t())
    return out


def _exact_norm(s):
    c = s["case"]

    def normed(x, weight, bias):
        if c["root_mean"]:
            z = x * torch.rsqrt(x.square().mean(1, keepdim=True) + EPS)
        else:
            var, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
            z = (x - mean) * torch.rsqrt(var + EPS)
        return z * weight.double() + (0.0 if bias is None else bias.double())

    t = s["x"].double()
    if c["post"]:
        t = normed(t, s["post_weight"], s["post_bias"])
    if c["gate"]:
        t = t * s["gate"].double()
    stream = torch.add(t, s["residual"].double(), alpha=c["residual_scale"])
    y = normed(stream, s["weight"], s["bias"])
    size = y.abs()
    return y, stream, size if _maxima_rows(c["M"]) > 1 else size.max(0, keepdim=True).values


_EXACT = {"attend": _exact_attend, "append": _exact_append, "lora": _exact_lora, "norm": _exact_norm}


def exact(case, seed):
    return _EXACT[case["kind"]](prepare(case, seed))
