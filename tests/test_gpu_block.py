"""The operators between the projections against the same in 64 bits: cache, attention of one new token, adapters, norms."""
import math

import pytest
import torch

from block_common import *

pytestmark = pytest.mark.gpu


# ---- attention of one new token ----------------------------------------------------------------

LENGTHS = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 300, 511, 513, 700]


def _attend_case(seed, lengths, H, heads, d, page, bits, layout="heads", scale=None, gain=1.0, width=None):
    g = gen(seed)
    need = sum(-(-max(n, 0) // page) for n in lengths)
    k, v, ks, vs = make_cache(g, need + 3, heads, page, d, bits, layout)
    table, spare = make_table(g, lengths, page, need + 3, width)
    q = normal(g, len(lengths), H, d) * gain
    say(f"[attend] S={len(lengths)} H={H}/{heads} d={d} page={page} bits={bits} {layout} longest={max(lengths)}")
    scale = d ** -0.5 if scale is None else scale
    got = B.muxq_paged_attention(q, k, v, table, ints(lengths), max(max(lengths), 1), scale=scale, k_scale=ks, v_scale=vs)
    torch.cuda.synchronize()
    want, tol = attend64(q, k, v, ks, vs, table, lengths, scale)
    check(got, want, tol, "attention")
    return got


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("d", [16, 32, 48, 64, 80, 96, 112, 128, 144, 192, 256])
def test_attention_head_sizes_and_lengths(d, bits):
    _attend_case(d, LENGTHS, 6, 3, d, 16, bits)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("H,heads", [(1, 1), (5, 1), (7, 7), (16, 1), (17, 1), (14, 2), (40, 2), (71, 1), (24, 3), (32, 8)])
def test_attention_shared_heads(H, heads, bits):
    _attend_case(H, [0, 1, 40, 333, 600], H, heads, 64, 16, bits, "tokens")


@pytest.mark.parametrize("layout", ["heads", "tokens"])
@pytest.mark.parametrize("page", [8, 16, 32, 64, 128, 256])
def test_attention_pages(page, layout):
    _attend_case(page, LENGTHS, 4, 2, 64, page, 16, layout)
    _attend_case(page + 1, LENGTHS, 4, 2, 128, page, 8, layout)


@pytest.mark.parametrize("lengths,H,heads,d,bits", [
    ([5000], 8, 8, 64, 16), ([20011], 32, 8, 128, 16), ([33333], 4, 1, 80, 8), ([70001, 3, 0, 1025], 4, 2, 128, 8),
    ([1, 9000, 1, 1], 2, 2, 64, 16), ([2048] * 40, 20, 20, 64, 16), ([1000, 30] * 100, 4, 4, 64, 8), ([0, 0], 4, 4, 64, 16)])
def test_attention_long_and_many(lengths, H, heads, d, bits):
    _attend_case(len(lengths), lengths, H, heads, d, 16, bits)


@pytest.mark.parametrize("seed", range(6))
def test_attention_shares_cut_anywhere(seed):
    # ragged lengths, idle places and very short sequences among long ones: shares end in every part of a sequence
    g = gen(100 + seed)
    S = [3, 17, 40, 64, 100, 5][seed]
    lengths = (torch.rand(S, generator=g, device=DEV) ** 3 * [9000, 6000, 4000, 3000, 2600, 30000][seed]).int().tolist()
    lengths[S // 2], lengths[-1] = 0, [9000, 6000, 4000, 3000, 2600, 30000][seed]
    H, heads, d = [(4, 4, 64), (16, 2, 64), (3, 3, 128), (8, 1, 80), (2, 2, 64), (18, 1, 256)][seed]
    _attend_case(seed, lengths, H, heads, d, 16, 8 if seed % 2 else 16)


def test_attention_with_a_bound_far_above_the_lengths():
    # the work is planned by the bound: shares with fewer steps than workgroups, most of them none
    g = gen(12)
    lengths = [5, 0, 300, 17]
    k, v, _, _ = make_cache(g, 40, 2, 16, 64, 16)
    table, _ = make_table(g, lengths, 16, 40, width=2000)
    q = normal(g, 4, 4, 64)
    say("[attend] bound of 32000 for 300 tokens")
    got = B.muxq_paged_attention(q, k, v, table, ints(lengths), 32000)
    none = B.muxq_paged_attention(q, k, v, table, ints([0, -3, 0, 0]), 32000)
    torch.cuda.synchronize()
    want, tol = attend64(q, k, v, None, None, table, lengths, 0.125)
    check(got, want, tol, "attention")
    assert (none == 0).all()


@pytest.mark.parametrize("bits", [16, 8])
def test_attention_sharp_and_flat_scores(bits):
    _attend_case(1, [1, 50, 3000], 4, 4, 64, 16, bits, gain=30.0)          # nearly one-hot
    _attend_case(2, [1, 50, 3000], 4, 4, 64, 16, bits, scale=0.0)          # a plain mean
    _attend_case(3, [1, 50, 3000], 4, 4, 64, 16, bits, scale=-0.3)
    _attend_case(4, [7, 50, 9000], 8, 2, 128, 16, bits, gain=1e-3)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("lengths", [[1, 17, 40, 0, 63], [2000, 5, 1234, 0, 4099]])
def test_attention_ignores_what_lies_beyond_a_sequence(lengths, bits):
    g = gen(5)
    page, d, heads, H = 16, 64, 2, 4
    n_pages = sum(-(-n // page) for n in lengths) + 4
    k, v, ks, vs = make_cache(g, n_pages, heads, page, d, bits)
    table, spare = make_table(g, lengths, page, n_pages, unused=spare_page(lengths, page, g, n_pages))
    q = normal(g, len(lengths), H, d)
    want, tol = attend64(q, k, v, ks, vs, table, lengths, 0.125)
    dirty = torch.ones(n_pages, page, dtype=torch.bool, device=DEV)
    for s, n in enumerate(lengths):
        for i in range(-(-n // page)):
            dirty[table[s, i].long(), :min(page, n - i * page)] = False
    for x, bad in ((k, math.nan), (v, math.inf)) if bits == 16 else ((ks, math.nan), (vs, math.inf)):
        x.transpose(1, 2)[dirty] = bad
    say(f"[attend] NaN and infinity beyond lengths {lengths} bits={bits}")
    got = B.muxq_paged_attention(q, k, v, table, ints(lengths), max(lengths), scale=0.125, k_scale=ks, v_scale=vs)
    torch.cuda.synchronize()
    check(got, want, tol, "attention")


def spare_page(lengths, page, g, n_pages):
    return n_pages - 1


def test_attention_masks_pages_outside_the_cache_and_clamps_lengths():
    g = gen(6)
    page, d, H = 16, 64, 3
    lengths = [200, 200, 16, 900, -5, 200]
    k, v, _, _ = make_cache(g, 120, H, page, d, 16)
    table, _ = make_table(g, lengths, page, 120, width=64)
    table[0, 2] = -1
    table[0, 11] = 120
    table[1, 0] = 1 << 30
    table[2, :] = -7                      # nothing is left of this one
    table[5, :13] = table[5, 0]           # one page again and again
    q = normal(g, len(lengths), H, d)
    say("[attend] pages outside the cache")
    got = B.muxq_paged_attention(q, k, v, table, ints(lengths), 500)
    torch.cuda.synchronize()
    want, tol = attend64(q, k, v, None, None, table, [min(n, 500) for n in lengths], d ** -0.5)
    check(got, want, tol, "attention")
    assert (got[2] == 0).all() and (got[4] == 0).all()


def test_attention_strides_places_and_streams():
    g = gen(7)
    page, d, H, heads = 32, 64, 6, 2
    lengths = [70, 1, 129, 515]
    big = normal(g, 40, heads, 2, page, 2 * d)          # keys and values side by side, tokens apart
    k, v = big[:, :, 0, :, :d], big[:, :, 1, :, d:]
    table, _ = make_table(g, lengths, page, 40, width=31)
    wide = normal(g, 4, 3, H, d)
    q = wide[:, 1]
    out = torch.zeros(4, 2, H, d, dtype=torch.float16, device=DEV)
    say("[attend] strided, another stream")
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        B.muxq_paged_attention(q, k, v, table, ints(lengths), 600, out=out[:, 1])
    side.synchronize()
    want, tol = attend64(q, k, v, None, None, table, lengths, d ** -0.5)
    check(out[:, 1], want, tol, "attention")
    assert (out[:, 0] == 0).all()


def test_attention_gives_the_same_bits_twice_and_keeps_off_its_neighbours():
    g = gen(8)
    lengths = [3000, 17, 0, 9999, 4096]
    k, v, ks, vs = make_cache(g, 1100, 4, 16, 128, 8)
    table, _ = make_table(g, lengths, 16, 1100)
    q = normal(g, 5, 16, 128)
    ws = B.alloc_attention_workspace(5, 16, 4, 128, 9999)
    say("[attend] twice")
    outs = []
    for fill in (0, 255):
        if ws is not None:
            ws.fill_(fill)
        room = torch.full((7, 16, 128), 3.0, dtype=torch.float16, device=DEV)
        B.muxq_paged_attention(q, k, v, table, ints(lengths), 9999, k_scale=ks, v_scale=vs, out=room[1:6], workspace=ws)
        torch.cuda.synchronize()
        assert (room[0] == 3).all() and (room[6] == 3).all()
        outs.append(room)
    assert torch.equal(*outs)


def test_attention_in_a_cache_beyond_32_bits():
    # keys and values of 5 GiB each; the pages in use lie at both ends
    g = gen(9)
    page, heads, d = 16, 8, 128
    n_pages = (5 << 30) // (page * heads * d * 2)
    k, v, _, _ = B.alloc_kv_cache(n_pages, page, heads, d)
    lengths = [100, 333]
    pages = list(range(n_pages - 20, n_pages)) + list(range(10))
    for x in (k, v):
        x[n_pages - 20:] = normal(g, 20, heads, page, d)
        x[:10] = normal(g, 10, heads, page, d)
    table = ints([pages[:7] + [0] * 14, pages[7:28]])
    q = normal(g, 2, 16, d)
    say("[attend] cache of 2 x 5 GiB")
    got = B.muxq_paged_attention(q, k, v, table, ints(lengths), 333)
    torch.cuda.synchronize()
    want, tol = attend64(q, k, v, None, None, table, lengths, d ** -0.5)       # before the append below
    slots = ints([(n_pages - 1) * page + 3, 5])
    kk, vv = B.muxq_kv_gather(slots, k, v)
    B.muxq_kv_append(kk[:1], vv[:1], ints([(n_pages - 1) * page + 15]), k, v)
    torch.cuda.synchronize()
    check(got, want, tol, "attention")
    assert torch.equal(kk[0], k[n_pages - 1, :, 3]) and torch.equal(vv[1], v[0, :, 5])
    assert torch.equal(k[n_pages - 1, :, 15], kk[0]) and torch.equal(v[n_pages - 1, :, 15], vv[0])


# ---- cache ---------------------------------------------------------------------------------------


def _append_case(seed, M, H, heads, d, page, bits, rot, interleaved, layout="heads", in_place=False, gain=1.0):
    g = gen(seed)
    n_pages = -(-M // page) + 3
    n_pos = 50
    qkv = normal(g, M, (H + 2 * heads) * d) * gain
    q, k, v = qkv.view(M, H + 2 * heads, d).split([H, heads, heads], 1)
    kc, vc, ks, vs = make_cache(g, n_pages, heads, page, d, bits, layout)
    slots = torch.randperm(n_pages * page, generator=g, device=DEV)[:M].int()
    positions = torch.randint(0, n_pos, (M,), generator=g, device=DEV).int()
    lost = []
    if M > 6:
        slots[1], slots[2], slots[3] = -1, n_pages * page, -(1 << 31)
        lost = [1, 2, 3]
        if rot:
            positions[4], positions[5] = -1, n_pos
            lost += [4, 5]
    cos_sin = None
    if rot:
        angle = torch.rand(n_pos, rot // 2, generator=g, device=DEV) * 7 - 3
        cos_sin = torch.cat([angle.cos(), angle.sin()], 1).contiguous()
    want = [x.double() for x in (q, k, v)]
    if rot:
        stay = [4, 5] if M > 6 else []
        safe = positions.clone()
        safe[stay] = 0
        for i in (0, 1):
            turned = rotate64(want[i], cos_sin, safe, interleaved)
            turned[stay] = want[i][stay]
            want[i] = turned
    room = 4 * U32 * qkv.double().view(M, -1, d).abs().amax(2, keepdim=True)
    room_q, room_k, _ = room.split([H, heads, heads], 1)
    before = [x.clone() for x in (kc, vc)] + ([ks.clone(), vs.clone()] if bits == 8 else [])
    say(f"[append] M={M} H={H}/{heads} d={d} page={page} bits={bits} rot={rot} {interleaved} {layout}")
    q_in = q.clone()
    q_out = B.muxq_kv_append(k, v, slots, kc, vc, k_scale=ks, v_scale=vs, q=q, q_out=q if in_place else None,
                             positions=positions if rot else None, cos_sin=cos_sin, interleaved=interleaved)
    back = B.muxq_kv_gather(slots, kc, vc, k_scale=ks, v_scale=vs)
    torch.cuda.synchronize()
    if not in_place:
        assert torch.equal(q, q_in)
    check(q_out, want[0], U16 * want[0].abs() + TINY16 + room_q, "queries")
    kept = torch.ones(M, dtype=torch.bool, device=DEV)
    kept[lost] = False
    for got, w, r in zip(back, want[1:], (room_k, torch.zeros_like(room_k))):
        outside = [i for i in lost if i < 4]
        assert (got[outside] == 0).all()
        if bits == 16:
            tol = U16 * w.abs() + TINY16 + r
        else:
            step = w.abs().amax(2, keepdim=True) / 127
            tol = step * 0.501 + r + U16 * w.abs() * 1.01 + TINY16
        check(got[kept], w[kept], tol[kept], "cache")
    # codes and scales by themselves, and nothing else in the cache moved
    rows = slots[kept].long()
    for x, x0 in zip((kc, vc), before):
        flat, flat0 = (y.transpose(1, 2).reshape(-1, heads, d) for y in (x, x0))
        flat0 = flat0.clone()
        if bits == 8:
            assert (flat[rows].abs().amax(2) <= 127).all() and (flat[rows].int().abs().amax(2) >= 126).all()
        flat0[rows] = flat[rows]
        assert torch.equal(flat, flat0)
    for x, x0, w in zip((ks, vs), before[2:], want[1:]):
        flat, flat0 = (y.transpose(1, 2).reshape(-1, heads) for y in (x, x0))
        top = w.abs().amax(2)[kept] / 127
        assert ((flat[rows].double() - top).abs() <= 8 * U32 * top + 1e-12).all()
        flat0 = flat0.clone()
        flat0[rows] = flat[rows]
        assert torch.equal(flat, flat0)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,rot", [(16, 8), (32, 32), (48, 16), (64, 64), (64, 0), (80, 40), (96, 96), (112, 56), (128, 128), (128, 64),
                                   (160, 8), (256, 256), (256, 120)])
def test_append_head_sizes_and_rotations(d, rot, interleaved, bits):
    _append_case(d + rot, 37, 5, 2, d, 16, bits, rot, interleaved)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("M,H,heads,page,layout", [(1, 1, 1, 8, "heads"), (2, 12, 12, 16, "tokens"), (65, 8, 1, 64, "tokens"),
                                                    (1000, 4, 4, 256, "heads"), (3001, 3, 3, 32, "tokens")])
def test_append_tokens_and_layouts(M, H, heads, page, layout, bits):
    _append_case(M, M, H, heads, 64, page, bits, 32, False, layout)
    _append_case(M + 1, M, H, heads, 80, page, bits, 80, True, layout, in_place=True)


def test_append_of_zeros_and_large_values():
    g = gen(3)
    kc, vc, ks, vs = make_cache(g, 2, 2, 16, 64, 8)
    k = torch.zeros(3, 2, 64, dtype=torch.float16, device=DEV)
    k[1] = 65504.0
    k[2, 0, 5] = 6e-8
    say("[append] zeros, the largest and the smallest values")
    B.muxq_kv_append(k, k, ints([0, 17, 30]), kc, vc, k_scale=ks, v_scale=vs)
    torch.cuda.synchronize()
    assert (kc[0, :, 0] == 0).all() and (ks[0, :, 0] == 0).all()
    assert (kc[1, :, 1] == 127).all() and kc[1, 0, 14, 5] == 127 and (kc[1, 1, 14] == 0).all()
    back, _ = B.muxq_kv_gather(ints([0, 17, 30]), kc, vc, k_scale=ks, v_scale=vs)
    torch.cuda.synchronize()
    assert torch.equal(back, k)
    # NaN and infinity: unspecified codes, no fault, and neighbours keep theirs
    k[1, 0, 3], k[1, 1, 7] = math.nan, math.inf
    before = kc.clone()
    B.muxq_kv_append(k[1:2], k[1:2], ints([20]), kc, vc, k_scale=ks, v_scale=vs)
    torch.cuda.synchronize()
    before[1, :, 4] = kc[1, :, 4]
    assert torch.equal(before, kc)


def test_append_without_queries_on_another_stream():
    g = gen(4)
    kc, vc, _, _ = make_cache(g, 4, 2, 16, 64, 16)
    k, v = normal(g, 9, 2, 64), normal(g, 9, 2, 64)
    slots = ints(list(range(40, 49)))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        assert B.muxq_kv_append(k, v, slots, kc, vc) is None
    side.synchronize()
    assert torch.equal(kc.transpose(1, 2).reshape(-1, 2, 64)[40:49], k)
    assert torch.equal(vc.transpose(1, 2).reshape(-1, 2, 64)[40:49], v)


# ---- adapters --------------------------------------------------------------------------------------


def _lora_case(seed, starts, adapters, K, N, r, n, in_place=False, pad=0, gain=1.0, factor=1.0):
    g = gen(seed)
    M = starts[-1]
    X = normal(g, M, K + pad)[:, :K]
    X[:, ::37] *= 40
    Y = normal(g, M, N + pad)[:, :N]
    A = (normal(g, n, r, K, dtype=torch.float32) * gain / math.sqrt(K)).half()
    Bm = (normal(g, n, N, r, dtype=torch.float32) / math.sqrt(r)).half()
    scales = (torch.rand(n, generator=g, device=DEV) * 3 - 1) * factor
    want, tol = lora64(X, A, Bm, scales, starts, adapters, Y)
    say(f"[lora] M={M} K={K} N={N} r={r} adapters={n} requests={len(adapters)} pad={pad}")
    out = Y if in_place else None
    got = B.muxq_lora(X, A, Bm, scales, ints(starts), ints(adapters), Y, out=out)
    torch.cuda.synchronize()
    assert (got.data_ptr() == Y.data_ptr()) == in_place
    beyond = want.abs() >= 65520.0              # infinity in fp16
    assert torch.equal(got[beyond].double(), torch.copysign(torch.full_like(want, math.inf), want)[beyond])
    check(got[~beyond], want[~beyond], tol[~beyond], "adapters")
    plain = [i for i, a in enumerate(adapters) if not 0 <= a < n]
    if not in_place:
        for i in plain:
            assert torch.equal(got[starts[i]:starts[i + 1]], Y[starts[i]:starts[i + 1]])


@pytest.mark.parametrize("r", [8, 16, 24, 32, 40, 64, 72, 96, 128])
def test_lora_ranks(r):
    _lora_case(r, [0, 1, 2, 40, 40, 77], [2, -1, 0, 1, 1], 264, 328, r, 3)
    _lora_case(r + 1, [0, 5], [0], 768, 136, r, 1, in_place=True, pad=8)


@pytest.mark.parametrize("K,N", [(8, 8), (8, 2304), (16, 40), (768, 8), (1000, 1016), (1280, 3840), (4096, 512), (8200, 264), (31, 33)])
def test_lora_shapes(K, N):
    K, N = (K + 7) // 8 * 8, (N + 7) // 8 * 8
    _lora_case(K, [0, 1, 18, 19], [1, 0, 7], K, N, 16, 2)
    _lora_case(N, [0, 130, 131, 257], [1, 0, 1], K, N, 8, 2, pad=16)


def test_lora_single_tokens_of_many_requests():
    g = gen(1)
    for M in (1, 2, 15, 16, 17, 64, 200):
        adapters = torch.randint(-1, 9, (M,), generator=g, device=DEV).tolist()
        _lora_case(M, list(range(M + 1)), adapters, 512, 768, 16, 9)


def test_lora_prompts_and_empty_requests():
    _lora_case(1, [0, 0, 0, 700, 700, 1500, 1501, 2000, 2000], [0, 1, 2, 0, 1, 5, -1, 2], 520, 392, 32, 3)
    _lora_case(2, [0, 3000], [1], 768, 768, 64, 2, in_place=True)
    _lora_case(3, [0, 1, 4097], [-1, 0], 256, 1032, 16, 1)


def test_lora_sums_beyond_fp16():
    # X A^T beyond 65504 and far below fp16's smallest: the products in between are not fp16 values
    _lora_case(5, [0, 3, 20], [0, 1], 512, 128, 16, 2, gain=3e4)
    _lora_case(7, [0, 3, 20], [0, 1], 512, 128, 16, 2, gain=3e4, factor=1e-4)
    _lora_case(6, [0, 3, 20], [0, 1], 512, 128, 16, 2, gain=2e-3)


def test_lora_rows_outside_requests_are_not_written():
    g = gen(2)
    X, Y = normal(g, 40, 64), normal(g, 40, 64)
    A, Bm, scales = normal(g, 1, 8, 64), normal(g, 1, 64, 8), torch.ones(1, device=DEV)
    out = torch.full_like(Y, 5.0)
    say("[lora] rows outside, bounds outside")
    B.muxq_lora(X, A, Bm, scales, ints([3, 10, 30]), ints([0, -1]), Y, out=out)
    torch.cuda.synchronize()
    assert (out[:3] == 5).all() and (out[30:] == 5).all() and torch.equal(out[10:30], Y[10:30])
    want, tol = lora64(X, A, Bm, scales, [3, 10], [0], Y)
    check(out[3:10], want[3:10], tol[3:10], "adapters")
    out.fill_(5.0)
    B.muxq_lora(X, A, Bm, scales, ints([-9, 10, 4000]), ints([0, 0]), Y, out=out)
    torch.cuda.synchronize()
    want, tol = lora64(X, A, Bm, scales, [0, 40], [0], Y)
    check(out, want, tol, "adapters")


# ---- norms ------------------------------------------------------------------------------------------


def _norm_case(seed, M, K, kind, *, residual=True, post=False, gate=None, bias=True, scale=1.0, offset=0.0, slabs=True,
               in_place=None, pad=0, eps=1e-5):
    g = gen(seed)
    x = (normal(g, M, K + pad, dtype=torch.float32) + offset).half()[:, :K]
    res = normal(g, M, K + pad)[:, :K] * 3 if residual else None
    w, b = normal(g, K) * 0.2 + 1, normal(g, K) if bias else None
    pw, pb = (normal(g, K) * 0.2 + 1, normal(g, K) if bias else None) if post else (None, None)
    gt = normal(g, *{"channel": (K,), "token": (M, K)}[gate]) if gate else None
    t, room = x.double(), torch.zeros(M, K, dtype=torch.float64, device=DEV)
    if post:
        t, move = norm64(t, pw, pb, kind, eps)
        room = 2.0 ** -18 * move + 4 * U32 * t.abs()
    if gate:
        t, room = t * gt.double(), room * gt.double().abs()
    if residual:
        t = scale * res.double() + t
        room = room + 4 * U32 * ((scale * res.double()).abs() + t.abs())
    y, move = norm64(t, w, b, kind, eps)
    shift = room.amax(1, keepdim=True) / t.abs().amax(1, keepdim=True).clamp_min(1e-30)
    tol_y = U16 * y.abs() + TINY16 + 4 * U32 * y.abs() + (2.0 ** -18 + 2 * shift) * move
    tol_r = U16 * t.abs() + TINY16 + room
    say(f"[norm] M={M} K={K} {kind} residual={residual} post={post} gate={gate} slabs={slabs} pad={pad} {in_place}")
    lay = B.workspace_layout(M, K, 64, 64)
    ws = torch.full((lay.total,), 0x7f, dtype=torch.uint8, device=DEV) if slabs else None
    outs = {"out": x} if in_place == "x" else {"out": x, "residual_out": res} if in_place == "both" else {}
    got, stream = B.muxq_norm(x, w, b, residual=res, residual_scale=scale, post_weight=pw, post_bias=pb, gate=gt, kind=kind,
                              eps=eps, slabs=ws[lay.absmax_partial:] if slabs else None, **outs)
    torch.cuda.synchronize()
    check(got, y, tol_y, "norm")
    if stream is not None:
        check(stream, t, tol_r, "stream")
    else:
        assert not (residual or gate or post)
    if slabs:
        n = B.norm_slabs(M, K)
        rows = ws[lay.absmax_partial:][:n * lay.k_pad * 2].view(torch.float16).view(n, lay.k_pad)
        assert torch.equal(rows[:, :K].amax(0), got.abs().amax(0)) and (rows[:, K:] == 0).all()
        after = ws[lay.absmax_partial + n * lay.k_pad * 2:]
        assert (after == 0x7f).all()
    return got


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("K", [8, 16, 72, 128, 200, 512, 520, 768, 1024, 1032, 1280, 1600, 2048, 2056, 4096, 5120, 8192, 8200, 12288, 16384,
                               16392, 32768])
def test_norm_widths(K, kind):
    _norm_case(K, 5, K, kind)
    _norm_case(K + 1, 67, K, kind, post=True, gate="channel", scale=0.5)


@pytest.mark.parametrize("M", [1, 2, 3, 8, 63, 64, 65, 100, 255, 256, 257, 1000, 4099])
def test_norm_tokens(M):
    _norm_case(M, M, 768, "layer")
    _norm_case(M + 1, M, 264, "rms", post=True, gate="token", bias=False)


@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_norm_parts(kind):
    for residual in (False, True):
        for post in (False, True):
            for gate in (None, "channel", "token"):
                _norm_case(1, 70, 328, kind, residual=residual, post=post, gate=gate, scale=-1.5, pad=8, slabs=gate is None)


def test_norm_in_place_and_without_maxima():
    _norm_case(1, 300, 1280, "layer", in_place="x")
    _norm_case(2, 300, 1280, "rms", in_place="both", post=True, gate="channel")
    _norm_case(3, 9, 4104, "layer", in_place="both", slabs=False, pad=24)


def test_norm_rows_far_from_zero():
    _norm_case(1, 70, 1024, "layer", offset=200.0, residual=False)
    _norm_case(2, 70, 1024, "layer", offset=-30.0, post=True)


def test_norm_of_constant_rows():
    x = torch.full((3, 64), 2.5, dtype=torch.float16, device=DEV)
    x[1] = 0
    w, b = torch.ones(64, dtype=torch.float16, device=DEV), torch.full((64,), 0.5, dtype=torch.float16, device=DEV)
    say("[norm] constant rows")
    y, _ = B.muxq_norm(x, w, b)
    z, _ = B.muxq_norm(x[1:2], w, b, kind="rms")
    torch.cuda.synchronize()
    assert (y == 0.5).all() and (z == 0.5).all()


@pytest.mark.parametrize("M,K,N", [(1, 768, 768), (24, 1280, 256), (300, 768, 512), (3000, 1024, 256)])
@pytest.mark.parametrize("x_gran", ["tensor", "token"])
def test_norm_hands_the_maxima_to_the_next_layer(M, K, N, x_gran):
    g = gen(M)
    x, res = normal(g, M, K), normal(g, M, K) * 2
    x[:, 5] *= 60
    w, b = torch.ones(K, dtype=torch.float16, device=DEV), torch.zeros(K, dtype=torch.float16, device=DEV)
    w[7], w[K - 1] = 9.0, 12.0                      # outlier channels behind the norm
    w_q, w_scale = B.muxq_quantize_weight(normal(g, K, N) * 0.02)
    ws, lay = B.alloc_workspace(M, K, N, 64), B.workspace_layout(M, K, N, 64)
    ws.fill_(0x7f)
    say(f"[norm] hand-over M={M} K={K} N={N} {x_gran}")
    y, _ = B.muxq_norm(x, w, b, residual=res, slabs=ws[lay.absmax_partial:])
    got = B.muxq_linear(y, w_q, w_scale, N, workspace=ws, x_gran=x_gran, absmax_ready=True, absmax_slabs=B.norm_slabs(M, K))
    want = B.muxq_linear(y, w_q, w_scale, N, x_gran=x_gran)
    torch.cuda.synchronize()
    assert torch.equal(got, want)


# ---- together ------------------------------------------------------------------------------------


def test_step_in_a_graph():
    # append, attention, adapters and norm captured once and replayed with new contents
    g = gen(11)
    S, H, heads, d, page, n_pages = 5, 4, 2, 64, 16, 200
    K = H * d
    kc, vc, ks, vs = make_cache(g, n_pages, heads, page, d, 8)
    table, _ = make_table(g, [600] * S, page, n_pages)
    qkv = normal(g, S, (H + 2 * heads) * d)
    q, k, v = qkv.view(S, -1, d).split([H, heads, heads], 1)
    lengths, slots = ints([1] * S), ints([-1] * S)
    positions = ints([0] * S)
    angle = torch.rand(600, d // 2, generator=g, device=DEV)
    cos_sin = torch.cat([angle.cos(), angle.sin()], 1).contiguous()
    q_out, o = torch.empty(S, H, d, dtype=torch.float16, device=DEV), torch.empty(S, H, d, dtype=torch.float16, device=DEV)
    ws = B.alloc_attention_workspace(S, H, heads, d, 600)
    A, Bm, scales = normal(g, 3, 8, K) * 0.1, normal(g, 3, K, 8), torch.ones(3, device=DEV)
    starts, adapters = ints(list(range(S + 1))), ints([0, 1, -1, 2, 1])
    res, w = normal(g, S, K), torch.ones(K, dtype=torch.float16, device=DEV)
    out, y, stream = (torch.empty(S, K, dtype=torch.float16, device=DEV) for _ in range(3))

    def step(into):
        B.muxq_kv_append(k, v, slots, kc, vc, k_scale=ks, v_scale=vs, q=q, q_out=q_out, positions=positions, cos_sin=cos_sin)
        B.muxq_paged_attention(q_out, kc, vc, table, lengths, 600, k_scale=ks, v_scale=vs, out=o, workspace=ws)
        B.muxq_lora(o.view(S, K), A, Bm, scales, starts, adapters, qkv[:, :K], out=into)
        B.muxq_norm(into, w, residual=res, kind="rms", out=y, residual_out=stream)

    say("[graph] eager, capture, replays")
    step(out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            step(out)
    torch.cuda.synchronize()
    for i, lens in enumerate(([1, 2, 3, 4, 5], [600, 17, 0, 256, 257], [300, 599, 1, 33, 32])):
        qkv.copy_(normal(g, S, qkv.shape[1]))
        lengths.copy_(ints(lens))
        positions.copy_(ints([max(n - 1, 0) for n in lens]))
        at = [slots_of(table[s].tolist(), [n - 1], page)[0] if n else -1 for s, n in enumerate(lens)]
        slots.copy_(ints(at))
        graph.replay()
        torch.cuda.synchronize()
        first = [t.clone() for t in (q_out, o, out, y, stream, kc, ks)]
        step(out)
        torch.cuda.synchronize()
        for a, b in zip(first, (q_out, o, out, y, stream, kc, ks)):
            assert torch.equal(a, b), f"replay {i}"
        want, tol = attend64(q_out, kc, vc, ks, vs, table, lens, d ** -0.5)
        check(o, want, tol, "attention in a graph")


# ---- refusals of the binding ---------------------------------------------------------------------


def test_bindings_refuse_tensors_that_do_not_fit():
    g = gen(1)
    kc, vc, ks, vs = make_cache(g, 4, 2, 16, 64, 8)
    kh, vh, _, _ = make_cache(g, 4, 2, 16, 64, 16)
    k, q, slots = normal(g, 3, 2, 64), normal(g, 3, 4, 64), ints([0, 1, 2])
    table, lengths = ints([[0, 1]] * 3), ints([5, 6, 7])
    X, Y, A, Bm = normal(g, 5, 64), normal(g, 5, 32), normal(g, 2, 8, 64), normal(g, 2, 32, 8)
    scales, starts, adapters = torch.ones(2, device=DEV), ints([0, 2, 5]), ints([0, 1])
    w = normal(g, 64)
    say("[refuse] through the binding")
    bad = [
        lambda: B.muxq_kv_append(k.float(), k, slots, kh, vh), lambda: B.muxq_kv_append(k, k, slots.long(), kh, vh),
        lambda: B.muxq_kv_append(k, k, slots[:2], kh, vh), lambda: B.muxq_kv_append(k, k[:, :1], slots, kh, vh),
        lambda: B.muxq_kv_append(k.cpu(), k, slots, kh, vh), lambda: B.muxq_kv_append(k, k, slots, kh, vh[:3]),
        lambda: B.muxq_kv_append(k, k, slots, kc, vc), lambda: B.muxq_kv_append(k, k, slots, kh, vh, k_scale=ks, v_scale=vs),
        lambda: B.muxq_kv_append(k, k, slots, kc, vc, k_scale=ks[:2], v_scale=vs), lambda: B.muxq_kv_append(k, k, slots, kh.float(), vh.float()),
        lambda: B.muxq_kv_append(k, k, slots, kh, vh, q=q[:2]), lambda: B.muxq_kv_append(k, k, slots, kh, vh, q=q.float()),
        lambda: B.muxq_kv_append(k, k, slots, kh, vh, cos_sin=torch.ones(9, 64, device=DEV)),
        lambda: B.muxq_kv_append(k, k, slots, kh, vh, cos_sin=torch.ones(9, 64, device=DEV).half(), positions=slots),
        lambda: B.muxq_kv_append(k, k, slots, kh.transpose(2, 3), vh.transpose(2, 3)),
        lambda: B.muxq_kv_gather(slots, kh, vh, k_out=k[:2]), lambda: B.muxq_kv_gather(slots.float(), kh, vh),
        lambda: B.muxq_paged_attention(q[:, :3], kh, vh, table, lengths, 32), lambda: B.muxq_paged_attention(q, kh, vh, table, lengths, 33),
        lambda: B.muxq_paged_attention(q, kh, vh, table[:2], lengths, 32), lambda: B.muxq_paged_attention(q, kh, vh, table, lengths[:2], 32),
        lambda: B.muxq_paged_attention(q, kh, vh, table.long(), lengths, 32), lambda: B.muxq_paged_attention(q.cpu(), kh, vh, table, lengths, 32),
        lambda: B.muxq_paged_attention(q, kh, vh, table, lengths, 32, out=q[:2]), lambda: B.muxq_paged_attention(q, kh, vh, table, lengths, 0),
        lambda: B.muxq_lora(X, A, Bm, scales, starts, adapters, Y.float()), lambda: B.muxq_lora(X, A[:1], Bm, scales, starts, adapters, Y),
        lambda: B.muxq_lora(X, A, Bm, scales, starts[:2], adapters, Y), lambda: B.muxq_lora(X, A, Bm.transpose(1, 2), scales, starts, adapters, Y),
        lambda: B.muxq_lora(X[:, :56], A, Bm, scales, starts, adapters, Y), lambda: B.muxq_lora(X, A, Bm, scales.half(), starts, adapters, Y),
        lambda: B.muxq_lora(X, A, Bm, scales, starts, adapters, Y, out=Y[:4]),
        lambda: B.muxq_norm(X, w[:32]), lambda: B.muxq_norm(X, w.float()), lambda: B.muxq_norm(X, w, residual=X[:3]),
        lambda: B.muxq_norm(X, w, gate=w[:8]), lambda: B.muxq_norm(X, w, post_bias=w), lambda: B.muxq_norm(X.t(), w),
        lambda: B.muxq_norm(X, w, slabs=torch.empty(64, dtype=torch.uint8, device=DEV)), lambda: B.muxq_norm(X, w, out=X[:2]),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(B.MuxqError):
            call()
            pytest.fail(f"call {i} was accepted")
    torch.cuda.synchronize()


@pytest.mark.parametrize("M,K,N,r", [(2000, 800, 328, 16), (900, 1752, 264, 24), (700, 2304, 136, 32), (420, 4104, 520, 40), (1100, 1608, 200, 64),
                                     (450, 3592, 72, 72), (3000, 600, 1000, 8)])
def test_lora_prompts_on_either_side_of_the_rows_and_launches(M, K, N, r):
    # tiles of 32 and of 16 rows, one launch and two, ragged ends in rows, channels and ranks
    _lora_case(M, [0, 1, 34, 34, M // 2 + 3, M - 5, M], [1, 0, 1, -1, 2, 0], K, N, r, 3)
    _lora_case(M + 1, [0, M], [0], K, N, r, 1, in_place=True, pad=8)


@pytest.mark.parametrize("requests", [510, 511, 512, 513, 1023, 1025, 3000])
def test_lora_many_requests(requests):
    # runs of 0 to 3 rows: the request of a tile is found among few, or in two rounds among many
    g = gen(requests)
    lengths = torch.randint(0, 4, (requests,), generator=g, device=DEV).tolist()
    starts = [0]
    for n in lengths:
        starts.append(starts[-1] + n)
    adapters = torch.randint(-1, 5, (requests,), generator=g, device=DEV).tolist()
    _lora_case(requests, starts, adapters, 64, 72, 8, 5)
