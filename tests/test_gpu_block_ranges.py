"""The operators between the projections at sizes where a kernel goes round once more: many heads and tokens to a lane, many rows of
a norm to a workgroup, shares longer than the page offsets that stand in LDS, hundreds and thousands of sequences."""
import pytest
import torch

from block_common import *
from test_gpu_block import _append_case, _norm_case

pytestmark = pytest.mark.gpu


# ---- cache: four heads to a lane from 2^18 lanes of one head on --------------------------------------------


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("M,H,heads,d,page,rot,interleaved,in_place,layout", [
    (9001, 5, 2, 80, 16, 80, False, False, "heads"),        # 9 heads: the last round has one
    (9001, 5, 2, 80, 32, 40, False, True, "tokens"),        # halves of 20: runs of 4
    (9000, 4, 3, 128, 64, 128, True, True, "heads"),        # 10 heads, interleaved pairs
    (9000, 4, 3, 64, 8, 24, True, False, "tokens"),
    (7000, 1, 5, 96, 256, 0, False, False, "heads"),        # 11 heads, no rotation
    (7000, 3, 1, 256, 16, 56, False, True, "heads"),        # one round and one head more
    (4097, 8, 4, 64, 16, 64, False, False, "heads"),        # just beyond the line, and just before it
    (4096, 8, 4, 64, 16, 64, False, False, "heads")])
def test_append_of_prompts(M, H, heads, d, page, rot, interleaved, in_place, layout, bits):
    _append_case(M + d, M, H, heads, d, page, bits, rot, interleaved, layout, in_place)


# ---- norms: more rows than workgroups, so that maxima and buffers of the sums go on from row to row ------------------


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("M,K", [(9001, 520), (4500, 1032), (4200, 1536), (1500, 2056), (1100, 4096), (700, 6152), (1030, 8192), (700, 8200), (600, 20000)])
def test_norm_of_many_rows(M, K, kind):
    _norm_case(M, M, K, kind)
    _norm_case(M + 1, M, K, kind, post=True, gate="token", scale=0.5, in_place="both")


# ---- attention of one new token ------------------------------------------------------------------------


def _shared_pages(seed, lengths, H, heads, d, page, bits, n_pages=300, layout="heads", bad=()):
    """Sequences whose tables point into one small cache; `bad`: (sequence, token) whose page is outside."""
    g = gen(seed)
    k, v, ks, vs = make_cache(g, n_pages, heads, page, d, bits, layout)
    table = torch.randint(0, n_pages, (len(lengths), -(-max(lengths) // page)), generator=g, device=DEV).int()
    for s, t in bad:
        table[s, t // page] = -1 if t % 2 else n_pages
    q = normal(g, len(lengths), H, d)
    say(f"[attend] S={len(lengths)} H={H}/{heads} d={d} page={page} bits={bits} longest={max(lengths)}")
    got = B.muxq_paged_attention(q, k, v, table, ints(lengths), max(lengths), k_scale=ks, v_scale=vs)
    torch.cuda.synchronize()
    want, tol = attend64(q, k, v, ks, vs, table, lengths, d ** -0.5)
    check(got, want, tol, "attention")


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("page", [8, 16, 256])
def test_attention_shares_of_many_thousand_tokens(page, bits):
    # 512 shares of about 10000 tokens: page offsets come to LDS 4096 tokens at a time; pages outside the cache in the first, in the
    # second, and in the last of them
    lengths = [12000 - 61 * i for i in range(64)]
    lengths[5], lengths[6], lengths[40] = 1, 0, 17
    bad = [(0, 100), (1, 5001), (1, 5300), (2, 11999), (9, 4096), (10, 4095), (20, 8192), (21, 8191), (30, 0)]
    _shared_pages(page, lengths, 16, 8, 128, page, bits, bad=bad)


def test_attention_shares_of_wide_heads():
    lengths = [9000, 8191, 8192, 8193, 4096, 4097, 12288, 300, 0, 7000, 11000, 5000]
    _shared_pages(3, lengths, 8, 8, 256, 16, 16, bad=[(0, 4500), (6, 12287)])
    _shared_pages(4, lengths, 8, 8, 192, 32, 8, bad=[(1, 4500), (6, 3)])


@pytest.mark.parametrize("S,longest,bits", [(257, 5000, 16), (300, 3000, 8), (1000, 2600, 16), (2048, 2501, 8)])
def test_attention_of_hundreds_of_sequences_with_shares(S, longest, bits):
    # steps are counted by several sequences to a thread
    g = gen(S)
    lengths = (torch.rand(S, generator=g, device=DEV) ** 6 * longest).int().tolist()
    lengths[0], lengths[S // 2], lengths[S - 1] = longest, 0, longest - 7
    _shared_pages(S, lengths, 4, 2, 64, 16, bits, bad=[(0, longest - 3), (S - 1, 40)])


@pytest.mark.parametrize("bits", [16, 8])
def test_attention_of_more_sequences_than_shares_count(bits):
    # a workgroup to a sequence and head, whatever its length: page offsets are fetched again there too
    S = 2100
    g = gen(S)
    lengths = (torch.rand(S, generator=g, device=DEV) * 40).int().tolist()
    lengths[3], lengths[S - 1], lengths[1000] = 9000, 4097, 4096
    _shared_pages(S, lengths, 4, 2, 64, 16, bits, bad=[(3, 8999), (3, 4099), (S - 1, 4096)])
