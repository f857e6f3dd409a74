"""Attention of one new token with pages outside the cache, in each form of its kernel: short sequences, longer ones, shares; heads that fill
their dimensions and others; fp16 and codes."""
import pytest
import torch

from block_common import *          # noqa: F401,F403
from block_common import attend64, check, gen, ints, make_cache, make_table, normal, say
from paper_2604_04701_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("page", [8, 32])
@pytest.mark.parametrize("d", [64, 48, 128, 80, 256, 144])
@pytest.mark.parametrize("lengths", [[90, 33, 128, 5], [600, 1000, 129, 31], [20, 4000, 3000, 5000]], ids=["short", "long", "shares"])
def test_attention_leaves_out_tokens_of_missing_pages(lengths, d, page, bits):
    say(f"[attend] missing pages {lengths} d={d} page={page} bits={bits}")
    g, heads, H = gen(d + page), 2, 6
    n_pages = sum(-(-n // page) for n in lengths) + 3
    k, v, ks, vs = make_cache(g, n_pages, heads, page, d, bits)
    table, _ = make_table(g, lengths, page, n_pages, unused=1 << 30)
    gone = torch.rand(table.shape, generator=g, device=DEV)
    table[gone < 0.2] = -1
    table[gone > 0.8] = n_pages
    table[0, 0], table[1, (lengths[1] - 1) // page], table[3, :] = -5, n_pages + 1, -1          # a first one, a last one, all of them
    q = normal(g, len(lengths), H, d)
    got = B.muxq_paged_attention(q, k, v, table, ints(lengths), max(lengths), k_scale=ks, v_scale=vs)
    want, tol = attend64(q, k, v, ks, vs, table, lengths, d ** -0.5)
    check(got, want, tol, "attention")
    assert (got[3] == 0).all()
