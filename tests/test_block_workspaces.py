"""Workspaces of the operators between the projections: needed where they should be, and one for the largest batch serves every smaller one."""
import ctypes as C
import random

import pytest

from paper_2604_04701_amd import binding as B
from test_block_host import AWAY, FAKE, attend, lora, norm


def test_adapters_of_fewer_rows_and_requests_fit():
    need = B.lib().muxq_lora_workspace_bytes
    rng = random.Random(3)
    assert need(8192, 4096, 4096, 32, 500) >= need(8192, 4096, 4096, 32, 1)
    assert need(16384, 4096, 4096, 32, 8) >= need(15192, 4096, 4096, 32, 8) and need(8192, 4096, 4096, 32, 8) >= need(7935, 4096, 4096, 32, 8)
    for _ in range(4000):
        K, r = 8 * rng.randint(1, 1200), 8 * rng.randint(1, 16)
        M, requests = int(2 ** rng.uniform(0, 16)), int(2 ** rng.uniform(0, 10))
        most = need(M, K, 512, r, requests)
        assert (most > 0) == (r * K >= 1 << 16)
        m, q = rng.randint(max(1, M // 2), M), rng.randint(1, requests)
        k, s = 8 * rng.randint(1, K // 8), 8 * rng.randint(1, r // 8)
        assert need(m, K, 512, r, q) <= most and need(m, k, 512, s, q) <= most, (M, K, r, requests, m, q)
        # pieces of K as the kernel divides it, with tiles of 32 rows where it takes them
        if most:
            two_rows = r <= 64 and m >= 32 * q and m * K >= 3 << 19
            tiles = m // (32 if two_rows else 16) + q
            steps = -(-K // 512)
            pieces = min(-(-512 // tiles), steps)
            piece = -(-steps // pieces) * 512
            assert -(-K // piece) * m * r * 4 <= most, (M, K, r, requests, m, q)


def test_workspaces_are_needed_and_checked():
    n = B.lib().muxq_lora_workspace_bytes(8192, 4096, 4096, 64, 4)
    assert n > 0
    big = dict(M=8192, K=4096, ldx=4096, N=4096, ldy=4096, ldo=4096, r=64)
    assert lora(**big, ws_bytes=n - 1) == 5 and lora(**big, ws=None) == 1 and lora(**big, ws=FAKE + 8) == 3
    n = B.lib().muxq_paged_attention_workspace_bytes(1, 8, 4, 64, 100000)
    assert n > 0
    long = dict(S=1, ldt=1 << 20, most=100000)
    assert attend(**long, ws_bytes=n - 1) == 5 and attend(**long, ws=None) == 1 and attend(**long, ws=FAKE + 16) == 3
    n = B.lib().muxq_norm_scratch_bytes(100000, 768)
    assert n > 0
    rows = dict(M=100000, K=768, ldx=768, ldr=768, ldro=768, ldy=768, slabs=FAKE)
    assert norm(**rows, scratch=FAKE, scratch_bytes=n - 1) == 5 and norm(**rows) == 1 and norm(**rows, scratch=FAKE + 8, scratch_bytes=n) == 3


@pytest.mark.parametrize("H,heads,d", [(32, 8, 128), (20, 20, 64), (4, 1, 256), (12, 4, 80)])
def test_attention_of_fewer_sequences_and_tokens_fits(H, heads, d):
    need = B.lib().muxq_paged_attention_workspace_bytes
    rng = random.Random(d)
    for _ in range(1000):
        S, most = min(int(2 ** rng.uniform(0, 16)), 65535), int(2 ** rng.uniform(0, 20))
        s, m = rng.randint(1, S), rng.randint(1, most)
        assert need(s, H, heads, d, m) <= need(S, H, heads, d, most), (S, most, s, m)


def test_no_cache_at_all():
    L = B.lib()
    assert L.muxq_kv_append(FAKE, FAKE, 8, 768, 768, FAKE, 4, 768, AWAY, 256, FAKE, FAKE, FAKE, 9, 64, 0, C.POINTER(B.KvCache)(), None) == 1
    assert L.muxq_paged_attention(FAKE, 4, 8, 512, C.POINTER(B.KvCache)(), FAKE, 8, FAKE, 128, 0.125, AWAY, 512, FAKE, 1 << 40, None) == 1
