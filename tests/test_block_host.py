"""Refusals of the entry points in muxq_block.h: bad arguments become status codes before anything is launched."""
import ctypes as C

import pytest

from paper_2604_04701_amd import binding as B

FAKE = 0x100000           # aligned, never dereferenced
AWAY = 1 << 40            # outputs stand apart from the inputs


def cache(**kw):
    a = dict(k=FAKE, v=FAKE, k_scale=None, v_scale=None, type=0, n_blocks=10, block_size=16, n_kv_heads=4, head_dim=64,
             reserved=0, ld_block=4 * 16 * 64, ld_head=16 * 64, ld_token=64)
    a.update(kw)
    return B.KvCache(*a.values())


def append(c=None, **kw):
    a = dict(k=FAKE, v=FAKE, M=8, ldk=768, ldv=768, q=FAKE, n_heads=4, ldq=768, q_out=AWAY, ldqo=256, slots=FAKE, positions=FAKE,
             cos_sin=FAKE, n_positions=9, rot=64, inter=0)
    a.update(kw)
    return B.lib().muxq_kv_append(*a.values(), C.byref(c if c is not None else cache()), None)


def attend(c=None, **kw):
    a = dict(q=FAKE, S=4, n_heads=8, ldq=512, c=C.byref(c if c is not None else cache()), table=FAKE, ldt=8, lengths=FAKE, most=128,
             scale=0.125, o=AWAY, ldo=512, ws=FAKE, ws_bytes=1 << 40)
    a.update(kw)
    return B.lib().muxq_paged_attention(*a.values(), None)


def gather(c=None, **kw):
    a = dict(slots=FAKE, M=8, c=C.byref(c if c is not None else cache()), k=AWAY, ldk=256, v=AWAY << 1, ldv=256)
    a.update(kw)
    return B.lib().muxq_kv_gather(*a.values(), None)


def lora(**kw):
    a = dict(x=FAKE, M=16, K=256, ldx=256, a=FAKE, b=FAKE, scales=FAKE, n=3, r=16, starts=FAKE, adapters=FAKE, requests=4, y=FAKE,
             ldy=512, N=512, out=AWAY, ldo=512, ws=FAKE, ws_bytes=1 << 40)
    a.update(kw)
    return B.lib().muxq_lora(*a.values(), None)


def norm(**kw):
    a = dict(x=FAKE, M=100, K=256, ldx=256, r=FAKE, ldr=256, r_scale=1.0, post_w=None, post_b=None, gate=None, ldg=0, w=FAKE, b=None,
             kind=0, eps=1e-5, r_out=AWAY, ldro=256, y=AWAY << 1, ldy=256, slabs=None, scratch=None, scratch_bytes=0)
    a.update(kw)
    return B.lib().muxq_norm(*a.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(k=None), 1), (dict(v=None), 1), (dict(type=1), 1), (dict(type=2), 4), (dict(reserved=1), 4),
    (dict(block_size=0), 2), (dict(block_size=4), 2), (dict(block_size=24), 2), (dict(block_size=512, ld_block=1 << 20), 2),
    (dict(head_dim=8), 2), (dict(head_dim=72), 2), (dict(head_dim=272), 2), (dict(n_kv_heads=0), 2), (dict(n_blocks=0), 2),
    (dict(n_blocks=1 << 28), 2), (dict(ld_token=48), 2), (dict(ld_token=72), 2), (dict(ld_head=512), 2), (dict(ld_block=4000), 2),
    (dict(ld_block=4 * 16 * 64 - 16), 2), (dict(ld_block=-4096), 2), (dict(k=FAKE + 8), 3), (dict(v=FAKE + 2), 3),
    (dict(type=1, k_scale=FAKE + 2, v_scale=FAKE), 3)])
def test_caches_that_are_refused(kw, status):
    c = cache(**kw)
    assert append(c) == status and attend(c) == status and gather(c) == status


def test_no_cache():
    assert B.lib().muxq_kv_gather(FAKE, 8, None, AWAY, 256, AWAY << 1, 256, None) == 1
    assert attend(c=None, table=None) == 1


@pytest.mark.parametrize("kw,status", [
    (dict(k=None), 1), (dict(v=None), 1), (dict(slots=None), 1), (dict(q_out=None), 1), (dict(positions=None), 1), (dict(cos_sin=None), 1),
    (dict(M=0), 2), (dict(M=(1 << 24) + 1), 2), (dict(ldk=248), 2), (dict(ldk=257), 2), (dict(ldv=128), 2), (dict(ldq=255), 2), (dict(ldqo=250), 2),
    (dict(n_heads=0), 2), (dict(rot=4), 2), (dict(rot=72), 2), (dict(rot=-8), 2), (dict(n_positions=0), 2),
    (dict(k=FAKE + 4), 3), (dict(q=FAKE + 8), 3), (dict(q_out=AWAY + 2), 3), (dict(slots=FAKE + 1), 3), (dict(cos_sin=FAKE + 4), 3),
    (dict(q_out=FAKE + 512), 4), (dict(q_out=FAKE, ldqo=256), 4), (dict(q=FAKE + 1536, q_out=FAKE, ldqo=768), 4)])
def test_append_refuses(kw, status):
    assert append(**kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(slots=None), 1), (dict(k=None), 1), (dict(v=None), 1), (dict(M=0), 2), (dict(ldk=255), 2), (dict(ldv=248), 2), (dict(k=AWAY + 8), 3),
    (dict(slots=FAKE + 2), 3), (dict(v=AWAY + 256), 4)])
def test_gather_refuses(kw, status):
    assert gather(**kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(q=None), 1), (dict(o=None), 1), (dict(table=None), 1), (dict(lengths=None), 1), (dict(S=0), 2), (dict(S=65536), 2), (dict(n_heads=6), 2),
    (dict(n_heads=0), 2), (dict(ldq=504), 2), (dict(ldo=513), 2), (dict(ldt=0), 2), (dict(most=0), 2), (dict(most=129), 2), (dict(ldt=1 << 28, most=(1 << 26) + 1), 2),
    (dict(scale=float("nan")), 4), (dict(scale=float("inf")), 4), (dict(q=FAKE + 8), 3), (dict(o=AWAY + 4), 3), (dict(table=FAKE + 2), 3),
    (dict(lengths=FAKE + 1), 3), (dict(o=FAKE + 64), 4)])
def test_attention_refuses(kw, status):
    assert attend(**kw) == status


def test_attention_workspace():
    need = B.lib().muxq_paged_attention_workspace_bytes
    assert need(0, 8, 8, 64, 100) == 0 and need(1, 8, 3, 64, 100) == 0 and need(1, 8, 8, 60, 100) == 0 and need(1, 8, 8, 64, 0) == 0
    n = need(1, 8, 4, 64, 100000)
    if n:
        long = dict(S=1, ldt=1 << 20, most=100000)
        assert attend(**long, ws_bytes=n - 1) == 5 and attend(**long, ws=None) == 1 and attend(**long, ws=FAKE + 16) == 3


@pytest.mark.parametrize("kw,status", [
    (dict(x=None), 1), (dict(a=None), 1), (dict(b=None), 1), (dict(scales=None), 1), (dict(starts=None), 1), (dict(adapters=None), 1),
    (dict(y=None), 1), (dict(out=None), 1), (dict(M=0), 2), (dict(K=252), 2), (dict(K=0), 2), (dict(N=500), 2), (dict(r=0), 2), (dict(r=12), 2),
    (dict(r=136), 2), (dict(n=0), 2), (dict(requests=0), 2), (dict(ldx=248), 2), (dict(ldx=260), 2), (dict(ldy=504), 2), (dict(ldo=510), 2), (dict(ldx=(1 << 25) + 8), 2), (dict(ldo=1 << 26), 2),
    (dict(x=FAKE + 8), 3), (dict(a=FAKE + 2), 3), (dict(out=AWAY + 4), 3), (dict(starts=FAKE + 2), 3), (dict(out=FAKE + 512), 4),
    (dict(x=AWAY), 4), (dict(y=AWAY + 16), 4)])
def test_lora_refuses(kw, status):
    assert lora(**kw) == status


def test_lora_workspace():
    need = B.lib().muxq_lora_workspace_bytes
    assert need(0, 256, 512, 16, 4) == 0 and need(16, 252, 512, 16, 4) == 0 and need(16, 256, 512, 12, 4) == 0 and need(16, 256, 512, 16, 0) == 0
    big = dict(M=8192, K=4096, ldx=4096, N=4096, ldy=4096, ldo=4096, r=64)
    n = need(8192, 4096, 4096, 64, 4)
    if n:
        assert lora(**big, ws_bytes=n - 1) == 5 and lora(**big, ws=None) == 1 and lora(**big, ws=FAKE + 8) == 3


@pytest.mark.parametrize("kw,status", [
    (dict(x=None), 1), (dict(w=None), 1), (dict(y=None), 1), (dict(post_b=FAKE), 1), (dict(M=0), 2), (dict(K=250), 2), (dict(K=32776), 2),
    (dict(ldx=248), 2), (dict(ldr=100), 2), (dict(ldro=257), 2), (dict(ldy=255), 2), (dict(gate=FAKE, ldg=8), 2), (dict(kind=2), 4),
    (dict(eps=-1.0), 4), (dict(eps=float("nan")), 4), (dict(r_scale=float("inf")), 4), (dict(x=FAKE + 8), 3), (dict(w=FAKE + 2), 3),
    (dict(slabs=FAKE + 8), 3), (dict(y=AWAY), 4), (dict(y=FAKE + 16), 4), (dict(r_out=FAKE + 512), 4)])
def test_norm_refuses(kw, status):
    assert norm(**kw) == status


def test_norm_sizes():
    L = B.lib()
    assert L.muxq_norm_slabs(1, 768) == 1 and L.muxq_norm_slabs(64, 768) == 64 and L.muxq_norm_slabs(65, 768) == 1
    assert L.muxq_norm_slabs(0, 768) == 0 and L.muxq_norm_slabs(5, 12) == 0 and L.muxq_norm_scratch_bytes(5, 12) == 0
    n = L.muxq_norm_scratch_bytes(100000, 768)
    if n:
        assert norm(M=100000, K=768, ldx=768, ldr=768, ldro=768, ldy=768, slabs=FAKE, scratch=FAKE, scratch_bytes=n - 1) == 5
        assert norm(M=100000, K=768, ldx=768, ldr=768, ldro=768, ldy=768, slabs=FAKE) == 1
