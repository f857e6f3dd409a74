"""Refusals of the entry points for several new tokens of a sequence, and what their bindings make of their tensors, without a GPU."""
import ctypes as C
import random

import pytest
import torch

from paper_2604_04701_amd import binding as B
from test_block_binding_host import Library
from test_block_host import AWAY, FAKE, cache

I32 = torch.int32


class OnGpu(torch.Tensor):
    """A tensor that passes for one on a GPU, the first one if it does not say otherwise."""
    is_cuda = True
    at = 0

    def get_device(self):
        return self.at


def gpu(*shape, dtype=torch.float16):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnGpu)


@pytest.fixture
def calls(monkeypatch):
    library = Library()
    monkeypatch.setattr(B, "lib", lambda: library)
    monkeypatch.setattr(B, "_stream", lambda: None)
    monkeypatch.setattr(B, "_device", lambda: 0)
    return library.calls


def rows(c=None, tree=False, **kw):
    a = dict(q=FAKE, M=10, n_heads=8, ldq=512, c=C.byref(c if c is not None else cache()), table=FAKE, ldt=8, starts=FAKE, lengths=FAKE,
             parents=FAKE, S=4, new=8, most=128, window=32, sinks=4, scale=0.125, o=AWAY, ldo=512, ws=FAKE, ws_bytes=1 << 40)
    assert not set(kw) - set(a)
    a.update(kw)
    for name in ("window", "sinks") if tree else ("parents",):
        del a[name]
    return getattr(B.lib(), "muxq_tree_attention" if tree else "muxq_window_attention")(*a.values(), None)


def verify(**kw):
    a = dict(target=FAKE, ldt=100, draft=FAKE, ldd=100, M=10, V=100, tokens=FAKE, parents=FAKE, uniforms=FAKE, starts=FAKE, S=4, nodes=8,
             path=AWAY, counts=AWAY + 64, next=AWAY + 128)
    assert not set(kw) - set(a)
    a.update(kw)
    return B.lib().muxq_verify_tree(*a.values(), None)


def copy(c=None, **kw):
    a = dict(src=FAKE, dst=FAKE, n=4, c=C.byref(c if c is not None else cache()))
    a.update(kw)
    return B.lib().muxq_kv_copy(*a.values(), None)


def compact(c=None, **kw):
    a = dict(path=FAKE, counts=FAKE, starts=FAKE, lengths=FAKE, table=FAKE, ldt=8, M=10, S=4, nodes=8, c=C.byref(c if c is not None else cache()))
    a.update(kw)
    return B.lib().muxq_kv_compact(*a.values(), None)


@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("kw,status", [
    (dict(q=None), 1), (dict(o=None), 1), (dict(table=None), 1), (dict(starts=None), 1), (dict(lengths=None), 1), (dict(M=0), 2), (dict(M=(1 << 24) + 1), 2),
    (dict(S=0), 2), (dict(S=65536), 2), (dict(n_heads=6), 2), (dict(n_heads=0), 2), (dict(ldq=504), 2), (dict(ldq=516), 2), (dict(ldo=513), 2),
    (dict(ldt=0), 2), (dict(most=0), 2), (dict(most=129), 2), (dict(ldt=1 << 28, most=(1 << 26) + 1), 2), (dict(new=0), 2), (dict(new=(1 << 24) + 1), 2),
    (dict(scale=float("nan")), 4), (dict(scale=float("inf")), 4), (dict(q=FAKE + 8), 3), (dict(o=AWAY + 4), 3), (dict(table=FAKE + 2), 3),
    (dict(starts=FAKE + 1), 3), (dict(lengths=FAKE + 1), 3), (dict(o=FAKE), 4), (dict(o=FAKE + 64), 4)])
def test_attention_refuses(kw, status, tree):
    assert rows(tree=tree, **kw) == status


def test_what_one_of_them_refuses():
    assert rows(window=-1) == 4 and rows(sinks=-1) == 4
    assert rows(tree=True, parents=None) == 1 and rows(tree=True, parents=FAKE + 2) == 3 and rows(tree=True, new=65) == 2


@pytest.mark.parametrize("kw,status", [
    (dict(k=None), 1), (dict(type=1), 1), (dict(type=2), 4), (dict(block_size=24), 2), (dict(head_dim=72), 2), (dict(n_blocks=0), 2),
    (dict(ld_token=48), 2), (dict(ld_block=4000), 2), (dict(k=FAKE + 8), 3), (dict(v=FAKE + 2), 3)])
def test_caches_that_are_refused(kw, status):
    c = cache(**kw)
    assert rows(c) == status and rows(c, tree=True) == status and copy(c) == status and compact(c) == status


@pytest.mark.parametrize("kw,status", [
    (dict(target=None), 1), (dict(tokens=None), 1), (dict(parents=None), 1), (dict(starts=None), 1), (dict(path=None), 1), (dict(counts=None), 1),
    (dict(next=None), 1), (dict(M=0), 2), (dict(M=(1 << 24) + 1), 2), (dict(S=0), 2), (dict(S=65536), 2), (dict(V=0, ldt=0), 2), (dict(ldt=99), 2),
    (dict(V=(1 << 22) + 1, ldt=1 << 23, ldd=1 << 23), 2), (dict(ldd=99), 2), (dict(nodes=0), 2), (dict(nodes=65), 2), (dict(target=FAKE + 2), 3),
    (dict(draft=FAKE + 1), 3), (dict(uniforms=FAKE + 2), 3), (dict(tokens=FAKE + 3), 3), (dict(path=AWAY + 2), 3),
    (dict(path=FAKE + 36), 4), (dict(counts=AWAY + 36), 4), (dict(next=AWAY + 76), 4), (dict(next=AWAY - 12), 4), (dict(starts=AWAY + 76), 4)])
def test_verification_refuses(kw, status):
    assert verify(**kw) == status


def test_verification_refuses_outputs_among_the_probabilities():
    last = 4 * (9 * 100 + 99)                   # the last number of target and draft
    assert verify(path=FAKE + last) == verify(next=FAKE + last) == 4
    assert verify(target=FAKE + (1 << 20), counts=FAKE + last) == verify(draft=FAKE + (1 << 20), counts=FAKE + last) == 4
    assert verify(draft=FAKE + (1 << 20), next=FAKE + (1 << 20) + last) == 4


@pytest.mark.parametrize("kw,status", [(dict(src=None), 1), (dict(dst=None), 1), (dict(n=0), 2), (dict(n=(1 << 24) + 1), 2), (dict(src=FAKE + 2), 3),
                                       (dict(dst=FAKE + 1), 3)])
def test_copy_refuses(kw, status):
    assert copy(**kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(path=None), 1), (dict(counts=None), 1), (dict(starts=None), 1), (dict(lengths=None), 1), (dict(table=None), 1), (dict(ldt=0), 2), (dict(M=0), 2),
    (dict(S=0), 2), (dict(S=65536), 2), (dict(nodes=0), 2), (dict(nodes=65), 2), (dict(path=FAKE + 2), 3), (dict(table=FAKE + 1), 3)])
def test_compaction_refuses(kw, status):
    assert compact(**kw) == status


def test_no_cache_at_all():
    none = C.POINTER(B.KvCache)()
    assert rows(c=None, table=None) == 1
    assert B.lib().muxq_kv_copy(FAKE, FAKE, 4, none, None) == 1
    assert B.lib().muxq_kv_compact(FAKE, FAKE, FAKE, FAKE, FAKE, 8, 10, 4, 8, none, None) == 1


def test_workspaces():
    L = B.lib()
    for need, tail in ((L.muxq_window_attention_workspace_bytes, (0, 0)), (L.muxq_tree_attention_workspace_bytes, ())):
        assert need(0, 8, 8, 64, 1, 100, *tail) == 0 and need(1, 8, 3, 64, 1, 100, *tail) == 0 and need(1, 8, 8, 60, 1, 100, *tail) == 0
        assert need(1, 8, 8, 64, 0, 100, *tail) == 0 and need(1, 8, 8, 64, 1, 0, *tail) == 0
    assert L.muxq_tree_attention_workspace_bytes(1, 8, 8, 64, 65, 100000) == 0
    assert L.muxq_window_attention_workspace_bytes(1, 8, 8, 64, 1, 100000, -1, 0) == 0
    for tree, n in ((False, L.muxq_window_attention_workspace_bytes(1, 8, 4, 64, 1, 100000, 0, 0)),
                    (True, L.muxq_tree_attention_workspace_bytes(1, 8, 4, 64, 8, 100000))):
        long = dict(S=1, M=8, ldt=1 << 20, most=100000, new=8 if tree else 1, window=0, sinks=0)
        if n:
            # (what a call needs is part of what serves all smaller ones)
            assert rows(tree=tree, **long, ws_bytes=1024) == 5 and rows(tree=tree, **long, ws=None) == 1 and rows(tree=tree, **long, ws=FAKE + 16) == 3


@pytest.mark.parametrize("H,heads,d", [(32, 8, 128), (20, 20, 64), (4, 1, 256), (12, 4, 80), (130, 2, 64)])
def test_a_workspace_for_the_largest_batch_serves_every_smaller_one(H, heads, d):
    L = B.lib()
    rng = random.Random(d)

    def log(lo, hi):
        return int(lo * (hi / lo) ** rng.random())
    for _ in range(1500):
        S, most, new = log(1, 4096), log(1, 1 << 22), log(1, 1 << 15)
        window, sinks = rng.choice([0, log(1, 1 << 16)]), rng.choice([0, log(1, 4096)])
        s, m, x = log(1, S), log(1, most), log(1, new)
        w = log(1, window or 1 << 18) if window or rng.random() < 0.5 else 0
        k = rng.randint(0, sinks) if window else log(1, 4096)
        need = L.muxq_window_attention_workspace_bytes
        assert need(s, H, heads, d, x, m, w, k) <= need(S, H, heads, d, new, most, window, sinks), (S, new, most, window, sinks, s, x, m, w, k)
        new, x = min(new, 64), min(x, 64)
        need = L.muxq_tree_attention_workspace_bytes
        assert need(s, H, heads, d, min(x, new), m) <= need(S, H, heads, d, new, most), (S, new, most, s, x, m)


def attention_args():
    return dict(q=gpu(5, 4, 64), k_cache=gpu(4, 2, 16, 64), v_cache=gpu(4, 2, 16, 64), block_table=gpu(3, 2, dtype=I32), starts=gpu(4, dtype=I32),
                lengths=gpu(3, dtype=I32), max_length=32, out=gpu(5, 4, 64))


ATTENTIONS = [(B.muxq_window_attention, dict(max_new=2)), (B.muxq_tree_attention, dict(max_nodes=2, parents=gpu(5, dtype=I32)))]


@pytest.mark.parametrize("call,more", ATTENTIONS, ids=["window", "tree"])
@pytest.mark.parametrize("kw", [
    dict(q=torch.zeros(5, 4, 64).half()), dict(q=gpu(5, 4, 64, dtype=torch.float32)), dict(q=gpu(5, 4, 128)[..., ::2]), dict(q=gpu(5, 8, 64)[:, ::2]),
    dict(q=gpu(5, 4, 32), out=gpu(5, 4, 32)), dict(out=gpu(5, 2, 64)), dict(starts=gpu(3, dtype=I32)), dict(starts=gpu(4)),
    dict(starts=torch.zeros(4, dtype=I32)), dict(lengths=gpu(3, dtype=torch.int64)), dict(lengths=gpu(6, dtype=I32)[::2]),
    dict(block_table=gpu(2, 2, dtype=I32)), dict(block_table=gpu(2, 3, dtype=I32).t()), dict(max_length=33), dict(k_cache=gpu(4, 2, 16, 128)[..., ::2]),
    dict(k_scale=gpu(4, 2, 16, dtype=torch.float32)), dict(workspace=torch.empty(64, dtype=torch.uint8))])
def test_tensors_that_attention_refuses(calls, call, more, kw):          # noqa: F811
    with pytest.raises(B.MuxqError):
        call(**{**attention_args(), **more, **kw})
    assert calls == []


def test_parents_that_are_refused(calls):          # noqa: F811
    for parents in (gpu(4, dtype=I32), gpu(5), torch.zeros(5, dtype=I32), gpu(10, dtype=I32)[::2]):
        with pytest.raises(B.MuxqError, match="parents"):
            B.muxq_tree_attention(**attention_args(), max_nodes=2, parents=parents)
    assert calls == []


def test_strides_go_through(calls):          # noqa: F811
    a = attention_args()
    a["q"] = gpu(5, 8, 64)[:, 2:6]
    a["block_table"] = gpu(3, 9, dtype=I32)[:, 1:3]
    B.muxq_window_attention(**a, max_new=2, window=7, sinks=3)
    (name, args), = calls
    assert name == "muxq_window_attention" and args[1:4] == (5, 4, 512) and args[6] == 9 and args[9:14] == (3, 2, 32, 7, 3)


def verify_args():
    return dict(target=gpu(5, 100, dtype=torch.float32), tokens=gpu(5, dtype=I32), starts=gpu(3, dtype=I32), parents=gpu(5, dtype=I32), max_nodes=4,
                draft=gpu(5, 100, dtype=torch.float32), uniforms=gpu(5, dtype=torch.float32), path=gpu(5, dtype=I32), counts=gpu(2, dtype=I32),
                next_token=gpu(2, dtype=I32))


@pytest.mark.parametrize("kw", [
    dict(target=gpu(5, 100)), dict(target=torch.zeros(5, 100)), dict(target=gpu(5, 200, dtype=torch.float32)[:, ::2]), dict(draft=gpu(5, 99, dtype=torch.float32)),
    dict(draft=gpu(4, 100, dtype=torch.float32)), dict(tokens=gpu(5, dtype=torch.int64)), dict(tokens=gpu(4, dtype=I32)), dict(parents=torch.zeros(5, dtype=I32)),
    dict(uniforms=gpu(4, dtype=torch.float32)), dict(uniforms=gpu(5)), dict(path=gpu(6, dtype=I32)), dict(counts=gpu(3, dtype=I32)), dict(next_token=gpu(2))])
def test_tensors_that_the_verification_refuses(calls, kw):          # noqa: F811
    with pytest.raises(B.MuxqError):
        B.muxq_verify_tree(**{**verify_args(), **kw})
    assert calls == []


def test_tensors_that_the_pages_refuse(calls):          # noqa: F811
    kv = dict(k_cache=gpu(4, 2, 16, 64), v_cache=gpu(4, 2, 16, 64))
    for src, dst in ((gpu(3, dtype=I32), gpu(2, dtype=I32)), (gpu(3), gpu(3, dtype=I32)), (torch.zeros(3, dtype=I32), gpu(3, dtype=I32))):
        with pytest.raises(B.MuxqError):
            B.muxq_kv_copy(src, dst, **kv)
    good = dict(path=gpu(5, dtype=I32), counts=gpu(2, dtype=I32), starts=gpu(3, dtype=I32), lengths=gpu(2, dtype=I32), block_table=gpu(2, 3, dtype=I32),
                max_nodes=4, **kv)
    for kw in (dict(path=gpu(5)), dict(counts=torch.zeros(2, dtype=I32)), dict(starts=gpu(2, dtype=I32)), dict(lengths=gpu(1, dtype=I32)),
               dict(block_table=gpu(3, 3, dtype=I32)), dict(block_table=gpu(3, 2, dtype=I32).t()), dict(block_table=torch.zeros(2, 3, dtype=I32))):
        with pytest.raises(B.MuxqError):
            B.muxq_kv_compact(**{**good, **kw})
    assert calls == []
    B.muxq_kv_compact(**good)
    assert calls[0][0] == "muxq_kv_compact"


def test_tensors_of_other_devices_are_refused(calls, monkeypatch):          # noqa: F811
    kv = dict(k_cache=gpu(4, 2, 16, 64), v_cache=gpu(4, 2, 16, 64))
    copies = dict(src=gpu(3, dtype=I32), dst=gpu(3, dtype=I32), **kv)
    moved = dict(path=gpu(5, dtype=I32), counts=gpu(2, dtype=I32), starts=gpu(3, dtype=I32), lengths=gpu(2, dtype=I32), block_table=gpu(2, 3, dtype=I32),
                 max_nodes=4, **kv)
    for call, args in ((B.muxq_window_attention, dict(attention_args(), max_new=2)),
                       (B.muxq_tree_attention, dict(attention_args(), max_nodes=2, parents=gpu(5, dtype=I32))),
                       (B.muxq_verify_tree, verify_args()), (B.muxq_kv_copy, copies), (B.muxq_kv_compact, moved)):
        tensors = [n for n, x in args.items() if torch.is_tensor(x)]
        for name in tensors:
            args[name].at = 1
            with pytest.raises(B.MuxqError, match="devices"):
                call(**args)
            args[name].at = 0
        assert calls == []
        call(**args)
        assert len(calls) == 1
        monkeypatch.setattr(B, "_device", lambda: 1)
        with pytest.raises(B.MuxqError, match="current"):
            call(**args)
        monkeypatch.setattr(B, "_device", lambda: 0)
        assert len(calls) == 1
        calls.clear()
