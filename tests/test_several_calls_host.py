"""What the bindings for several new tokens make of workspaces, strides and numbers, without a GPU."""
import pytest
import torch

from paper_2604_04701_amd import binding as B
from test_block_host import cache
from test_several_host import ATTENTIONS, OnGpu, attention_args, calls, gpu, rows, verify_args          # noqa: F401


@pytest.mark.parametrize("call,more", ATTENTIONS, ids=["window", "tree"])
def test_a_workspace_of_another_device_is_refused(calls, call, more):          # noqa: F811
    ws = gpu(1 << 20, dtype=torch.uint8)
    call(**attention_args(), **more, workspace=ws)
    assert len(calls) == 1
    ws.at = 1
    with pytest.raises(B.MuxqError, match="workspace"):
        call(**attention_args(), **more, workspace=ws)
    assert len(calls) == 1


I32, F32 = torch.int32, torch.float32
FAR = 1 << 32


def far(shape, stride, dtype=torch.float16):
    """A tensor with strides that no memory here holds."""
    return torch.empty_strided(shape, stride, dtype=dtype, device="meta").as_subclass(OnGpu)


def moves(**kw):
    return dict(path=gpu(5, dtype=I32), counts=gpu(3, dtype=I32), starts=gpu(4, dtype=I32), lengths=gpu(3, dtype=I32), block_table=gpu(3, 2, dtype=I32),
                max_nodes=4, k_cache=gpu(4, 2, 16, 64), v_cache=gpu(4, 2, 16, 64)) | kw


@pytest.mark.parametrize("call,more", ATTENTIONS, ids=["window", "tree"])
def test_row_strides_beyond_31_bits_are_refused(calls, call, more):          # noqa: F811
    for kw in (dict(q=far((5, 4, 64), (FAR + 512, 64, 1))), dict(out=far((5, 4, 64), (FAR + 512, 64, 1))), dict(block_table=far((3, 2), (FAR + 2, 1), I32))):
        with pytest.raises(B.MuxqError):
            call(**attention_args() | more | kw)
    with pytest.raises(B.MuxqError):
        B.muxq_verify_tree(**verify_args() | dict(target=far((5, 100), (FAR + 100, 1), F32)))
    with pytest.raises(B.MuxqError):
        B.muxq_verify_tree(**verify_args() | dict(draft=far((5, 100), (FAR + 100, 1), F32)))
    with pytest.raises(B.MuxqError):
        B.muxq_kv_compact(**moves(block_table=far((3, 2), (FAR + 2, 1), I32)))
    assert calls == []


def test_numbers_beyond_31_bits_are_refused(calls):          # noqa: F811
    window, tree = (dict(attention_args(), **more) for _, more in ATTENTIONS)
    for call, args, names in ((B.muxq_window_attention, dict(window, window=0, sinks=0), ("max_new", "window", "sinks")),
                              (B.muxq_tree_attention, tree, ("max_nodes",)), (B.muxq_verify_tree, verify_args(), ("max_nodes",)),
                              (B.muxq_kv_compact, moves(), ("max_nodes",))):
        for name in names:
            for n in (FAR + 2, FAR, -FAR + 2, -1):
                with pytest.raises(B.MuxqError):
                    call(**args | {name: n})
            assert calls == []
        call(**args)
        assert len(calls) == 1
        calls.clear()


def test_a_single_row_may_carry_any_stride(calls):          # noqa: F811
    """As a view of another order gives it; there is no second row that it leads to."""
    one = dict(q=gpu(4, 1, 64).transpose(0, 1), out=gpu(4, 1, 64).transpose(0, 1), k_cache=gpu(4, 2, 16, 64), v_cache=gpu(4, 2, 16, 64),
               block_table=gpu(1, 2, dtype=I32), starts=gpu(2, dtype=I32), lengths=gpu(1, dtype=I32), max_length=32)
    assert one["q"].stride() == one["out"].stride() == (64, 64, 1)
    B.muxq_window_attention(**one, max_new=1)
    B.muxq_tree_attention(**one, max_nodes=1, parents=gpu(1, dtype=I32))
    for name, args in calls:
        assert args[1:4] == (1, 4, 256) and args[16 if "window" in name else 15] == 256, name
    calls.clear()
    # tables of one page each
    table = gpu(1, 3, dtype=I32).t()
    assert table.stride() == (1, 3)
    B.muxq_window_attention(**attention_args() | dict(block_table=table, max_length=16), max_new=1)
    B.muxq_kv_compact(**moves(block_table=table))
    assert [args[6 if "window" in name else 5] for name, args in calls] == [1, 1]


@pytest.mark.parametrize("heads,n_heads,M,status", [(128, 128, 1 << 24, 2), (64, 256, (1 << 22) + 1, 2), (1, 1024, (1 << 20) + 1, 2)])
def test_calls_of_more_workgroups_than_a_grid_has_are_refused(heads, n_heads, M, status):
    """Rows times heads beyond 2^30, for shapes and not by the launch."""
    c = cache(n_kv_heads=heads, ld_block=heads * 16 * 64)
    wide = dict(M=M, new=M, n_heads=n_heads, ldq=n_heads * 64, ldo=n_heads * 64, o=1 << 46, window=0, sinks=0)
    assert rows(c, **wide) == status
