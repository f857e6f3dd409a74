"""What the bindings of muxq_block.h make of their tensors, without a GPU: tensors that only say that they are on one, and a
library that records its arguments."""
import pytest
import torch

from paper_2604_04701_amd import binding as B


class OnGpu(torch.Tensor):
    """A tensor that passes for one on the GPU; what is made from it by indexing does too."""
    is_cuda = True


class Library:
    """Entry points that write their arguments down and succeed."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def entry(*args):
            self.calls.append((name, args))
            return 0
        return entry


@pytest.fixture
def calls(monkeypatch):
    library = Library()
    monkeypatch.setattr(B, "lib", lambda: library)
    monkeypatch.setattr(B, "_stream", lambda: None)
    return library.calls


def gpu(*shape, dtype=torch.float16):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnGpu)


def norm_args(M, K):
    return dict(x=gpu(M, K), weight=gpu(K), out=gpu(M, K), residual_out=gpu(M, K))


@pytest.mark.parametrize("M", [1, 3])
def test_gates_that_are_refused(calls, M):
    K = 64
    wrong = {"every second channel": gpu(M, 2 * K)[:, ::2], "binary32": gpu(M, K, dtype=torch.float32), "host memory": torch.zeros(M, K).half()}
    for what, gate in wrong.items():
        with pytest.raises(B.MuxqError, match="gate"):
            B.muxq_norm(**norm_args(M, K), gate=gate)
        assert calls == [], what


@pytest.mark.parametrize("M,of,stride", [(1, 64, 64), (1, 128, 64), (3, 64, 64), (3, 128, 128)])
def test_gates_of_rows(calls, M, of, stride):
    gate = gpu(M, of)[:, :64]
    B.muxq_norm(**norm_args(M, 64), gate=gate)
    (name, args), = calls
    assert name == "muxq_norm" and args[9] == gate.data_ptr() and args[10] == stride


def lora_args():
    return dict(X=gpu(4, 64), A=gpu(2, 8, 64), B=gpu(2, 32, 8), scales=gpu(2, dtype=torch.float32), starts=gpu(3, dtype=torch.int32),
                adapters=gpu(2, dtype=torch.int32), Y=gpu(4, 32), out=gpu(4, 32))


def attend_args():
    return dict(q=gpu(3, 4, 64), k_cache=gpu(4, 2, 16, 64), v_cache=gpu(4, 2, 16, 64), block_table=gpu(3, 2, dtype=torch.int32),
                lengths=gpu(3, dtype=torch.int32), max_length=32, out=gpu(3, 4, 64))


ROOMS = [(B.muxq_lora, lora_args, "workspace"), (B.muxq_paged_attention, attend_args, "workspace"), (B.muxq_norm, lambda: norm_args(70, 64), "scratch")]


@pytest.mark.parametrize("call,args,name", ROOMS, ids=[c.__name__ for c, _, _ in ROOMS])
def test_workspaces_that_are_refused(calls, call, args, name):
    for what, room in (("host memory", torch.empty(512, dtype=torch.uint8)), ("every second byte", gpu(1024, dtype=torch.uint8)[::2])):
        with pytest.raises(B.MuxqError, match="workspace"):
            call(**args(), **{name: room})
        assert calls == [], what
    for room in (gpu(512, dtype=torch.uint8), gpu(128, dtype=torch.float32)):
        calls.clear()
        call(**args(), **{name: room})
        (_, given), = calls
        assert given[-3:] == (room.data_ptr(), 512, None)


def test_mfma_probe_does_not_time_the_loading_of_its_kernel(calls, monkeypatch):
    class Event:
        def __init__(self, **_):
            pass

        def record(self):
            calls.append(("record", ()))

        def elapsed_time(self, _):
            return 1.0
    monkeypatch.setattr(torch.cuda, "Event", Event)
    monkeypatch.setattr(torch.cuda, "synchronize", lambda: None)
    codes = torch.zeros(64, dtype=torch.int8)
    tops, _ = B.muxq_probe_mfma_rate(codes, codes, iters=200, n_workgroups=256)
    assert [name for name, _ in calls] == ["muxq_probe_mfma_rate", "record", "muxq_probe_mfma_rate", "record"]
    assert calls[0][1][3] == 1 and calls[2][1][3] == 200 and tops == pytest.approx(256 * 4 * 200 * 8 * 65536.0 / 1e-3 / 1e12)
