"""What the bindings for several new tokens make of workspaces, strides and numbers, without a GPU."""
import pytest

from paper_2604_04701_amd import binding as B
from test_several_host import ATTENTIONS, attention_args, calls, gpu          # noqa: F401

import torch


@pytest.mark.parametrize("call,more", ATTENTIONS, ids=["window", "tree"])
def test_a_workspace_of_another_device_is_refused(calls, call, more):          # noqa: F811
    ws = gpu(1 << 20, dtype=torch.uint8)
    call(**attention_args(), **more, workspace=ws)
    assert len(calls) == 1
    ws.at = 1
    with pytest.raises(B.MuxqError, match="workspace"):
        call(**attention_args(), **more, workspace=ws)
    assert len(calls) == 1
