"""The decode step of GPT-2 blocks: each operator between the projections against 64 bits on the step's own values, and the
captured step against the eager one, token by token."""
import pytest
import torch

from block_common import *
from paper_2604_04701_amd import decode_block as D

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kv_dtype", [torch.float16, torch.int8])
@pytest.mark.parametrize("rotated", [False, True])
def test_step_against_64_bits(kv_dtype, rotated):
    stack, batch, x = D.make(256, 4, blocks=2, S=5, context=70, kv_dtype=kv_dtype, rotated=rotated, seed=3)
    say(f"[decode] 2 blocks of 256, {kv_dtype}, rotated={rotated}")
    for _ in range(3):
        out, seen = D.run_step(stack, batch, x)
        torch.cuda.synchronize()
        assert torch.isfinite(out).all()
        for block, s in zip(stack, seen):
            k, v, ks, vs = block.cache
            starts, adapters = batch.starts.tolist(), batch.adapters.tolist()
            y, move = norm64(s["stream"].double(), *block.ln[0], "layer", 1e-5)
            # (the norm sees the stream before its rounding: half a unit of it, through the norm)
            check(s["h"], y, U16 * y.abs() + TINY16 + (2.0 ** -18 + 4 * U16) * move, "first norm")
            want, tol = lora64(s["h"], block.A, block.B, block.scales, starts, adapters, s["qkv"])
            check(s["tuned"], want, tol, "adapters")
            q, kk, vv = s["tuned"].view(5, 12, 64).split(4, 1)
            want = q.double()
            if rotated:
                want = rotate64(want, batch.cos_sin, batch.positions, False)
            check(s["q"], want, U16 * want.abs() + TINY16 + 4 * U32 * q.double().abs().amax(2, keepdim=True), "queries")
            _, back = B.muxq_kv_gather(batch.slots, k, v, k_scale=ks, v_scale=vs)
            step = vv.double().abs().amax(2, keepdim=True) / 127 * (0.501 if kv_dtype == torch.int8 else 0.0)
            check(back, vv.double(), step + 1.01 * U16 * vv.double().abs() + TINY16, "cached values")
            want, tol = attend64(s["q"], k, v, ks, vs, batch.table, batch.lengths.tolist(), 0.125)
            check(s["o"], want, tol, "attention")
            y, move = norm64(s["stream2"].double(), *block.ln[1], "layer", 1e-5)
            check(s["h2"], y, U16 * y.abs() + TINY16 + (2.0 ** -18 + 4 * U16) * move, "second norm")
            plain = B.muxq_linear(s["h"], block.c_attn[0], block.c_attn[1], 768, "channel", bias=block.c_attn[2])
            torch.cuda.synchronize()
            assert torch.equal(plain, s["qkv"])          # the maxima that the norm handed over are those of the layer's input
        batch.next_token()


def test_captured_step_follows_the_tokens():
    stack, batch, x = D.make(256, 4, blocks=2, S=6, context=40, seed=5, rotated=True)
    B.muxq_init()
    say("[decode] captured step")
    D.run_step(stack, batch, x)
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        out, _ = D.run_step(stack, batch, x)
    torch.cuda.synchronize()
    for _ in range(4):
        batch.next_token()
        x.copy_(torch.randn_like(x, dtype=torch.float32).half())
        graph.replay()
        torch.cuda.synchronize()
        first = out.clone()
        again, _ = D.run_step(stack, batch, x)
        torch.cuda.synchronize()
        assert torch.equal(first, again)
