"""Attention of prompts on streams of its own: what the streams read and write was made by another one, so each waits."""
import pytest
import torch

from harness import need_gpu
from test_prompt_attn import Prompt

pytestmark = pytest.mark.gpu


def to_host(pair):
    return [x.double().cpu().numpy() for x in pair]


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("D,rows,seq", [(64, [300, 5], [900, 2000]), (128, [700, 1, 90], [700, 3000, 4000])])
def test_two_streams_share_a_plan(D, rows, seq, bf16):
    need_gpu()
    t = Prompt(65, 4, 1, D, rows, seq)
    t.upload()
    t.make_plan()
    outs, spaces = [t.outputs(bf16) for _ in range(2)], [t.ws, torch.zeros_like(t.ws)]
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    for st in streams:
        st.wait_stream(torch.cuda.current_stream())
    for i in range(4):
        for (out, lse), ws, st in zip(outs, spaces, streams):
            t.P.prompt_attn(t.shape, t.inp, t.rows, t.plan, out, lse, ws, stream=st)
    torch.cuda.synchronize()
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
    ref, rlse, mag = t.oracle()
    t.compare(*to_host(outs[0]), ref, rlse, mag, bf16)


def test_plan_and_attention_on_a_stream_of_their_own():
    """The plan is made on the stream that reads it; the default stream waits before it looks."""
    need_gpu()
    t = Prompt(66, 4, 2, 64, [40, 200, 1], [90, 200, 1000])
    t.upload()
    out, lse = t.outputs(False)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    t.P.prompt_plan(t.shape, t.rows, t.dseq, True, 0, t.plan, stream=st)
    t.P.prompt_attn(t.shape, t.inp, t.rows, t.plan, out, lse, t.ws, stream=st)
    torch.cuda.current_stream().wait_stream(st)
    ref, rlse, mag = t.oracle()
    t.compare(*to_host((out, lse)), ref, rlse, mag, False)
