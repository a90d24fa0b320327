"""The workspace of attention of chunks: only its header is zero at first, whatever the rest holds."""

import pytest
import torch

import chunk_reference as ref
from test_gpu_chunk import i32, make, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("path", [1, 0])
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("value", [0xff, 0x5a])
def test_anything_behind_the_header(path, fp8, value):
    from paper_2609_04010_gb300 import binding as b
    c = make([1, 200, 0, 3, 1], [20000, 900, 5, 0, 77], fp8=fp8, seed=61)
    out, lse = (torch.empty(c["q"].shape[:n], dtype=t, device="cuda") for n, t in ((3, torch.bfloat16), (2, torch.float32)))
    a = b.chunk_attn_args(c["q"], c["cache"], c["table"], i32(c["starts"]), i32(c["lens"]), out, lse, path=path)
    ws = b.new_chunk_attn_workspace(a)
    assert ws.numel() == b.chunk_attn_workspace_size(a) and not ws[:256].any()
    ws[256:] = value
    b.chunk_attention_args(a, ws)
    assert b.read_device_status(ws) == (0, 0)
    ref.check((out, lse), ref.attend(c), c, path == 1)


def test_the_plain_call_fills_only_the_header(monkeypatch):
    from paper_2609_04010_gb300 import binding as b
    c = make([1, 200], [20000, 900], seed=62)
    want = run(c)[:2]
    filled = []
    zeros = torch.zeros

    def watch(*args, **kwargs):
        t = zeros(*args, **kwargs)
        filled.append(t.numel() * t.element_size())
        return t
    monkeypatch.setattr(torch, "zeros", watch)
    got = b.chunk_attention(c["q"], c["cache"], c["table"], i32(c["starts"]), i32(c["lens"]))
    assert sum(filled) <= got[0].numel() * 2
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_the_status_is_in_the_workspace():
    from paper_2609_04010_gb300 import binding as b
    c = make([1, 20], [300, 90], seed=63)
    starts, lens = i32(c["starts"]), i32(c["lens"])
    ws = b.new_chunk_attn_workspace(b.chunk_attn_args(c["q"], c["cache"], c["table"], starts, lens,
                                                      torch.empty_like(c["q"].contiguous())))
    c["table"][1, 0] = len(c["cache"][0]) + 3
    out, lse = b.chunk_attention(c["q"], c["cache"], c["table"], starts, lens, ws=ws)
    assert b.read_device_status(ws) == (5, b.FLAG_BAD_PAGE) and not out[1:].any()
    assert bool((lse[1:] == float("-inf")).all()) and bool(torch.isfinite(lse[0]).all())
