"""Calls on a stream of their own while the caller's current stream is busy: their results are there when
that stream is done, and stay, whatever the current stream does then."""

import numpy as np
import pytest
import torch

from test_gpu_chunk import i32, make
from test_gpu_pages import fork_case

pytestmark = pytest.mark.gpu
BUSY = 400_000_000  # clock cycles, about 0.2 s


def on_a_busy_day(call):
    """call(stream)'s results as the stream left them, and as they are when all work is done. Meanwhile
    the current stream is asleep, then fills whatever memory the call gave back."""
    call(None)  # (modules are loaded)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(BUSY)
    res = call(s)
    filled = [torch.full((n,), 0x5a, dtype=torch.uint8, device="cuda") for n in (1 << 10, 1 << 14, 1 << 18, 1 << 25, 1 << 26)]
    with torch.cuda.stream(s):
        early = [t.clone() for t in res]
    s.synchronize()
    awake = not torch.cuda.current_stream().query()
    early = [t.cpu() for t in early]
    torch.cuda.synchronize()
    del filled
    assert awake, "the current stream was done before the call's stream: nothing was tested"
    return early, [t.cpu() for t in res]


def check(call):
    want = [t.cpu() for t in call(None)]
    for _ in range(3):
        early, late = on_a_busy_day(call)
        for w, e, l in zip(want, early, late):
            assert torch.equal(e, w) and torch.equal(l, w)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("want_lse", [False, True])
def test_chunk_attention(fp8, want_lse):
    from paper_2609_04010_gb300 import binding as b
    c = make([300, 1, 5, 1], [700, 9000, 41, 0], fp8=fp8, seed=31)
    starts, lens = i32(c["starts"]), i32(c["lens"])

    def call(stream):
        out, lse = b.chunk_attention(c["q"], c["cache"], c["table"], starts, lens, want_lse=want_lse, stream=stream)
        return [t for t in (out, lse) if t is not None]
    check(call)


def test_rope():
    from paper_2609_04010_gb300 import binding as b
    g = torch.Generator(device="cuda").manual_seed(32)
    q, k = (torch.randn(300, h, 128, generator=g, device="cuda").bfloat16() for h in (8, 2))
    positions, t = i32(np.arange(300) - 2), b.rope_turns(b.rope_frequencies(128)[0])
    check(lambda stream: b.rope_kv(q, k, None, positions, t, stream=stream))


def test_fork():
    from paper_2609_04010_gb300 import binding as b
    c = fork_case(300, 16, seed=33, hi=2000)
    first = {k: i32(np.atleast_1d(c[k])) for k in ("parent", "kv_len", "table", "shares", "free", "count")}

    def call(stream):
        with torch.cuda.stream(stream):
            t = {k: v.clone() for k, v in first.items()}
        res = b.fork_sequences(t["parent"], t["kv_len"], t["table"], t["shares"], t["free"], t["count"], 16,
                               stream=stream)
        return [*t.values(), res["copies"], res["flags"]]
    check(call)


def test_verify_attention():
    """Its workspace holds counters, which are zeros when the launch begins."""
    from paper_2609_04010_gb300 import binding as b
    c = make([16, 16], [5000, 900], Hq=8, Hkv=2, seed=34)
    q = c["q"].reshape(2, 16, 8, 128).contiguous()
    lens = i32(c["lens"])
    check(lambda stream: list(b.verify_attention(q, *c["cache"], c["table"].clamp_min(0), lens, stream=stream)))


def test_map_slots():
    from paper_2609_04010_gb300 import binding as b
    n = 200
    new = i32(np.arange(n) % 7)
    first = dict(kv_len=i32(np.arange(n) * 3), table=i32(np.full((n, 60), -1)), free=i32(np.arange(5000)), count=i32([5000]))

    def call(stream):
        with torch.cuda.stream(stream):
            t = {k: v.clone() for k, v in first.items()}
        res = b.map_slots(new, t["kv_len"], t["table"], 16, 5000, t["free"], t["count"], 700, stream=stream)
        return [*t.values(), *res.values()]
    check(call)


def test_a_captured_stream():
    """Calls that are given the stream under capture, with what they make in the graph's own memory."""
    from paper_2609_04010_gb300 import binding as b
    c = make([300, 1, 5], [700, 9000, 41], seed=35)
    starts, lens = i32(c["starts"]), i32(c["lens"])
    positions, t = i32(np.arange(c["rows"])), b.rope_turns(b.rope_frequencies(128)[0])

    def call(stream):
        q, _ = b.rope_kv(c["q"], None, None, positions, t, stream=stream)
        return b.chunk_attention(q, c["cache"], c["table"], starts, lens, stream=stream)
    want = [x.clone() for x in call(None)]
    s, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(g, stream=s):
        got = call(s)
    for _ in range(3):
        for x in got:
            x.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
