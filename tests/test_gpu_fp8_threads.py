"""Calls of several host threads at once, each with its own stream, workspace and tensors: sizes
whose blocks need different amounts of shared memory must not fail one another's launches."""

import threading

import pytest
import torch

from test_gpu_kv_fp8 import i32

pytestmark = pytest.mark.gpu


def attention_call(B, G):
    from paper_2609_04010_gb300 import binding as b
    q = torch.randn(B, G, 8, 64, device="cuda").bfloat16()
    cache, scale = b.new_kv_cache_fp8(4, 2, 16, 64)
    out = torch.empty_like(q)
    a = b.attn_fp8_args(q, cache, scale, i32([[0, 1, 2, 3]] * B), i32([G + 5] * B), out)
    ws = b.new_workspace(b.attn_fp8_workspace_size(a))
    return lambda stream: b.verify_attention_fp8_args(a, ws, stream), (q, cache, scale, out, ws, a)


def slots_call(B):
    from paper_2609_04010_gb300 import binding as b
    i = dict(dtype=torch.int32, device="cuda")
    t = dict(new=torch.ones(B, **i), kv=torch.zeros(B, **i), new_len=torch.empty(B, **i), table=torch.full((B, 4), -1, **i),
             free=torch.arange(B, **i), count=torch.full((1,), B, **i), new_count=torch.empty(1, **i),
             start=torch.empty(B + 1, **i), slots=torch.empty(B, **i))
    a = b.slot_args(t["new"], t["kv"], t["new_len"], t["table"], 16, B, t["free"], t["count"], t["new_count"],
                    t["start"], t["slots"])
    ws = b.new_workspace(b.slot_workspace_size(a))
    return lambda stream: b.map_slots_args(a, ws, stream), (t, ws, a)


@pytest.mark.parametrize("kind", ["few rows", "many rows", "slots"])
def test_calls_of_different_sizes_at_once(kind):
    if kind == "slots":
        calls = [slots_call(n) for n in (4000, 8192, 4000, 8192)]
    else:
        calls = [attention_call(n, 2 if kind == "few rows" else 10) for n in (1, 900, 1, 1000)]
    torch.cuda.synchronize()
    errors, go = [], threading.Barrier(len(calls))

    def work(call):
        try:
            stream = torch.cuda.Stream()
            go.wait()
            for _ in range(1500):
                call(stream)
            stream.synchronize()
        except Exception as e:  # noqa: BLE001
            errors.append(repr(e))

    threads = [threading.Thread(target=work, args=(c[0],)) for c in calls]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors
