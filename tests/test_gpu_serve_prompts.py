"""The serving example: rotary positions, cache writes, attention of chunks, forks and page copies
together, each call's results against the definitions on what it was given, and the cache's
contents against a plain list of every sequence's keys and values."""

import importlib.util
import os

import numpy as np
import pytest
import torch

import serving_reference as ref

pytestmark = pytest.mark.gpu


def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "serve_prompts.py")
    spec = importlib.util.spec_from_file_location("serve_prompts", path)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def watched(mod, monkeypatch, **kw):
    """A server whose attention calls are checked as they are made, and whose rotated keys and values
    are kept by sequence and layer in plain lists."""
    b = mod.b
    s = mod.Server(**kw)
    held = [[[] for _ in range(s.L)] for _ in range(s.B)]  # [sequence][layer] of (keys, values) a call
    now = dict(layer=0, checks=0)
    attend, rotate, append = b.chunk_attention, b.rope_kv, b.append_kv_fp8

    def keep(k, v, starts):
        for i in range(s.B):
            if starts[i + 1] > starts[i]:
                held[i][now["layer"]].append((k[starts[i]:starts[i + 1]].clone(), v[starts[i]:starts[i + 1]].clone()))

    def rope_kv(q, k, v, positions, turns, *args, **kwargs):
        before = k.clone(), q.clone()
        got_q, got_k = rotate(q, k, v, positions, turns, *args, **kwargs)
        freq, factor = b.rope_frequencies(s.D // 2, 10000.0, "yarn", 4.0, original_max=128)
        for got, old in ((got_k, before[0]), (got_q, before[1])):
            want = ref.rope(old, positions, freq, False, factor)
            size = old.double().abs().amax(-1, keepdim=True) * factor
            # one rounding of the result, and 2^-20 of the pair's size for sines and sums
            assert bool(((got.double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -19 * size).all())
        now["keys"] = got_k
        if v is not None:
            now["values"] = v
        return got_q, got_k

    def append_kv_fp8(k, v, *args):
        now["values"] = v
        append(k, v, *args)

    def chunk_attention(q, cache, table, row_start, kv_len, **kwargs):
        out, lse = attend(q, cache, table, row_start, kv_len, **kwargs)
        starts, lens = row_start.tolist(), kv_len.tolist()
        keep(now["keys"], now["values"], starts)
        want = ref.chunk_attention(q, cache, table, starts, lens, window=kwargs.get("window", 0))
        ref.check_chunk((out, lse), want, s.D, True)
        if not s.eight_bit:  # the pages hold exactly every sequence's keys and values
            for i in range(s.B):
                rows = held[i][now["layer"]]
                if starts[i + 1] > starts[i]:
                    for kind in (0, 1):
                        have = torch.cat([r[kind] for r in rows])
                        pages = table[i, :-(-lens[i] // s.P)].long()
                        stored = cache[kind][pages].transpose(1, 2).flatten(0, 1)[:lens[i]]
                        assert torch.equal(stored, have)
        now["layer"] = (now["layer"] + 1) % s.L
        now["checks"] += 1
        return out, lse
    monkeypatch.setattr(b, "chunk_attention", chunk_attention)
    monkeypatch.setattr(b, "rope_kv", rope_kv)
    monkeypatch.setattr(b, "append_kv_fp8", append_kv_fp8)
    return s, held, now


@pytest.mark.parametrize("eight_bit", [False, True])
@pytest.mark.parametrize("heads,dim,window,page", [((8, 2), 64, 0, 16), ((6, 2), 128, 50, 32)])
def test_prompts_samples_and_ends(monkeypatch, eight_bit, heads, dim, window, page):
    mod = example()
    s, held, now = watched(mod, monkeypatch, batch=6, num_q_heads=heads[0], num_kv_heads=heads[1], head_dim=dim,
                           window=window, page_size=page, eight_bit=eight_bit, num_pages=90)
    r = np.random.default_rng(1)

    def tokens(n):
        return r.integers(0, 512, n).tolist()
    s.submit({0: tokens(150), 2: tokens(33), 3: tokens(1)})
    while any(s.waiting):
        s.step(budget=64)
    assert s.kv_len.tolist() == [150, 0, 33, 1, 0, 0]

    def fork(parent):
        before = {k: getattr(s, k).cpu().numpy().copy() for k in ("kv_len", "table", "shares", "free")}
        count = int(s.free_count)
        res = s.fork(parent)
        want = ref.fork(np.array(parent), before["kv_len"], before["table"], before["shares"], before["free"], count, s.P, 0)
        assert np.array_equal(s.kv_len.cpu(), want["new_kv_len"]) and np.array_equal(s.table.cpu(), want["new_table"])
        assert np.array_equal(s.shares.cpu(), want["new_shares"]) and np.array_equal(res["copies"].cpu(), want["copies"])
        assert int(s.free_count) == want["new_count"][0] and not want["flags"].any()
        held[:] = [[list(layer) for layer in held[q]] if q >= 0 else [[] for _ in range(s.L)] for q in parent]

    fork([0, 0, 2, 2, 0, 3])  # 3's own place is taken by a sample of 2, it lives on as 5
    s.submit({i: tokens(1 + 3 * i) for i in range(6)})
    while any(s.waiting):
        s.step(budget=20)
    fork([1, -1, 2, 5, 0, 5])
    s.submit({0: tokens(1), 2: tokens(1), 3: tokens(40), 4: tokens(1)})
    logits = s.step(budget=1000)
    assert [x is None for x in logits] == [False, True, False, False, False, True]
    fork([-1] * 6)
    assert int(s.free_count) == 90 and not s.shares.any() and not s.kv_len.any()
    assert now["checks"] >= 2 * 5 and mod.b.read_device_status(s.status) == (0, 0)


def test_example_runs(capsys):
    example().main()
    assert "pages left: 240 of 240 status: (0, 0)" in capsys.readouterr().out
