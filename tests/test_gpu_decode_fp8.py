"""The 8-bit cache operators and the logit constraints together, as examples/decode_fp8.py runs
them: each stage of a step against the plain references on what the stage before left."""

import importlib.util
import os

import numpy as np
import pytest

torch = pytest.importorskip("torch")
import fp8_reference as ref  # noqa: E402

pytestmark = pytest.mark.gpu


def example():
    path = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples", "decode_fp8.py")
    spec = importlib.util.spec_from_file_location("decode_fp8", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def host(t):
    return t.cpu().numpy()


@pytest.mark.parametrize("gamma,Hq,H,D,P", [(1, 4, 2, 64, 16), (5, 8, 2, 64, 32), (16, 8, 2, 128, 16)])
def test_decoding(gamma, Hq, H, D, P):
    r = np.random.default_rng(gamma)
    V = 300
    d = example().Decoder(3, gamma, Hq, H, D, V, P, max_pages=256 // P, seed=3)
    prompts = [r.integers(0, V, n).tolist() for n in (2, 40, 131)]
    d.prefill(prompts)
    said = [list(p) for p in prompts]
    temp = torch.tensor([0.0, 0.0, 0.9], device="cuda")
    rep = torch.tensor([1.0, 1.5, 1.25], device="cuda")
    freq = torch.tensor([0.5, 0.0, 0.25], device="cuda")
    words = r.integers(0, 2 ** 32, (3, gamma, (V + 31) // 32), dtype=np.uint32) | np.uint32(0x10)
    allowed = torch.from_numpy(words.view(np.int32)).cuda()
    for _ in range(3):
        s = d.step(temp, repetition=rep, frequency=freq, allowed=allowed)
        n = host(s["num_accepted"]) + 1
        assert (n >= 1).all()
        # attention: the reference on the cache as the call read it (the derived bounds are
        # those of the operator's own tests)
        codes = host(d.cache.view(torch.uint8))
        scale, table, kv_len = host(d.scale), host(d.table), host(s["kv_len"])
        q = s["q"].view(3, gamma, Hq, D).double().cpu().numpy()
        ro, rl, mass, kmax = ref.attention(q, codes, scale, table, kv_len, gamma, P)
        qmax = np.repeat(np.abs(q).reshape(3, gamma, H, -1).max((1, 3)), Hq // H, 1)[:, None]
        ds = (D ** -0.5 * kmax * (2.0 ** -18 + 128 * 2.0 ** -24) * qmax)[..., None]
        vmax = np.abs(ref.decode(codes)).max() * scale[:, :, 1].max()
        tol = (2.0 ** -8 + 2 * ds) * mass + 2.0 ** -12 * vmax + 2.0 ** -9 * np.abs(ro)
        assert np.all(np.abs(s["out"].double().cpu().numpy() - ro) <= tol)
        # constraints: up to four fp32 roundings of values up to 1.5 |x| + the penalties
        hist, hl = host(d.history), host(s["history_len"])
        want = ref.adjust(host(s["raw"]), block=host(s["block"]), history=hist, history_len=hl,
                          prompt_len=host(d.prompt_len), repetition=host(rep), frequency=host(freq),
                          allowed=words)
        got = host(s["target"]).astype(np.float64)
        fin = np.isfinite(want)
        assert np.array_equal(fin, np.isfinite(got))
        bound = 2.0 ** -22 * (1.5 * np.abs(host(s["raw"]).astype(np.float64)) + 64)
        assert np.all(np.abs(got[fin] - want[fin]) <= bound[fin])
        # acceptance: greedy sequences emit the constrained argmax; all obey the mask
        out = host(s["out_tokens"])
        for b in range(3):
            assert out[b, 0] == said[b][-1]
            for i in range(1, n[b] + 1):
                t = int(out[b, i])
                assert words[b, i - 1, t // 32] >> np.uint32(t % 32) & 1
                if temp[b] == 0:
                    assert t == int(got[b, i - 1].argmax())
            said[b] += out[b, 1:n[b] + 1].tolist()
        # the cache holds every token but the last, and the history says which
        assert host(d.kv_len).tolist() == [len(x) - 1 for x in said]
        assert host(d.last).tolist() == [x[-1] for x in said]
        for b in range(3):
            assert host(d.history)[b, :len(said[b]) - 1].tolist() == said[b][:-1]
    # keys and values of all tokens held are those of their own projections, to e4m3's step
    # at the page's scale (rounded up to eight times as the scale rose)
    from paper_2609_04010_gb300 import binding as bnd
    assert bnd.read_device_status(d.status) == (0, 0)
    codes, scale, table = host(d.cache.view(torch.uint8)), host(d.scale), host(d.table)
    for b in range(3):
        toks = torch.tensor(said[b][:-1], device="cuda")
        _, _, k, v = d._project(toks)
        for kind, x in ((0, k), (1, v)):
            x = x.double().cpu().numpy()
            at = np.arange(len(said[b]) - 1)
            page = table[b, at // P]
            sc = scale[page, :, kind][..., None]
            held = ref.decode(codes[page, :, kind, at % P]) * sc
            assert np.all(np.abs(held - x) <= 8 * (2.0 ** -4 * np.abs(x) + 2.0 ** -10 * sc) + 2.0 ** -7 * np.abs(x).max())


@pytest.mark.parametrize("gamma,Hq", [(1, 4), (3, 16), (20, 8)])
def test_calls_that_overlap_see_what_those_before_wrote(gamma, Hq):
    """Slots, append and attention issued back to back, each launch free to start while the one
    before ends, directly and as one graph: the same results as with a wait after each call."""
    from paper_2609_04010_gb300 import binding as b
    B, H, D, P, V, steps = 5, 2, 128, 16, 1000, 6
    g = torch.Generator(device="cuda").manual_seed(gamma)

    def rand(*shape):
        return torch.randn(shape, device="cuda", generator=g)

    k, v = (rand(steps, B * gamma, H, D).bfloat16() for _ in range(2))
    q, logits = rand(steps, B, gamma, Hq, D).bfloat16(), rand(steps, B, gamma, V)
    block = torch.randint(0, V, (steps, B, gamma), device="cuda", generator=g, dtype=torch.int32)
    new = torch.full((B,), gamma, dtype=torch.int32, device="cuda")
    rep = torch.full((B,), 1.5, device="cuda")
    got = []
    for way in ("wait", "issue", "graph"):
        cache, scale = b.new_kv_cache_fp8(B * 10, H, P, D)
        table = torch.full((B, 10), -1, dtype=torch.int32, device="cuda")
        free = torch.arange(B * 10, dtype=torch.int32, device="cuda")
        count = torch.tensor([B * 10], dtype=torch.int32, device="cuda")
        kv_len = torch.zeros(B, dtype=torch.int32, device="cuda")
        rows = [torch.empty(n, dtype=torch.int32, device="cuda") for n in (B + 1, B * gamma)]
        out, lse, adj = torch.zeros_like(q), torch.zeros(q.shape[:4], device="cuda"), torch.zeros_like(logits)
        sa = b.slot_args(new, kv_len, kv_len, table, P, B * 10, free, count, count, *rows)
        sw = b.new_workspace(b.slot_workspace_size(sa))
        calls, held = [], [sa]
        for i in range(steps):
            pa = b.append_fp8_args(k[i], v[i], rows[1], cache, scale)
            ta = b.attn_fp8_args(q[i], cache, scale, table, kv_len, out[i], lse[i])
            ja = b.adjust_args(logits[i], adj[i], block[i], repetition=rep)
            tw = b.new_workspace(b.attn_fp8_workspace_size(ta))
            held += [pa, ta, ja, tw]
            calls += [lambda: b.map_slots_args(sa, sw), lambda pa=pa: b.append_kv_fp8_args(pa),
                      lambda ta=ta, tw=tw: b.verify_attention_fp8_args(ta, tw),
                      lambda ja=ja: b.adjust_logits_args(ja)]
        torch.cuda.synchronize()
        if way == "graph":
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                for c in calls:
                    c()
            graph.replay()
        else:
            for c in calls:
                c()
                if way == "wait":
                    torch.cuda.synchronize()
        torch.cuda.synchronize()
        got.append((out, lse, adj, cache.view(torch.uint8), scale, table, kv_len, count))
    for other in got[1:]:
        for x, y in zip(got[0], other):
            assert torch.equal(x, y)


def test_the_example_runs(capsys):
    example().main()
    assert "status: 0" in capsys.readouterr().out
