"""Attention of ragged chunks over the paged caches against the definition in 64 bits. Tolerances:
serving_reference.tolerance. AUTO is the tensor-core kernel where the call fits it."""

import numpy as np
import pytest
import torch

import serving_reference as ref

pytestmark = pytest.mark.gpu
AUTO, CUDA_CORES = 0, 1


def i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def make(new, ctx, Hq=8, Hkv=2, D=128, P=16, fp8=False, seed=0, spread=1.0, extra_rows=0, scales="powers"):
    """new[b] tokens after ctx[b] keys; a shuffled pool with unused pages of NaN."""
    r = np.random.default_rng(seed)
    g = torch.Generator(device="cuda").manual_seed(seed)
    new, ctx = np.asarray(new), np.asarray(ctx)
    lens = new + ctx
    need = -(-lens // P)
    N = int(need.sum()) + 3
    pool = r.permutation(N)
    table = np.full((len(new), max(1, int(need.max())) + 2), -1)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = pool[at:at + n]
        at += n
    unused = torch.from_numpy(pool[at:]).cuda()
    if fp8:
        x = torch.randn(N, Hkv, 2, P, D, generator=g, device="cuda") * spread
        e = torch.randint(-3, 4, (N, Hkv, 2), generator=g, device="cuda").float()
        scale = torch.exp2(e) * (1.0 if scales == "powers" else 1.0 + torch.rand(N, Hkv, 2, generator=g, device="cuda"))
        scale /= 4
        values = (x / scale[..., None, None]).clamp(-448, 448).to(torch.float8_e4m3fn)
        values.view(torch.uint8)[unused] = 0x7f
        cache = values, scale
    else:
        k, v = (torch.randn(N, Hkv, P, D, generator=g, device="cuda").bfloat16() for _ in range(2))
        k *= spread
        k[unused] = v[unused] = float("nan")
        cache = k, v
    starts = np.concatenate([[0], np.cumsum(new)])
    rows = int(starts[-1]) + extra_rows
    wide = torch.randn(rows, Hq + 3, D, generator=g, device="cuda").bfloat16()
    return dict(q=wide[:, 1:1 + Hq], cache=cache, table=i32(table), starts=starts.tolist(), lens=lens.tolist(),
                rows=rows, D=D, fp8=fp8)


def tail(c):
    """What the last pages hold past the sequences: NaN."""
    for b, n in enumerate(c["lens"]):
        P = c["cache"][0].shape[3 if c["fp8"] else 2]
        if n % P:
            page = int(c["table"][b, n // P])
            if c["fp8"]:
                c["cache"][0].view(torch.uint8)[page, :, :, n % P:] = 0x7f
            else:
                for x in c["cache"]:
                    x[page, :, n % P:] = float("nan")
    return c


def run(c, path=AUTO, ws=None, stream=None, **kw):
    from paper_2609_04010_gb300 import binding as b
    out = torch.full(c["q"].shape, 5.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full(c["q"].shape[:2], 5.0, device="cuda")
    a = b.chunk_attn_args(c["q"], c["cache"], c["table"], i32(c["starts"]), i32(c["lens"]), out, lse, path=path, **kw)
    if ws is None:
        ws = b.new_workspace(b.chunk_attn_workspace_size(a))
    b.chunk_attention_args(a, ws, stream)
    code, flags = b.read_device_status(ws, stream)
    return out, lse, code, flags


def check(c, path=AUTO, softmax_scale=0.0, causal=True, window=0, repeat=2):
    want = ref.chunk_attention(c["q"], c["cache"], c["table"], c["starts"], c["lens"], softmax_scale, causal, window)
    used = c["starts"][-1]
    first = None
    for _ in range(repeat):
        out, lse, code, flags = run(c, path, softmax_scale=softmax_scale, causal=causal, window=window)
        assert code == 0, flags
        ref.check_chunk((out[:used], lse[:used]), [x[:used] for x in want], c["D"], path != CUDA_CORES)
        assert bool((out[used:] == 5).all()) and bool((lse[used:] == 5).all()), "rows past the last were written"
        if first is not None:
            assert torch.equal(out, first[0]) and torch.equal(lse, first[1]), "two calls differ"
        first = out, lse


PATHS = [CUDA_CORES, AUTO]
HEADS = [(8, 8), (8, 2), (32, 8), (12, 3), (10, 2), (16, 1), (7, 1)]


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("D,P", [(64, 16), (128, 16), (128, 32), (64, 64), (128, 64)])
@pytest.mark.parametrize("causal", [True, False])
def test_ragged(path, fp8, D, P, causal):
    c = make([1, 0, 7, 64, 1, 130, 33], [0, 50, 3, 100, 511, 129, 0], D=D, P=P, fp8=fp8, seed=D + P, extra_rows=5)
    check(tail(c), path, causal=causal)


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("Hq,Hkv", HEADS)
def test_heads(path, fp8, Hq, Hkv):
    c = make([3, 90, 1, 41], [70, 0, 300, 257], Hq=Hq, Hkv=Hkv, fp8=fp8, seed=Hq)
    check(tail(c), path)


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("window", [1, 2, 16, 100, 128, 129, 1000])
@pytest.mark.parametrize("causal", [True, False])
def test_window(path, window, causal):
    c = make([1, 200, 5, 1], [700, 131, 0, 0], Hq=8, Hkv=2, seed=window, D=64)
    check(tail(c), path, causal=causal, window=window)


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("fp8", [False, True])
def test_pages_before_the_window_are_not_read(path, fp8):
    """Their table entries are gone, and what the window's first page holds before it is NaN."""
    c = make([40, 1], [600, 901], P=32, fp8=fp8, seed=5)
    for b, first in ((0, 600 - 99), (1, 901 - 99)):
        page = int(c["table"][b, first // 32])
        if fp8:
            c["cache"][0].view(torch.uint8)[page, :, :, :first % 32] = 0x7f
        else:
            for x in c["cache"]:
                x[page, :, :first % 32] = float("nan")
        c["table"][b, :first // 32] = -1
    check(c, path, window=100)


@pytest.mark.parametrize("n", [1, 2, 31, 63, 64, 65, 127, 128, 129, 255, 256, 257])
@pytest.mark.parametrize("path", PATHS)
def test_lengths_around_tiles(path, n):
    c = make([n, n, 1], [0, n, n - 1], Hq=4, Hkv=2, D=64, seed=n)
    check(tail(c), path)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("shape", ["one token", "few tokens", "prompt", "mixed"])
def test_long(shape, fp8):
    new, ctx = {"one token": ([1], [16000]), "few tokens": ([5, 3], [9000, 20001]),
                "prompt": ([2100], [3001]), "mixed": ([1] * 30 + [700], list(range(10, 6010, 200)) + [900])}[shape]
    c = make(new, ctx, Hq=8, Hkv=2, fp8=fp8, seed=len(new))
    check(tail(c))


@pytest.mark.parametrize("batch", [1, 100, 1500])
def test_single_tokens(batch):
    r = np.random.default_rng(batch)
    c = make([1] * batch, r.integers(0, 300 if batch > 100 else 3000, batch), Hq=4, Hkv=1, D=64, seed=batch)
    check(tail(c))


@pytest.mark.parametrize("path", PATHS)
def test_groups_too_wide_for_a_tile(path):
    """Hq / Hkv = 200: on CUDA cores whatever the path asked for; tensor cores refuse it."""
    from paper_2609_04010_gb300 import binding as b
    c = make([3, 1], [40, 5], Hq=200, Hkv=1, D=64)
    want = ref.chunk_attention(c["q"], c["cache"], c["table"], c["starts"], c["lens"])
    out, lse, code, _ = run(c, path)
    assert code == 0
    ref.check_chunk((out, lse), want, 64, False)
    with pytest.raises(b.SpecError) as e:
        run(c, b.ATTN_TENSOR_CORES)
    assert e.value.code in (1, 2)


@pytest.mark.parametrize("group", [64, 128, 100])
def test_wide_groups(group):
    check(make([3, 1, 9], [40, 500, 0], Hq=group, Hkv=1, D=64, seed=group))


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_hidden_values_do_not_reach_a_row(path, fp8, value):
    """A token's bad key or value reaches only the rows that see it."""
    if fp8 and value != value or not fp8:
        c = make([200, 70], [100, 300], Hq=4, Hkv=2, fp8=fp8, seed=11)
        at = 100 + 150
        page = int(c["table"][0, at // 16])
        if fp8:
            c["cache"][0].view(torch.uint8)[page, 1, 1, at % 16, 5] = 0x7f
            c["cache"][0].view(torch.uint8)[int(c["table"][1, 330 // 16]), 0, 0, 330 % 16, 7] = 0x7f
        else:
            c["cache"][1][page, 1, at % 16, 5] = value
            c["cache"][0][int(c["table"][1, 330 // 16]), 0, 330 % 16, 7] = float("nan")
        want = ref.chunk_attention(c["q"], c["cache"], c["table"], c["starts"], c["lens"])[0]
        out, lse, code, _ = run(c, path)
        assert code == 0
        assert not torch.isnan(out[:150]).any() and torch.isfinite(out[:150]).all()
        assert bool((~torch.isfinite(out[150:200, 2:, 5])).all())      # rows that see it
        assert torch.isfinite(out[150:200, 2:, :5]).all() and torch.isfinite(out[150:200, :2]).all()
        assert torch.isfinite(out[200:230]).all() and torch.isnan(out[230:, :2]).all()
        ok = torch.isfinite(want)
        assert float((out.double() - want).abs()[ok].max()) < 0.05


@pytest.mark.parametrize("path", PATHS)
def test_window_hides_bad_values_behind(path):
    c = make([150], [200], Hq=4, Hkv=2, seed=12)
    c["cache"][1][int(c["table"][0, 210 // 16]), 0, 210 % 16, 9] = float("nan")
    out, _, code, _ = run(c, path, window=64)
    seen = torch.arange(150, device="cuda") + 200
    hit = (seen >= 210) & (seen < 210 + 64)
    assert code == 0 and torch.isnan(out[hit][:, :2, 9]).all()
    assert torch.isfinite(out[~hit]).all() and torch.isfinite(out[:, 2:]).all()


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("size", [1e2, 1e9, 1e17])
def test_large_scores_stay_finite(path, size):
    """Scores far past 2^24: nearly all the weight on one key, finite outputs, right where it is clear."""
    c = make([140, 1], [20, 700], Hq=4, Hkv=2, seed=13)
    c["cache"][0].mul_(size)
    want, _, _, _ = ref.chunk_attention(c["q"], c["cache"], c["table"], c["starts"], c["lens"])
    out, lse, code, _ = run(c, path)
    assert code == 0 and torch.isfinite(out).all()
    if size > 1e3:
        close = ((out.double() - want).abs() < 2.0 ** -6 * (1 + want.abs())).all(-1).float().mean()
        assert float(close) > 0.99
    assert bool((out.abs() <= 5.5).all())


@pytest.mark.parametrize("path", PATHS)
def test_scores_of_infinity(path):
    """A row whose only key has a score of -inf: NaN and -inf, as softmax has it; its neighbours stay."""
    c = make([2, 2], [0, 0], Hq=1, Hkv=1, D=64, seed=14)
    page = int(c["table"][0, 0])
    c["q"][0] = 1
    c["cache"][0][page, 0, 0] = float("-inf")
    out, lse, code, _ = run(c, path)
    assert code == 0 and torch.isnan(out[0]).all() and lse[0, 0] == float("-inf")
    assert torch.isfinite(out[2:]).all()


@pytest.mark.parametrize("path", PATHS)
def test_rising_scores(path):
    """Each key's score above the one before: every tile raises the maximum."""
    c = make([300], [900], Hq=4, Hkv=1, D=64, seed=15)
    c["q"][:] = 1
    for i in range(1200):
        c["cache"][0][int(c["table"][0, i // 16]), 0, i % 16] = i / 64.0
    check(c, path, softmax_scale=0.5)


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("scale", [0.01, 1.0, 7.5])
def test_softmax_scale(path, scale):
    check(make([60, 3], [70, 400], seed=16, D=64), path, softmax_scale=scale)


@pytest.mark.parametrize("path", PATHS)
def test_any_scales_of_the_8_bit_cache(path):
    """Scales that are no powers of two."""
    check(make([70, 5], [100, 900], fp8=True, scales="any", seed=17, spread=0.3), path)


# ----------------------------------------------------------------------------------
# What cannot be served
# ----------------------------------------------------------------------------------
@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("fp8", [False, True])
def test_bad_pages(path, fp8):
    from paper_2609_04010_gb300 import binding as b
    c = make([5, 200, 1, 300], [50, 60, 700, 0], fp8=fp8, seed=18)
    good, _, _, _ = run(c, path)
    c["table"][1, 255 // 16], c["table"][2, 0] = -1, 10 ** 9
    out, lse, code, flags = run(c, path)
    s = c["starts"]
    assert code == 5 and flags == b.FLAG_BAD_PAGE
    for i in range(4):
        rows = slice(s[i], s[i + 1])
        if i in (1, 2):
            assert not out[rows].any() and bool((lse[rows] == float("-inf")).all())
        else:
            assert torch.equal(out[rows], good[rows])


@pytest.mark.parametrize("path", PATHS)
def test_bad_lengths(path):
    from paper_2609_04010_gb300 import binding as b
    c = make([5, 20, 1, 30], [50, 60, 70, 0], seed=19)
    good, good_lse, _, _ = run(c, path)
    c["lens"] = [55, 19, 2 ** 30, 30]
    out, lse, code, flags = run(c, path)
    s = c["starts"]
    assert code == 5 and flags == b.FLAG_BAD_KV_LEN
    for i in range(4):
        rows = slice(s[i], s[i + 1])
        if i in (1, 2):
            assert not out[rows].any() and bool((lse[rows] == float("-inf")).all())
        else:
            assert torch.equal(out[rows], good[rows]) and torch.equal(lse[rows], good_lse[rows])


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("starts", [[0, 5, 5, 3, 40], [-1, 5, 25, 26, 56], [0, 5, 25, 26, 57],
                                    [0, 56, 0, 56, 0], [60, 70, 80, 90, 100], [2 ** 31 - 1, -2 ** 31, 0, 3, 3]])
def test_bad_row_starts(path, starts):
    """Rows out of order or out of range: nothing is read or written out of range, and flagged."""
    from paper_2609_04010_gb300 import binding as b
    c = make([5, 20, 1, 30], [50, 60, 70, 0], seed=20)
    c["starts"] = starts
    c["lens"] = [100, 100, 100, 60]
    c["table"][:] = c["table"][:, :1].clamp_min(0)
    _, _, code, flags = run(c, path)
    assert code == 5 and flags & b.FLAG_BAD_KV_LEN


@pytest.mark.parametrize("path", PATHS)
def test_without_rows(path):
    c = make([0, 0], [5, 0], seed=21, extra_rows=4)
    out, lse, code, _ = run(c, path)
    assert code == 0 and bool((out == 5).all()) and bool((lse == 5).all())
    c["q"], c["rows"] = c["q"][:0], 0
    assert run(c, path)[2] == 0


# ----------------------------------------------------------------------------------
# How it is called
# ----------------------------------------------------------------------------------
def test_no_lse_and_the_plain_call():
    from paper_2609_04010_gb300 import binding as b
    c = make([9, 1], [30, 80], seed=22)
    out, lse, _, _ = run(c)
    again, none = b.chunk_attention(c["q"], c["cache"], c["table"], i32(c["starts"]), i32(c["lens"]), want_lse=False)
    assert none is None and torch.equal(again, out)


def test_streams_and_workspaces():
    """Two calls at once on two streams, each with its workspace."""
    from paper_2609_04010_gb300 import binding as b
    cases = [make([300, 1, 1], [700, 3000, 41], seed=s) for s in (23, 24)]
    want = [run(c)[:2] for c in cases]
    outs, streams = [], [torch.cuda.Stream() for _ in cases]
    for _ in range(5):
        for c, s in zip(cases, streams):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                outs.append(b.chunk_attention(c["q"], c["cache"], c["table"], i32(c["starts"]), i32(c["lens"])))
    torch.cuda.synchronize()
    for i, (o, l) in enumerate(outs):
        assert torch.equal(o, want[i % 2][0]) and torch.equal(l, want[i % 2][1])


@pytest.mark.parametrize("fp8", [False, True])
def test_graphs_share_a_workspace(fp8):
    """Two captured calls of one configuration, replayed in turn on one stream, other lengths each time."""
    from paper_2609_04010_gb300 import binding as b
    c = make([1, 40, 1, 200], [900, 0, 1, 350], fp8=fp8, seed=25)
    lens, starts = i32(c["lens"]), i32(c["starts"])
    outs = [torch.empty(c["q"].shape, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    args = [b.chunk_attn_args(c["q"], c["cache"], c["table"], starts, lens, o, causal=i == 0) for i, o in enumerate(outs)]
    ws = b.new_workspace(b.chunk_attn_workspace_size(args[0]))
    for a in args:
        b.chunk_attention_args(a, ws)
    torch.cuda.synchronize()
    graphs = []
    for a in args:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            b.chunk_attention_args(a, ws)
        graphs.append(g)
    for shift in (0, 7, 40):
        now = [max(n - shift, s1 - s0) for n, s0, s1 in zip(c["lens"], c["starts"], c["starts"][1:])]
        lens.copy_(i32(now))
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for i in range(2):
            want = ref.chunk_attention(c["q"], c["cache"], c["table"], c["starts"], now, causal=i == 0)
            ref.check_chunk((outs[i], None), want, c["D"], True)


def test_workspace_of_another_device_type_is_refused():
    from paper_2609_04010_gb300 import binding as b
    c = make([2], [3], seed=26)
    a = b.chunk_attn_args(c["q"], c["cache"], c["table"], i32(c["starts"]), i32(c["lens"]), torch.empty_like(c["q"].contiguous()))
    with pytest.raises(ValueError):
        b.chunk_attention_args(a, torch.zeros(1 << 20, dtype=torch.uint8))
    with pytest.raises(b.SpecError):
        b.chunk_attention_args(a, b.new_workspace(256))


def test_waits_run_out():
    """With idle copy producers every wait ends, the status says so, and the workspace serves on."""
    from paper_2609_04010_gb300 import binding as b
    c = make([1, 300, 2], [900, 50, 10], seed=27)
    out, lse = torch.empty(c["q"].shape, dtype=torch.bfloat16, device="cuda"), torch.empty(c["q"].shape[:2], device="cuda")
    a = b.chunk_attn_args(c["q"], c["cache"], c["table"], i32(c["starts"]), i32(c["lens"]), out, lse)
    ws = b.new_workspace(b.chunk_attn_workspace_size(a))
    b.test_chunk_attention_wait_timeout_args(a, ws)
    assert b.read_device_status(ws) == (6, b.FLAG_TIMEOUT)
    b.chunk_attention_args(a, ws)
    assert b.read_device_status(ws)[0] == 0
    want = ref.chunk_attention(c["q"], c["cache"], c["table"], c["starts"], c["lens"])
    ref.check_chunk((out, lse), want, 128, True)


@pytest.mark.parametrize("D,P", [(64, 16), (128, 16), (64, 64)])
def test_scales_of_pages_far_apart(D, P):
    """Neighbouring pages' scales 2^12 apart, in long contexts, for single tokens and chunks: each tile's
    scores and weights meet their own page's, call after call."""
    c = make([1, 300, 1, 20, 65], [6000, 2500, 900, 4000, 0], Hq=8, Hkv=2, D=D, P=P, fp8=True, seed=28)
    values, scale = c["cache"]
    r = np.random.default_rng(28)
    scale.copy_(torch.from_numpy(np.exp2(r.integers(-12, 1, scale.shape)).astype(np.float32)))
    values.view(torch.uint8).copy_(torch.randint(0, 0x60, values.shape, dtype=torch.uint8, device="cuda"))
    check(tail(c), softmax_scale=0.02, repeat=6)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("new", [3, 64, 200])
def test_hidden_values_in_units_that_blocks_share(fp8, new):
    """A value that is not finite, seen by later tokens only, behind a context that many blocks share: the
    unit is computed again, and its joined parts must not come over that."""
    c = make([new], [30000], Hq=8, Hkv=2, D=128, P=16, fp8=fp8, seed=29, spread=0.3)
    for at, h in ((30000 + new - 1, 0), (30000 + new // 2, 1)):
        page, slot = int(c["table"][0, at // 16]), at % 16
        if fp8:
            c["cache"][0].view(torch.uint8)[page, h, 1, slot, 3] = 0x7f
        else:
            c["cache"][1][page, h, slot, 3] = float("nan")
    for _ in range(6):
        check(c, repeat=1)
