"""Attention of ragged chunks over the 8-bit cache, held to what the header promises (weights off by 2^-11,
chunk_reference.check_8_bit), at lengths, windows, groups and values where it can go wrong."""

import math

import numpy as np
import pytest
import torch

import chunk_reference as ref
import serving_reference
from test_gpu_chunk import i32, make, run, tail

pytestmark = pytest.mark.gpu
AUTO, CUDA_CORES = 0, 1


def check(c, path=AUTO, repeat=2, **kw):
    want = ref.attend(c, **kw)
    used, first = c["starts"][-1], None
    for _ in range(repeat):
        out, lse, code, flags = run(c, path, **kw)
        assert code == 0, flags
        ref.check((out[:used], lse[:used]), [x[:used] for x in want], c, path == CUDA_CORES)
        assert bool((out[used:] == 5).all()) and bool((lse[used:] == 5).all()), "rows past the last were written"
        assert first is None or torch.equal(out.nan_to_num(7), first[0]) and torch.equal(lse.nan_to_num(7), first[1])
        first = out.nan_to_num(7), lse.nan_to_num(7)
    return want


@pytest.mark.parametrize("D,P", [(64, 16), (128, 16), (128, 32), (64, 64), (128, 64)])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("scales", ["powers", "any"])
def test_ragged(D, P, causal, scales):
    c = make([1, 0, 7, 64, 1, 130, 33], [0, 50, 3, 100, 511, 129, 0], D=D, P=P, fp8=True, seed=D + P, extra_rows=5,
             scales=scales)
    check(tail(c), causal=causal)


@pytest.mark.parametrize("path", [CUDA_CORES, AUTO])
@pytest.mark.parametrize("n", [1, 2, 31, 63, 64, 65, 127, 128, 129, 255, 256, 257])
def test_lengths_around_tiles(path, n):
    check(tail(make([n, n, 1], [0, n, n - 1], Hq=4, Hkv=2, D=64, fp8=True, seed=n)), path)


@pytest.mark.parametrize("path", [CUDA_CORES, AUTO])
@pytest.mark.parametrize("window", [1, 2, 16, 100, 128, 129, 1000])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("D", [64, 128])
def test_window(path, window, causal, D):
    check(tail(make([1, 200, 5, 1], [700, 131, 0, 0], Hq=8, Hkv=2, fp8=True, seed=window, D=D)), path, causal=causal,
          window=window)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("group", [17, 33, 64, 100, 127, 128])
def test_wide_groups(fp8, D, group):
    check(make([3, 1, 9, 70], [40, 500, 0, 1000], Hq=group, Hkv=1, D=D, fp8=fp8, seed=group))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("batch,new", [(129, 1), (200, 3), (1500, 1), (2, 3000)])
def test_many_sequences_or_units(D, batch, new):
    """Past 128 of either, where the set-up takes its large block and the queries' blocks are as large."""
    r = np.random.default_rng(batch)
    check(tail(make([new] * batch, r.integers(0, 300, batch), Hq=16 if batch == 2 else 4, Hkv=1, D=D, fp8=True, seed=batch)))


@pytest.mark.parametrize("path", [CUDA_CORES, AUTO])
@pytest.mark.parametrize("D", [64, 128])
def test_rising_scores(path, D):
    """Each page's keys above the one before: every tile raises the maximum, by less and by more than the
    weights' room."""
    for step in (0.5, 3.0, 40.0):
        c = make([300], [900], Hq=4, Hkv=1, D=D, fp8=True, seed=65)
        c["q"][:] = 1
        values, scale = c["cache"]
        for i in range(75):
            page = int(c["table"][0, i])
            values.view(torch.uint8)[page, 0, 0] = 0x38  # 1
            scale[page, 0, 0] = (i + 1) * step / D
        check(c, path, softmax_scale=0.5)


@pytest.mark.parametrize("path", [CUDA_CORES, AUTO])
@pytest.mark.parametrize("scale", [0.01, 1.0, 7.5])
def test_softmax_scale(path, scale):
    check(make([60, 3], [70, 400], seed=66, D=64, fp8=True, spread=0.5), path, softmax_scale=scale)


@pytest.mark.parametrize("path", [CUDA_CORES, AUTO])
@pytest.mark.parametrize("size", [1e3, 1e9, 1e17])
def test_large_scores_stay_finite(path, size):
    """Scores far past 2^24: finite outputs, off by what the scores' roundings can move. Scores that are off by
    at most s change the outputs by sum w_k (e^d_k / Z - 1) (v_k - out), Z = sum w_k e^d_k, |d_k| <= s: at most
    (e^2s - 1) sum w_k |v_k - out|, which is small where one key has nearly all the weight."""
    c = make([140, 1], [20, 700], Hq=4, Hkv=2, fp8=True, seed=67)
    c["cache"][1][:, :, 0] *= size
    out64, _, spread, reach, steps = ref.attend(c)
    out, lse, code, _ = run(c, path)
    assert code == 0 and torch.isfinite(out).all() and torch.isfinite(lse).all()
    score = (128 + 5) * 2.0 ** -24 * reach + 2.0 ** -17
    moved = torch.expm1((2 * score).clamp(max=700.0))[..., None] * from_the_output(c, out64)
    tol = 2.0 ** -8 * out64.abs() + 2.0 ** -11 * spread + 2.0 ** -33 * steps + moved + 1e-30
    err = (out.double() - out64).abs()
    assert bool((err <= tol * (1 + 2.0 ** -7)).all())
    close = (err < 2.0 ** -6 * (1 + out64.abs())).all(-1).float().mean()
    assert size < 1e6 or float(close) > 0.99


def from_the_output(c, out):
    """sum_k w_k |v_k - out|, causal, scale 1 / sqrt(D)."""
    dev = torch.zeros_like(out)
    for b, n in enumerate(c["lens"]):
        r0, r1 = c["starts"][b], c["starts"][b + 1]
        pages = c["table"][b, :-(-n // 16)].long()
        for h in range(out.shape[1]):
            k, v = (serving_reference.keys(c["cache"], pages, h // 2, i, n) for i in (0, 1))
            x = c["q"][r0:r1, h].double() @ k.T / math.sqrt(c["D"])
            seen = torch.arange(n, device="cuda")[None] <= torch.arange(n - (r1 - r0), n, device="cuda")[:, None]
            w = torch.softmax(torch.where(seen, x, -math.inf), -1)
            for r in range(r1 - r0):
                dev[r0 + r, h] = (w[r][:, None] * (v - out[r0 + r, h]).abs()).sum(0)
    return dev


@pytest.mark.parametrize("path", [CUDA_CORES, AUTO])
@pytest.mark.parametrize("fp8", [False, True])
def test_moderate_scores_hold_the_tolerance(path, fp8):
    """Scores of some hundreds: the tolerance's linear part is still below a tenth."""
    c = make([140, 1], [20, 700], Hq=4, Hkv=2, fp8=fp8, seed=68)
    if fp8:
        c["cache"][1][:, :, 0] *= 20
    else:
        c["cache"][0].mul_(20)
    want = check(c, path)
    assert 50 < float(want[3].max()) < 5000


@pytest.mark.parametrize("path", [CUDA_CORES, AUTO])
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("new,ctx", [(1, 0), (3, 200), (1, 20000), (200, 900)])
def test_infinite_queries(path, fp8, new, ctx):
    """A query element of -inf on keys that are all positive there: scores of -inf, out NaN and a
    log-sum-exp of -inf; one of +inf: NaN. Other rows keep every bit."""
    c = make([new, 2], [ctx, 300], Hq=4, Hkv=2, D=128, fp8=fp8, seed=69)
    if fp8:
        c["cache"][0].view(torch.uint8)[:, :, 0, :, 9] = 0x30
    else:
        c["cache"][0][..., 9] = 0.5
    good, good_lse, _, _ = run(c, path)
    c["q"][0, 1, 9], c["q"][new, 3, 9] = float("-inf"), float("inf")
    out, lse, code, _ = run(c, path)
    assert code == 0 and torch.isnan(out[0, 1]).all() and lse[0, 1] == float("-inf") and torch.isnan(out[new, 3]).all()
    other = torch.ones(out.shape[:2], dtype=torch.bool, device="cuda")
    other[0, 1] = other[new, 3] = False
    assert torch.equal(out[other], good[other]) and torch.equal(lse[other], good_lse[other])


@pytest.mark.parametrize("size", [3e38, 1e-30, 1e-38, 0.0])
def test_queries_at_the_ends_of_bf16(size):
    """Their largest element near the type's largest and smallest values: the softmax's scale brings the
    scores back (where it can), and nothing overflows on the way."""
    c = make([70, 1], [40, 900], Hq=4, Hkv=2, D=64, fp8=True, seed=70)
    c["q"].copy_((c["q"].float() / c["q"].float().abs().amax() * size).bfloat16())
    scale = min(max(1 / size, 1e-37), 1e29) if size else 1.0
    check(c, softmax_scale=scale)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("D", [64, 128])
def test_waits_run_out(fp8, D):
    """With idle copy producers every wait ends, the status says so, and the workspace serves on."""
    from paper_2609_04010_gb300 import binding as b
    c = make([1, 300, 2], [900, 50, 10], D=D, fp8=fp8, seed=71)
    out, lse = torch.empty(c["q"].shape, dtype=torch.bfloat16, device="cuda"), torch.empty(c["q"].shape[:2], device="cuda")
    a = b.chunk_attn_args(c["q"], c["cache"], c["table"], i32(c["starts"]), i32(c["lens"]), out, lse)
    ws = b.new_chunk_attn_workspace(a)
    for _ in range(2):
        b.test_chunk_attention_wait_timeout_args(a, ws)
        assert b.read_device_status(ws) == (6, b.FLAG_TIMEOUT)
        b.chunk_attention_args(a, ws)
        assert b.read_device_status(ws) == (0, 0)
        ref.check((out, lse), ref.attend(c), c)
