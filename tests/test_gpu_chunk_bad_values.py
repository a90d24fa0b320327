"""NaN among keys, values and queries of attention of chunks: what a row's mask hides does not reach it,
however many units hold such values; what a row sees does, however small its weight is and wherever
the work is cut."""

import pytest
import torch

import chunk_reference as ref
from test_gpu_chunk import make, run

pytestmark = pytest.mark.gpu
AUTO, CUDA_CORES = 0, 1


def spoil(c, kind, b, at, heads=slice(None), dims=slice(None)):
    """Keys (0) or values (1) of sequence b at token `at` become NaN."""
    P = c["cache"][0].shape[3 if c["fp8"] else 2]
    page = int(c["table"][b, at // P])
    if c["fp8"]:
        c["cache"][0].view(torch.uint8)[page, heads, kind, at % P, dims] = 0x7f
    else:
        c["cache"][kind][page, heads, at % P, dims] = float("nan")


def check(c, path=AUTO, repeat=2, **kw):
    want = ref.attend(c, **kw)
    for _ in range(repeat):
        out, lse, code, flags = run(c, path, **kw)
        assert code == 0, flags
        ref.check((out, lse), want, c, path == CUDA_CORES)
    return want


# ----------------------------------------------------------------------------------
# Hidden values, in more units than a list of one note per unit and warp would hold
# ----------------------------------------------------------------------------------
@pytest.mark.parametrize("fp8", [True, False])
@pytest.mark.parametrize("D", [64, 128])
def test_hidden_values_in_every_unit(fp8, D):
    """64 sequences of 16 new tokens, 8 KV heads: in each unit a value of the tile's first half and one of
    its second that only later tokens see."""
    c = make([16] * 64, [56 + 128 * (i % 3) for i in range(64)], Hq=32, Hkv=8, D=D, fp8=fp8, seed=41)
    for b in range(64):
        base = c["lens"][b] - 16 - 56
        spoil(c, 1, b, base + 60, dims=slice(0, 1))
        spoil(c, 1, b, base + 66, dims=slice(1, 2))
    want = check(c, repeat=4)
    assert bool(torch.isfinite(want[0][:, :, 2:]).all()) and not bool(torch.isfinite(want[0]).all())


@pytest.mark.parametrize("fp8", [True, False])
def test_hidden_values_under_a_window(fp8):
    """Every 32nd value of a long chunk NaN, a window of 8 tokens."""
    c = make([1500, 900], [1000, 77], Hq=8, Hkv=8, D=64, fp8=fp8, seed=42)
    for b, n in enumerate(c["lens"]):
        for at in range(5, n, 32):
            spoil(c, 1, b, at, dims=slice(0, 1))
    want = check(c, repeat=4, window=8)
    assert 0.5 < float(torch.isfinite(want[0][:, :, 0]).float().mean()) < 0.9


# ----------------------------------------------------------------------------------
# What a row sees, in units that several blocks share
# ----------------------------------------------------------------------------------
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("new", [1, 40, 200])
def test_bad_keys_fill_a_part(fp8, new):
    """Keys NaN over whole tiles, so that all scores of some block's part are: not a part without keys."""
    c = make([new], [30000], Hq=4, Hkv=2, D=128, fp8=fp8, seed=43)
    P = 16
    for page in range(7168 // P, 9728 // P):  # 20 tiles
        at = int(c["table"][0, page])
        if fp8:
            c["cache"][0].view(torch.uint8)[at, 0, 0] = 0x7f
        else:
            c["cache"][0][at, 0] = float("nan")
    want = check(c)
    assert bool(torch.isnan(want[0][:, :2]).all()) and bool(torch.isfinite(want[0][:, 2:]).all())


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("new", [1, 200])
def test_a_last_key_alone_in_its_tile(fp8, new):
    """The last part's tile holds one key that the row sees, and it is NaN."""
    for ctx in (30080 - new + 1, 12800 - new + 1):  # the last token begins a tile
        c = make([new], [ctx], Hq=4, Hkv=2, D=64, fp8=fp8, seed=44)
        assert c["lens"][0] % 128 == 1
        spoil(c, 0, 0, c["lens"][0] - 1, heads=1)
        want = check(c)
        assert bool(torch.isnan(want[0][-1, 2:]).all()) and bool(torch.isfinite(want[0][-1, :2]).all())


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("new,ctx", [(1, 30000), (1, 100), (3, 9000), (200, 9000), (70, 0)])
def test_a_bad_query(fp8, new, ctx):
    """A NaN query row: NaN and NaN, and no other row is touched."""
    c = make([new, 2], [ctx, 300], Hq=4, Hkv=2, D=128, fp8=fp8, seed=45)
    c["q"][new // 2, 1, 77] = float("nan")
    want = check(c)
    assert bool(torch.isnan(want[0][new // 2, 1]).all()) and bool(torch.isnan(want[1][new // 2, 1]))
    assert int(torch.isnan(want[0]).sum()) == 128


# ----------------------------------------------------------------------------------
# What a row sees with a weight that underflows
# ----------------------------------------------------------------------------------
def sink(c, b, tokens):
    """Queries of ones, and keys of these tokens far below: weights below 2^-150."""
    c["q"][:] = 1
    for at in tokens:
        page = int(c["table"][b, at // 16])
        if c["fp8"]:
            c["cache"][0].view(torch.uint8)[page, :, 0, at % 16] = 0xfe  # -448
            c["cache"][1][page, :, 0] = 0.125
        else:
            c["cache"][0][page, :, at % 16] = -32


@pytest.mark.parametrize("path", [CUDA_CORES, AUTO])
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("new,ctx,low,bad", [
    (1, 200, range(128, 201), 140), (1, 200, range(0, 128), 5), (1, 30000, range(20000, 20100), 20050), (200, 300, [50], 50),
    (64, 200, [130], 130)])
def test_bad_values_of_no_weight(path, fp8, new, ctx, low, bad):
    c = make([new, 3], [ctx, 40], Hq=4, Hkv=2, D=64, fp8=fp8, seed=46, spread=0.25)
    sink(c, 0, low)
    spoil(c, 1, 0, bad, heads=1, dims=slice(7, 8))
    want = check(c, path)
    assert bool(torch.isnan(want[0][:new, 2:, 7]).all()) and int(torch.isnan(want[0]).sum()) == 2 * new


@pytest.mark.parametrize("path", [CUDA_CORES, AUTO])
@pytest.mark.parametrize("fp8", [False, True])
def test_bad_values_of_no_weight_beside_hidden_ones(path, fp8):
    """A unit that is computed again because of the one keeps the other."""
    c = make([70], [300], Hq=4, Hkv=2, D=64, fp8=fp8, seed=47, spread=0.25)
    sink(c, 0, [33])
    spoil(c, 1, 0, 33, heads=0, dims=slice(7, 8))
    spoil(c, 1, 0, 350, heads=0, dims=slice(9, 10))
    want = check(c, path)
    assert bool(torch.isnan(want[0][:, :2, 7]).all()) and bool(torch.isfinite(want[0][:50, :, 9]).all())
    assert bool(torch.isnan(want[0][50:, :2, 9]).all())
