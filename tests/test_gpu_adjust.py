"""Penalties, biases and grammar masks on logits against the 64-bit host reference.

Tolerance: the kernel makes at most five fp32 roundings per logit (division or product,
count product, two subtractions, bias), each at most 2^-24 of its result's magnitude M, which
the inputs bound; a bf16 result is then rounded by at most 2^-9 of itself."""

import numpy as np
import pytest
import torch

import fp8_reference as ref

pytestmark = pytest.mark.gpu


def dev(a, dtype):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a, dtype=dtype)).cuda()


def make(B, G, V, seed, f32=True, hist=40, bias=6, mask=True, density=0.5):
    r = np.random.default_rng(seed)
    x = (r.standard_normal((B, G, V)) * 3).astype(np.float32)
    if not f32:
        x = torch.from_numpy(x).to(torch.bfloat16).float().numpy()
    c = dict(x=x, f32=f32, block=np.minimum(V * r.random((B, G)) ** 3, V - 1).astype(np.int32))
    if hist:
        c["history"] = np.minimum(V * r.random((B, hist)) ** 3, V - 1).astype(np.int32)
        c["history_len"] = r.integers(0, hist + 1, B).astype(np.int32)
        c["prompt_len"] = (c["history_len"] * r.random(B)).astype(np.int32)
    c["repetition"] = (1 + r.random(B)).astype(np.float32)
    c["frequency"], c["presence"] = r.random(B).astype(np.float32), r.random(B).astype(np.float32)
    if bias:
        c["bias_tokens"] = r.integers(0, V, (B, bias)).astype(np.int32)
        c["bias_values"] = r.normal(0, 4, (B, bias)).astype(np.float32)
    if mask:
        W = (V + 31) // 32
        bits = r.random((B, G, W * 32)) < density
        c["allowed"] = np.packbits(bits, axis=-1, bitorder="little").view(np.int32).reshape(B, G, W)
    return c


ARGS = ("block", "history", "history_len", "prompt_len", "repetition", "frequency", "presence",
        "bias_tokens", "bias_values", "allowed")


def run(c, block_shift=0, in_place=False):
    from paper_2609_04010_gb300 import binding as b
    x = torch.from_numpy(c["x"]).cuda()
    if not c["f32"]:
        x = x.to(torch.bfloat16)
    keep = x.clone()
    t = {k: dev(c.get(k), None if c.get(k) is None else c[k].dtype) for k in ARGS}
    t["block_tokens"] = t.pop("block")
    out = b.adjust_logits(x, block_shift=block_shift, out=x if in_place else None, **t)
    torch.cuda.synchronize()
    if not in_place:
        assert torch.equal(x.view(torch.uint8), keep.view(torch.uint8))
    return out.float().cpu().numpy().astype(np.float64)


def check(c, block_shift=0, in_place=False):
    got = run(c, block_shift, in_place)
    want = ref.adjust(c["x"], block_shift=block_shift, **{k: c.get(k) for k in ARGS})
    G = c["x"].shape[1]
    n = (c["history"].shape[1] if c.get("history") is not None else 0) + G
    fmax = 0 if c.get("frequency") is None else np.abs(c["frequency"]).max()
    rmax = 1 if c.get("repetition") is None else np.abs(c["repetition"]).max()
    bmax = 0 if c.get("bias_values") is None else np.abs(c["bias_values"]).max()
    x = np.where(np.isfinite(c["x"]), np.abs(c["x"]), 0)
    M = x * max(rmax, 1) + fmax * n + 1 + bmax
    tol = 5 * 2.0 ** -24 * M
    if not c["f32"]:
        tol = tol + 2.0 ** -8 * np.abs(np.where(np.isfinite(want), want, 0))
    fin = np.isfinite(want)
    assert np.array_equal(fin, np.isfinite(got))
    assert np.array_equal(got[~fin & ~np.isnan(want)], want[~fin & ~np.isnan(want)])
    assert np.array_equal(np.isnan(got), np.isnan(want))
    assert (np.abs(got[fin] - want[fin]) <= tol[fin]).all()
    # what nothing touches comes through bit for bit
    return got, want


@pytest.mark.parametrize("f32", [True, False])
@pytest.mark.parametrize("V", [1, 7, 31, 32, 33, 1000, 1024, 4096, 4097, 4103, 9001])
def test_vocabularies(V, f32):
    check(make(2, 3, V, seed=V, f32=f32))


@pytest.mark.parametrize("f32", [True, False])
@pytest.mark.parametrize("B,G", [(1, 1), (1, 64), (5, 1), (7, 16), (3, 33)])
def test_shapes(B, G, f32):
    check(make(B, G, 517, seed=B * 100 + G, f32=f32))
    check(make(B, G, 1024, seed=B * 100 + G, f32=f32), in_place=True)


@pytest.mark.parametrize("f32", [True, False])
@pytest.mark.parametrize("shift", [0, 1])
def test_block_shift_and_in_place(shift, f32):
    c = make(3, 8, 320, seed=4, f32=f32)
    c["block"][:] = np.random.default_rng(1).integers(0, 9, c["block"].shape)  # repeats in the block
    check(c, shift)
    check(c, shift, in_place=True)


@pytest.mark.parametrize("drop", ["block", "history", "prompt_len", "repetition", "frequency",
                                  "presence", "bias_tokens", "allowed"])
def test_optional_parts(drop):
    c = make(3, 5, 700, seed=9)
    gone = {"history": ("history", "history_len", "prompt_len"),
            "bias_tokens": ("bias_tokens", "bias_values")}.get(drop, (drop,))
    for k in gone:
        c[k] = None
    check(c)


def test_only_a_mask_and_nothing_at_all():
    c = make(2, 4, 515, seed=10, hist=0, bias=0)
    for k in ("block", "repetition", "frequency", "presence"):
        c[k] = None
    got, want = check(c)
    assert np.array_equal(got, want)
    c["allowed"] = None
    got, _ = check(c)
    assert np.array_equal(got, c["x"].astype(np.float64))


@pytest.mark.parametrize("density", [0.0, 0.001, 0.999, 1.0])
def test_mask_densities_and_empty_rows(density):
    c = make(3, 6, 2080, seed=11, density=density)
    got, _ = check(c)
    if density == 0.0:
        assert np.all(got == -np.inf)


def test_special_values():
    """NaN and infinities: hidden ones become -inf, visible ones follow fp32 arithmetic."""
    c = make(2, 4, 600, seed=12)
    c["x"][:, :, 0:400:7] = np.nan
    c["x"][:, :, 1:400:7] = np.inf
    c["x"][:, :, 2:400:7] = -np.inf
    c["x"][:, :, 3:400:7] = np.finfo(np.float32).min
    c["bias_values"][:, 0] = -np.inf
    c["bias_tokens"][:, 0] = 500
    c["repetition"][:] = 1.0  # the lowest value times r > 1 leaves the type's range
    check(c)


def test_tokens_out_of_range_and_lengths():
    c = make(3, 4, 300, seed=13)
    c["history"][:, ::3] = -1
    c["history"][:, 1::7] = 300
    c["bias_tokens"][:, 1] = 2 ** 31 - 1
    c["block"][:, 2] = -5
    c["history_len"][:] = [-4, 10 ** 6, 17]
    c["prompt_len"][:] = [3, -2, 99]
    check(c)


def test_first_place_of_a_repeated_bias_counts():
    c = make(2, 3, 100, seed=14, bias=40)
    c["bias_tokens"][:] = np.random.default_rng(2).integers(0, 5, (2, 40))
    check(c)


def test_long_history():
    check(make(1, 2, 5000, seed=15, hist=16384))


def test_unaligned_rows():
    """Logits that start between two 16-byte boundaries (a slice of a larger buffer)."""
    from paper_2609_04010_gb300 import binding as b
    V = 1016
    base = torch.randn(2 * 3 * V + 3, device="cuda").to(torch.bfloat16)
    x = base[3:].view(2, 3, V)
    rep = torch.full((2,), 1.5, device="cuda")
    hist = torch.arange(0, 40, dtype=torch.int32, device="cuda").repeat(2, 1).contiguous()
    hl = torch.full((2,), 40, dtype=torch.int32, device="cuda")
    out = torch.empty(2 * 3 * V + 1, dtype=torch.bfloat16, device="cuda")[1:].view(2, 3, V)
    b.adjust_logits(x, history=hist, history_len=hl, repetition=rep, out=out)
    want = ref.adjust(x.float().cpu().numpy(), history=hist.cpu().numpy(), history_len=[40, 40],
                      repetition=[1.5, 1.5])
    assert np.abs(out.float().cpu().numpy() - want).max() <= 2.0 ** -8 * np.abs(want).max()


def test_other_stream_and_graph():
    from paper_2609_04010_gb300 import binding as b
    c = make(4, 4, 4000, seed=16)
    want = run(c)
    x, out = torch.from_numpy(c["x"]).cuda(), torch.zeros(4, 4, 4000, device="cuda")
    t = {k: dev(c[k], c[k].dtype) for k in ARGS}
    t["block_tokens"] = t.pop("block")
    a = b.adjust_args(x, out, **t)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        b.adjust_logits_args(a)
    g.replay()
    torch.cuda.synchronize()
    assert np.array_equal(out.cpu().numpy().astype(np.float64), want)
