"""The attention over the 8-bit KV cache with 33 and more query rows a KV head (a kernel of its
own on the tensor cores), where it can go wrong: against the 64-bit host reference with the bounds
of test_gpu_attention_fp8.py, and against the call's own result without the disturbance."""

import numpy as np
import pytest
import torch

import fp8_reference as ref
from test_gpu_attention_fp8 import Case, TENSOR_CORES, i32, random_tree

pytestmark = pytest.mark.gpu

# (gamma, Hq, Hkv): 48 rows of each of two heads, 256 and 264 rows of one head
LAYOUTS = [(12, 8, 2), (16, 16, 1), (33, 8, 1)]


@pytest.mark.parametrize("G,Hq,H", LAYOUTS)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B", [1, 400])
def test_nan_values_reach_the_rows_that_see_them(G, Hq, H, D, B):
    """A NaN among a block token's values, in every third sequence; with 400 sequences a block has
    several of them after one another."""
    c = Case(B, G, Hq, H, D, 16, 121, seed=4)
    want = c.run(TENSOR_CORES)
    j = 5
    for s in range(0, B, 3):
        c.codes[c.table[s, (121 + j) // 16], H - 1, 1, (121 + j) % 16, 3 + s % 7] = 0x7f
    o, l = c.run(TENSOR_CORES)
    assert np.array_equal(l, want[1])
    per = Hq // H
    for s in range(B):
        seen = want[0][s].copy()
        if s % 3 == 0:
            seen[j:, Hq - per:, 3 + s % 7] = np.nan
        assert np.array_equal(o[s], seen, equal_nan=True), s


@pytest.mark.parametrize("G,Hq,H", LAYOUTS)
@pytest.mark.parametrize("D,P,ctx", [(128, 16, 0), (128, 64, 95), (64, 32, 127), (64, 16, 500), (128, 32, 1023)])
def test_contexts_and_pages(G, Hq, H, D, P, ctx):
    Case(1, G, Hq, H, D, P, ctx, seed=ctx + P).check(TENSOR_CORES)


def check_some(c, at, times=1):
    """As Case.check for the sequences `at` of a batch that runs as a whole, `times` times over."""
    B, G, Hq, D = c.q.shape
    q, table, kv_len = c.q, c.table, c.kv_len
    c.q, c.table, c.kv_len = q.repeat(times, 1, 1, 1), np.tile(table, (times, 1)), np.tile(kv_len, times)
    o, l = c.run(TENSOR_CORES)
    c.q, c.table, c.kv_len = q, table, kv_len
    x, tree = q[at].double().numpy(), None if c.tree is None else c.tree[at]
    ro, rl, mass, kmax = ref.attention(x, c.codes, c.scale, table[at], kv_len[at], G, c.P, 0.0, tree)
    ds = (D ** -0.5 * kmax * (2.0 ** -18 + 128 * 2.0 ** -24) * np.abs(x).max((1, 2, 3))[:, None, None])[..., None]
    used = np.abs(ref.decode(c.codes[(c.codes & 0x7f) != 0x7f])).max() * c.scale[:, :, 1].max()
    tol = (2.0 ** -8 + 2 * ds) * mass + 2.0 ** -12 * used + 2.0 ** -9 * np.abs(ro)
    for o, l in zip(o.reshape(times, B, *o.shape[1:]), l.reshape(times, B, *l.shape[1:])):
        assert (np.abs(o[at] - ro) / tol).max() <= 1
        assert (np.abs(l[at] - rl) / (ds[..., 0] + 2.0 ** -20 * (1 + np.abs(rl)))).max() <= 1
        assert np.linalg.norm(o[at] - ro) <= 2.0 ** -8 * np.linalg.norm(ro)


@pytest.mark.parametrize("G,Hq,H", LAYOUTS)
def test_ragged_batch_of_several_tiles_a_block(G, Hq, H):
    """More tiles than blocks: a block goes through several tiles of a unit and several units."""
    ctx = np.random.default_rng(1).integers(0, 1500, 90)
    check_some(Case(90, G, Hq, H, 64, 16, ctx, seed=2, tree=random_tree), [0, 17, 44, 89])


def growing(B, G, Hq, H, D, ctx, step, seed):
    """Keys that score higher the later they come. All rows' queries are ones; the keys of a page
    are one number, `step` more than the page before."""
    c = Case(B, G, Hq, H, D, 16, ctx, seed=seed)
    c.q[:] = 1.0
    for s in range(B):
        for i in range(-(-int(c.kv_len[s]) // 16)):
            page, n = c.table[s, i], min(16, int(c.kv_len[s]) - i * 16)
            c.codes[page, :, 0, :n] = ref.encode(np.full((H, n, D), min(448.0, 1.0 + step * i)))
            c.scale[page, :, 0] = 2.0 ** -6
    return c


@pytest.mark.parametrize("G,Hq,H", LAYOUTS)
@pytest.mark.parametrize("B,ctx", [(1, 1500), (60, 1500)])
@pytest.mark.parametrize("step", [4, 0.5, -0.5])
def test_growing_maximum(G, Hq, H, B, ctx, step):
    """The running maximum rises in every tile (or never after the first), by one tile a block and
    by several, where outputs held in tensor memory are scaled again."""
    c = growing(min(B, 3), G, Hq, H, 128, ctx, abs(step), seed=9)
    if step < 0:  # falling scores: negated keys
        c.codes[:, :, 0] ^= 0x80
        c.codes[(c.codes & 0x7f) == 0x7f] = 0xff
    check_some(c, list(range(len(c.kv_len))), max(1, B // 3))


@pytest.mark.parametrize("G,Hq,H", LAYOUTS)
def test_scales(G, Hq, H):
    """Scales that differ by page, that are no powers of two, of empty pages, far apart."""
    Case(2, G, Hq, H, 128, 16, 300, seed=1, scales=lambda r, s: r.uniform(1e-3, 1e-2, s)).check(TENSOR_CORES)
    Case(2, G, Hq, H, 64, 32, 300, seed=2, scales=lambda r, s: 2.0 ** r.integers(-14, -4, s)).check(TENSOR_CORES)
    c = Case(2, G, Hq, H, 128, 16, 300, seed=3)
    for page in c.table[:, 3]:
        c.codes[page] = 0
        c.scale[page] = 2.0 ** -32
    c.check(TENSOR_CORES)
    c.scale[c.table[:, 3]] = 0.0  # another quantiser's empty page
    c.check(TENSOR_CORES)


@pytest.mark.parametrize("G,Hq,H", LAYOUTS)
def test_sharp_and_flat_weights(G, Hq, H):
    Case(2, G, Hq, H, 128, 16, 300, seed=1, q_scale=30.0).check(TENSOR_CORES)
    Case(2, G, Hq, H, 128, 16, 300, seed=2, q_scale=1e-6).check(TENSOR_CORES)
    Case(2, G, Hq, H, 128, 16, 300, seed=3, q_scale=0.0).check(TENSOR_CORES)
    Case(2, G, Hq, H, 64, 16, 300, seed=4).check(TENSOR_CORES, softmax_scale=0.01)


@pytest.mark.parametrize("G,Hq,H", LAYOUTS)
@pytest.mark.parametrize("what", ["page", "short", "long"])
@pytest.mark.parametrize("B", [3, 120])
def test_bad_sequences(G, Hq, H, what, B):
    """A page id out of range and lengths out of range: zeros, -inf, a flag; others unharmed."""
    from paper_2609_04010_gb300 import binding as b
    c = Case(B, G, Hq, H, 128, 16, 400, seed=2)
    good = c.run(TENSOR_CORES)
    if what == "page":
        c.table[1, 20] = 10 ** 6
        flag = b.FLAG_BAD_PAGE
    else:
        c.kv_len[1] = 3 if what == "short" else c.table.shape[1] * 16 + 1
        flag = b.FLAG_BAD_KV_LEN
    o, l = c.run(TENSOR_CORES, want_flags=flag)
    assert np.all(o[1] == 0) and np.all(l[1] == -np.inf)
    rest = np.arange(B) != 1  # a unit's parts may be cut elsewhere
    assert np.abs(o[rest] - good[0][rest]).max() <= 2.0 ** -7 * np.abs(good[0][rest]).max()
    assert np.abs(l[rest] - good[1][rest]).max() < 1e-4


@pytest.mark.parametrize("G,Hq,H", LAYOUTS)
@pytest.mark.parametrize("D", [64, 128])
def test_nan_keys_reach_the_rows_that_see_them(G, Hq, H, D):
    c = Case(1, G, Hq, H, D, 16, 121, seed=4)
    want = c.run(TENSOR_CORES)
    c.codes[c.table[0, 126 // 16], H - 1, 0, 126 % 16, 3] = 0x7f  # block key 5
    o, l = c.run(TENSOR_CORES)
    at = Hq - Hq // H
    assert np.isnan(o[0, 5:, at:]).all() and np.isnan(l[0, 5:, at:]).all()
    for x, y in ((o, want[0]), (l, want[1])):
        x[0, 5:, at:] = y[0, 5:, at:]
        assert np.array_equal(x, y)


@pytest.mark.parametrize("G,Hq,H", LAYOUTS)
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_nan_query_stays_in_its_row(G, Hq, H, bad):
    c = Case(1, G, Hq, H, 128, 16, 300, seed=4)
    want = c.run(TENSOR_CORES)
    c.q[0, 2, 3, 5] = bad
    o, l = c.run(TENSOR_CORES)
    assert np.isnan(o[0, 2, 3]).all() and np.isnan(l[0, 2, 3])
    o[0, 2, 3], l[0, 2, 3] = want[0][0, 2, 3], want[1][0, 2, 3]
    assert np.array_equal(o, want[0]) and np.array_equal(l, want[1])


@pytest.mark.parametrize("D,P", [(128, 64), (64, 16)])
def test_long_context(D, P):
    """One sequence split over the whole GPU, a second of one key beside it."""
    Case(1, 12, 8, 2, D, P, 40000, seed=5).check(TENSOR_CORES)
    Case(2, 16, 16, 1, D, P, [9000, 1], seed=6).check(TENSOR_CORES)


def test_far_pages():
    """Pages whose bytes start past 2^32."""
    from paper_2609_04010_gb300 import binding as b
    c = Case(1, 16, 32, 8, 128, 64, 300, seed=7)
    want = c.run(TENSOR_CORES)
    n = c.codes.shape[0]
    pages = 2 ** 32 // c.codes[0].size + 40
    cache = torch.empty(pages, *c.codes.shape[1:], dtype=torch.uint8, device="cuda")
    cache[pages - n:] = torch.from_numpy(c.codes).cuda()
    scale = torch.ones(pages, 8, 2, device="cuda")
    scale[pages - n:] = torch.from_numpy(c.scale).cuda()
    table = np.where(c.table >= 0, c.table + pages - n, -1)
    o, l = b.verify_attention_fp8(c.q.cuda(), cache.view(torch.float8_e4m3fn), scale, i32(table), i32(c.kv_len),
                                  path=TENSOR_CORES)
    assert np.array_equal(o.float().cpu().numpy().astype(np.float64), want[0])
    assert np.array_equal(l.cpu().numpy().astype(np.float64), want[1])


def test_other_stream_and_graph():
    from paper_2609_04010_gb300 import binding as b
    c = Case(4, 12, 8, 2, 128, 16, [300, 5, 1000, 64], seed=8)
    want = c.run(TENSOR_CORES)
    t, _ = c.device()
    out, lse = torch.zeros_like(t[0]), torch.zeros(t[0].shape[:3], device="cuda")
    a = b.attn_fp8_args(*t, out, lse, path=TENSOR_CORES)
    ws = b.new_workspace(b.attn_fp8_workspace_size(a))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b.verify_attention_fp8_args(a, ws)  # first use outside the capture
    torch.cuda.synchronize()
    out.zero_()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        b.verify_attention_fp8_args(a, ws)
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    assert np.array_equal(out.float().cpu().numpy().astype(np.float64), want[0])
    assert np.array_equal(lse.cpu().numpy().astype(np.float64), want[1])
