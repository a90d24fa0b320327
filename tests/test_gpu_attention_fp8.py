"""Attention over the 8-bit KV cache against the 64-bit host reference, on every path.

Tolerances. With s the scores, p the weights and o the outputs:
  * a query enters a tensor-core score as the sum of two e4m3 terms, exact to 2^-18 of the
    largest |q| of its KV group, and a score is an fp32 sum of at most 128 products; so
    |ds| <= scale * kmax * (2^-18 + 128 * 2^-24) * max|q|, kmax = max_t sum_d |k_td|;
  * a weight enters as two e4m3 terms, exact to 2^-8 of itself, or to 2^-13 of the row's
    largest weighted value 2^m where it is small; ds moves it by another (e^|2 ds| - 1);
    so |do| <= (2^-8 + 2 |ds|) * sum_t p_t |v_t| + 2^-12 * max_t |v_t| + 2^-9 * |o| (bf16)
    (the floor's terms have independent signs: 2^-13 * max|v| for one key bounds them);
  * lse = m + log(sum): |ds| + 2^-20 * (1 + |lse|).
"""

import numpy as np
import pytest
import torch

import fp8_reference as ref

pytestmark = pytest.mark.gpu

CUDA_CORES, TENSOR_CORES = 1, 2
PATHS = [CUDA_CORES, TENSOR_CORES]


def i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


class Case:
    """A paged 8-bit cache whose unused pages and places hold NaN bytes."""

    def __init__(self, B, G, Hq, H, D, P, ctx, seed=0, tree=None, q_scale=1.0, scales=None):
        r = np.random.default_rng(seed)
        self.G, self.P = G, P
        self.kv_len = np.resize(np.asarray(ctx), B).astype(np.int64) + G
        need = -(-self.kv_len // P)
        pages = int(need.sum()) + 3
        perm = r.permutation(pages)
        self.table, at = np.full((B, int(need.max()) + 2), -1, np.int64), 0
        self.codes = np.full((pages, H, 2, P, D), 0xFF, np.uint8)
        self.scale = (2.0 ** r.integers(-9, -4, (pages, H, 2)) if scales is None
                      else scales(r, (pages, H, 2))).astype(np.float32)
        for b in range(B):
            for i in range(int(need[b])):
                page = perm[at]
                at += 1
                self.table[b, i] = page
                n = min(P, int(self.kv_len[b]) - i * P)
                x = r.standard_normal((H, 2, n, D)) * 100
                self.codes[page, :, :, :n] = ref.encode(x)
        q = torch.from_numpy((r.standard_normal((B, G, Hq, D)) * q_scale).astype(np.float32))
        self.q = q.to(torch.bfloat16)
        self.tree = tree(r, B, G) if tree else None

    def device(self):
        t = [self.q.cuda(), torch.from_numpy(self.codes).cuda().view(torch.float8_e4m3fn),
             torch.from_numpy(self.scale).cuda(), i32(self.table), i32(self.kv_len)]
        tree = None if self.tree is None else torch.from_numpy(self.tree.view(np.int64)).cuda()
        return t, tree

    def run(self, path, ws=None, want_flags=0, **kw):
        from paper_2609_04010_gb300 import binding as b
        t, tree = self.device()
        out, lse = torch.full_like(t[0], 7.0), torch.full(t[0].shape[:3], 7.0, device="cuda")
        a = b.attn_fp8_args(*t, out, lse, path=path, tree_mask=tree, **kw)
        if ws is None:
            ws = b.new_workspace(b.attn_fp8_workspace_size(a))
        b.verify_attention_fp8_args(a, ws)
        torch.cuda.synchronize()
        first = out.clone(), lse.clone()
        b.verify_attention_fp8_args(a, ws)  # the workspace's counters are back at zero
        torch.cuda.synchronize()
        assert torch.equal(first[1].nan_to_num(5), lse.nan_to_num(5))
        assert torch.equal(first[0].nan_to_num(5), out.nan_to_num(5))
        assert b.read_device_status(ws)[1] == want_flags
        return out.float().cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64)

    def check(self, path, softmax_scale=0.0, rows=None):
        o, l = self.run(path, softmax_scale=softmax_scale)
        q = self.q.double().numpy()
        ro, rl, mass, kmax = ref.attention(q, self.codes, self.scale, self.table, self.kv_len,
                                           self.G, self.P, softmax_scale, self.tree)
        sc = softmax_scale or q.shape[-1] ** -0.5
        B, G, Hq, _ = q.shape
        H = self.codes.shape[1]
        qmax = np.repeat(np.abs(q).reshape(B, G, H, -1).max((1, 3)), Hq // H, 1)[:, None]
        ds = (sc * kmax * (2.0 ** -18 + 128 * 2.0 ** -24) * qmax)[..., None]
        used = self.codes[(self.codes & 0x7f) != 0x7f]
        vmax = np.abs(ref.decode(used)).max() * np.clip(self.scale[:, :, 1], 2.0 ** -32, 2.0 ** 32).max()
        tol = (2.0 ** -8 + 2 * ds) * mass + 2.0 ** -12 * vmax + 2.0 ** -9 * np.abs(ro) + 1e-30
        fin = np.isfinite(rl)
        assert np.array_equal(fin, np.isfinite(l)) and np.all(l[~fin] == -np.inf)
        assert np.all(o[~fin] == 0)
        err = np.abs(o - ro) / tol
        assert np.isfinite(o).all() and err.max() <= 1, (err.max(), np.unravel_index(err.argmax(), err.shape))
        lerr = np.abs(l[fin] - rl[fin]) / (ds[..., 0][fin] + 2.0 ** -20 * (1 + np.abs(rl[fin])))
        assert lerr.size == 0 or lerr.max() <= 1, lerr.max()
        # and as a whole: rounding to bf16 and the split weights average out
        assert np.linalg.norm(o - ro) <= 2.0 ** -8 * np.linalg.norm(ro) + 1e-30


def random_tree(r, B, G):
    bits = np.zeros((B, G), np.uint64)
    bits[:, 0] = 1
    for c in range(1, G):
        parent = r.integers(0, c, B)
        bits[:, c] = bits[np.arange(B), parent] | (np.uint64(1) << np.uint64(c))
    return bits


def empty_tree(r, B, G):
    """Some nodes see nothing of the block, not even themselves."""
    bits = random_tree(r, B, G)
    bits[:, ::2] = 0
    return bits


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("P", [16, 32, 64])
@pytest.mark.parametrize("ctx", [0, 1, 15, 16, 63, 64, 65, 127, 128, 129, 500])
def test_contexts_and_pages(path, D, P, ctx):
    Case(1, 4, 4, 2, D, P, ctx, seed=ctx + P).check(path)


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("G,Hq,H", [(1, 8, 8), (1, 32, 8), (1, 7, 1), (2, 12, 3), (5, 6, 2), (7, 9, 3),
                                    (16, 32, 8), (17, 8, 2), (32, 16, 2), (33, 4, 2), (64, 2, 2),
                                    (64, 8, 2), (32, 16, 1), (3, 80, 2), (64, 16, 1), (8, 5, 5)])
@pytest.mark.parametrize("D", [64, 128])
def test_head_layouts(path, G, Hq, H, D):
    Case(2, G, Hq, H, D, 16, [37, 200], seed=G * Hq).check(path)


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("G,Hq,H", [(1, 4, 1), (8, 8, 2), (31, 8, 2), (64, 2, 2), (64, 12, 3)])
@pytest.mark.parametrize("ctx", [0, 100, 121])
def test_trees(path, G, Hq, H, ctx):
    Case(2, G, Hq, H, 128, 16, ctx, seed=G, tree=random_tree).check(path)
    Case(2, G, Hq, H, 64, 32, ctx, seed=G, tree=empty_tree).check(path)


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("B", [1, 3, 70, 200])
def test_ragged_batches(path, B):
    """Lengths from one key to several tiles in one call; more units than blocks."""
    ctx = np.random.default_rng(B).integers(0, 700, B)
    Case(B, 3, 8, 2, 64, 16, ctx, seed=B).check(path)


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("D,P", [(128, 64), (64, 16)])
def test_long_context(path, D, P):
    """One sequence split over the whole GPU."""
    Case(1, 2, 4, 1, D, P, 40000, seed=5).check(path)
    Case(2, 1, 8, 4, D, P, [9000, 1], seed=6).check(path)


@pytest.mark.parametrize("path", PATHS)
def test_scales(path):
    """Scales that differ by page, that are no powers of two, of empty pages, far apart."""
    Case(2, 4, 8, 2, 128, 16, 300, seed=1, scales=lambda r, s: r.uniform(1e-3, 1e-2, s)).check(path)
    Case(2, 4, 8, 2, 64, 32, 300, seed=2, scales=lambda r, s: 2.0 ** r.integers(-14, -4, s)).check(path)
    c = Case(2, 4, 8, 2, 128, 16, 300, seed=3)
    for page in c.table[:, 3]:
        c.codes[page] = 0
        c.scale[page] = 2.0 ** -32
    c.check(path)
    c.scale[c.table[:, 3]] = 0.0  # another quantiser's empty page
    c.check(path)


@pytest.mark.parametrize("path", PATHS)
def test_sharp_and_flat_weights(path):
    """One key takes nearly all the weight; all keys weigh the same; given softmax scales."""
    Case(2, 4, 8, 2, 128, 16, 300, seed=1, q_scale=30.0).check(path)
    Case(2, 4, 8, 2, 128, 16, 300, seed=2, q_scale=1e-6).check(path)
    Case(2, 4, 8, 2, 128, 16, 300, seed=3, q_scale=0.0).check(path)
    Case(2, 4, 8, 2, 64, 16, 300, seed=4).check(path, softmax_scale=0.01)


@pytest.mark.parametrize("path", PATHS)
def test_growing_maximum(path):
    """Keys that score higher the later they come: the running maximum rises in every tile."""
    c = Case(1, 2, 4, 1, 128, 16, 1500, seed=9)
    c.q[:] = 1.0
    for i, page in enumerate(c.table[0, :94]):
        n = min(16, int(c.kv_len[0]) - i * 16)
        c.codes[page, 0, 0, :n] = ref.encode(np.full((n, 128), min(448.0, 1.0 + 4 * i)))
        c.scale[page, 0, 0] = 2.0 ** -6
    c.check(path)


@pytest.mark.parametrize("path", PATHS)
def test_bad_sequences(path):
    """A page id out of range and lengths out of range: zeros, -inf, a flag; others unharmed."""
    from paper_2609_04010_gb300 import binding as b
    for what in ("page", "short", "long"):
        c = Case(3, 4, 8, 2, 128, 16, 400, seed=2)
        good = c.run(path)
        if what == "page":
            c.table[1, 20] = 10 ** 6
            flag = b.FLAG_BAD_PAGE
        else:
            c.kv_len[1] = 3 if what == "short" else c.table.shape[1] * 16 + 1
            flag = b.FLAG_BAD_KV_LEN
        o, l = c.run(path, want_flags=flag)
        assert np.all(o[1] == 0) and np.all(l[1] == -np.inf)
        for s in (0, 2):
            assert np.abs(o[s] - good[0][s]).max() <= 2.0 ** -7 * np.abs(good[0][s]).max()
            assert np.abs(l[s] - good[1][s]).max() < 1e-4


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("D", [64, 128])
def test_hidden_nan_does_not_leak(path, D):
    """NaN keys and values of block tokens reach the rows that see them and no others."""
    for kind in (0, 1):
        c = Case(1, 8, 8, 2, D, 16, 121, seed=4)
        want = c.run(path)
        pos = 121 + 5
        page, place = c.table[0, pos // 16], pos % 16
        c.codes[page, 1, kind, place, 3] = 0x7f
        o, l = c.run(path)
        assert np.array_equal(o[0, :5], want[0][0, :5]) and np.array_equal(l[0, :5], want[1][0, :5])
        assert np.array_equal(o[:, :, :4], want[0][:, :, :4])  # the other KV head
        if kind == 0:
            assert np.isnan(o[0, 5:, 4:]).all() and np.isnan(l[0, 5:, 4:]).all()
        else:
            assert np.isnan(o[0, 5:, 4:, 3]).all() and np.array_equal(l, want[1])
            rest = np.arange(D) != 3
            assert np.array_equal(o[0, 5:, 4:][..., rest], want[0][0, 5:, 4:][..., rest])


@pytest.mark.parametrize("path", PATHS)
def test_nan_query_stays_in_its_row(path):
    c = Case(1, 4, 8, 2, 128, 16, 300, seed=4)
    want = c.run(path)
    for bad in (float("nan"), float("inf")):
        c.q[0, 2, 3, 5] = bad
        o, l = c.run(path)
        assert np.isnan(o[0, 2, 3]).all() and np.isnan(l[0, 2, 3])
        o[0, 2, 3], l[0, 2, 3] = want[0][0, 2, 3], want[1][0, 2, 3]
        assert np.array_equal(o, want[0]) and np.array_equal(l, want[1])


@pytest.mark.parametrize("path", PATHS)
def test_far_pages(path):
    """Pages whose bytes start past 2^32."""
    from paper_2609_04010_gb300 import binding as b
    c = Case(1, 2, 8, 8, 128, 64, 300, seed=7)
    want = c.run(path)
    n = c.codes.shape[0]
    pages = 2 ** 32 // c.codes[0].size + 40
    cache = torch.empty(pages, *c.codes.shape[1:], dtype=torch.uint8, device="cuda")
    cache[pages - n:] = torch.from_numpy(c.codes).cuda()
    scale = torch.ones(pages, 8, 2, device="cuda")
    scale[pages - n:] = torch.from_numpy(c.scale).cuda()
    table = np.where(c.table >= 0, c.table + pages - n, -1)
    o, l = b.verify_attention_fp8(c.q.cuda(), cache.view(torch.float8_e4m3fn), scale, i32(table),
                                  i32(c.kv_len), path=path)
    assert np.array_equal(o.float().cpu().numpy().astype(np.float64), want[0])
    assert np.array_equal(l.cpu().numpy().astype(np.float64), want[1])


@pytest.mark.parametrize("path", PATHS)
def test_other_stream_and_graph(path):
    from paper_2609_04010_gb300 import binding as b
    c = Case(4, 4, 8, 2, 128, 16, [300, 5, 1000, 64], seed=8)
    want = c.run(path)
    t, _ = c.device()
    out, lse = torch.zeros_like(t[0]), torch.zeros(t[0].shape[:3], device="cuda")
    a = b.attn_fp8_args(*t, out, lse, path=path)
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


def test_no_lse_and_auto():
    from paper_2609_04010_gb300 import binding as b
    c = Case(2, 4, 8, 2, 128, 16, 100, seed=3)
    t, _ = c.device()
    o, l = b.verify_attention_fp8(*t, want_lse=False)
    o2, _ = b.verify_attention_fp8(*t)
    assert l is None and torch.equal(o, o2)
    c.check(0)


@pytest.mark.parametrize("G,Hq", [(1, 4), (9, 8)])
def test_more_sequences_than_one_launch_takes(G, Hq):
    """The tensor-core kernels take 2,048 sequences at a time; the parts meet nowhere."""
    Case(2051, G, Hq, 2, 64, 16, [40, 3, 0, 129], seed=9, tree=random_tree).check(TENSOR_CORES)


def test_wait_timeout_is_reported_and_survived():
    """The kernel with an idle copy producer: its bounded waits run out, it reports, and the
    same workspace serves the next call."""
    from paper_2609_04010_gb300 import binding as b
    c = Case(3, 4, 8, 2, 128, 16, [300, 5, 1000], seed=8)
    want = c.run(TENSOR_CORES)
    t, _ = c.device()
    out, lse = torch.zeros_like(t[0]), torch.zeros(t[0].shape[:3], device="cuda")
    a = b.attn_fp8_args(*t, out, lse, path=TENSOR_CORES)
    ws = b.new_workspace(b.attn_fp8_workspace_size(a))
    b.test_attention_fp8_wait_timeout_args(a, ws)
    assert b.read_device_status(ws) == (6, b.FLAG_TIMEOUT)
    assert int(ws[256:256 + 64].sum()) == 0
    b.verify_attention_fp8_args(a, ws)
    torch.cuda.synchronize()
    assert b.read_device_status(ws) == (0, 0)
    assert np.array_equal(out.float().cpu().numpy().astype(np.float64), want[0])
    assert np.array_equal(lse.cpu().numpy().astype(np.float64), want[1])


def test_wait_timeout_with_many_rows_is_reported_and_survived():
    """The same for the kernel that takes 33 and more query rows."""
    from paper_2609_04010_gb300 import binding as b
    c = Case(2, 12, 8, 2, 64, 32, [300, 5], seed=8)
    want = c.run(TENSOR_CORES)
    t, _ = c.device()
    out, lse = torch.zeros_like(t[0]), torch.zeros(t[0].shape[:3], device="cuda")
    a = b.attn_fp8_args(*t, out, lse, path=TENSOR_CORES)
    ws = b.new_workspace(b.attn_fp8_workspace_size(a))
    b.test_attention_fp8_wait_timeout_args(a, ws)
    assert b.read_device_status(ws) == (6, b.FLAG_TIMEOUT)
    b.verify_attention_fp8_args(a, ws)
    torch.cuda.synchronize()
    assert b.read_device_status(ws) == (0, 0)
    assert np.array_equal(out.float().cpu().numpy().astype(np.float64), want[0])
    assert np.array_equal(lse.cpu().numpy().astype(np.float64), want[1])
