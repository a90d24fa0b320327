"""Pages and slots, and the quantising write into the 8-bit KV cache, against the host
references: whole numbers and stored codes equal, no tolerance."""

import numpy as np
import pytest
import torch

import fp8_reference as ref

pytestmark = pytest.mark.gpu


def i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def bf16(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda().to(torch.bfloat16)


def as_np(t):
    return t.float().cpu().numpy().astype(np.float64)


# ----------------------------------------------------------------------------------
# Pages and slots
# ----------------------------------------------------------------------------------
def slot_case(B, P, seed, hi_len=200, hi_new=90, spare=1.0, reserved=0, odd=False):
    r = np.random.default_rng(seed)
    MP = -(-(hi_len + hi_new) // P) + 1
    kv_len, new = r.integers(0, hi_len + 1, B), r.integers(0, hi_new + 1, B)
    held = -(-(kv_len + reserved) // P)
    pool = r.permutation(int(held.sum()) + B * MP)
    table, at = np.full((B, MP), -1, np.int32), 0
    for b in range(B):
        n = min(held[b], MP)
        table[b, :n] = pool[at:at + n]
        at += n
    need = np.maximum(0, -(-(kv_len + new) // P) - held)
    if odd:
        kv_len[B // 2], new[0], new[B - 1] = -3, -5, MP * P + 7
        table[1, 0] = len(pool) + 5  # a page id out of range
    return dict(num_new=new, kv_len=kv_len, table=table, page_size=P, num_pages=len(pool),
                free=pool[at:].astype(np.int32), count=int(need.sum() * spare), reserved=reserved)


def run_slots(c, max_rows, in_place=True):
    from paper_2609_04010_gb300 import binding as b
    table, kv, count = i32(c["table"]), i32(c["kv_len"]), i32([c["count"]])
    new, free = i32(c["num_new"]), i32(c["free"])
    if in_place:
        res = b.map_slots(new, kv, table, c["page_size"], c["num_pages"], free, count, max_rows,
                          reserved=c["reserved"])
    else:
        B = len(c["kv_len"])
        i = dict(dtype=torch.int32, device="cuda")
        res = dict(row_start=torch.empty(B + 1, **i), slots=torch.empty(max_rows, **i),
                   new_len=torch.empty(B, **i), new_count=torch.empty(1, **i))
        a = b.slot_args(new, kv, res["new_len"], table, c["page_size"], c["num_pages"], free, count,
                        res["new_count"], res["row_start"], res["slots"], reserved=c["reserved"])
        ws = b.new_workspace(b.slot_workspace_size(a))
        for _ in range(3):  # nothing read is changed: every call gives the same
            b.map_slots_args(a, ws)
        assert np.array_equal(kv.cpu(), c["kv_len"]) and int(count) == c["count"]
        assert int(ws.sum()) == 0
        kv, count = res["new_len"], res["new_count"]
    return {k: v.cpu().numpy() for k, v in dict(res, new_len=kv, table=table, count=count).items()}


def check_slots(c, max_rows, in_place=True):
    want = ref.map_slots(c["num_new"], c["kv_len"], c["table"], c["page_size"], c["num_pages"],
                         c["free"], c["count"], max_rows, c["reserved"])
    got = run_slots(c, max_rows, in_place)
    for k in set(want) & set(got):
        assert np.array_equal(np.ravel(got[k]), np.ravel(want[k])), k


@pytest.mark.parametrize("B", [1, 2, 33, 512, 513, 1300])
@pytest.mark.parametrize("P", [16, 64, 5])
@pytest.mark.parametrize("spare", [1.0, 0.6])
def test_slots_ragged(B, P, spare):
    c = slot_case(B, P, seed=B * 7 + P, spare=spare)
    check_slots(c, max(1, int(c["num_new"].sum())) + 5)


@pytest.mark.parametrize("rows", [1, 17, 600])
def test_slots_row_limit(rows):
    """Rows past max_rows are not written, their pages are taken all the same."""
    check_slots(slot_case(9, 16, seed=3, hi_new=200), rows)


def test_slots_bad_requests_and_pages():
    c = slot_case(12, 16, seed=5, odd=True)
    check_slots(c, int(np.maximum(c["num_new"], 0).sum()) + 2)
    c = slot_case(12, 16, seed=6, spare=0.0)
    c["count"] = -4
    check_slots(c, 400)


def test_slots_reserved_pages_and_long_prompts():
    c = slot_case(64, 16, seed=8, reserved=16, hi_new=16)
    c["num_new"][:] = 16
    check_slots(c, 64 * 16)
    check_slots(slot_case(3, 64, seed=9, hi_len=0, hi_new=40000), 3 * 40000)


def test_slots_all_zero_lengths():
    c = slot_case(4, 16, seed=1)
    c["num_new"][:] = 0
    check_slots(c, 3)


def test_slots_separate_state_is_repeatable():
    check_slots(slot_case(40, 32, seed=11, spare=0.8), 3000, in_place=False)


# ----------------------------------------------------------------------------------
# Quantising write
# ----------------------------------------------------------------------------------
def filled(pages, H, P, D, seed, garbage=False):
    r = np.random.default_rng(seed)
    codes = r.integers(0, 256, (pages, H, 2, P, D)).astype(np.uint8)
    if not garbage:
        codes[(codes & 0x7f) == 0x7f] = 0x08
    scale = 2.0 ** r.integers(-8, 3, (pages, H, 2))
    return codes, scale.astype(np.float32)


def run_append(k, v, slots, codes, scale, status=None):
    from paper_2609_04010_gb300 import binding as b
    cache = torch.from_numpy(codes.copy()).cuda().view(torch.float8_e4m3fn)
    sc = torch.from_numpy(scale.copy()).cuda()
    b.append_kv_fp8(k, v, i32(slots), cache, sc, status_ws=status)
    torch.cuda.synchronize()
    return cache.view(torch.uint8).cpu().numpy(), sc.cpu().numpy()


def check_append(k, v, slots, codes, scale, status=None):
    P = codes.shape[3]
    got, gs = run_append(k, v, slots, codes, scale, status)
    want, ws = ref.append(as_np(k), as_np(v), np.asarray(slots), codes, scale, P)
    assert np.array_equal(gs.astype(np.float64), ws)
    # a page that starts anew holds nothing of use at its unwritten places
    used = np.ones(codes.shape[0] * P, bool)
    for s in slots:
        if 0 <= s < len(used) and s % P == 0:
            used[s:s + P] = False
    used[[s for s in slots if 0 <= s < len(used)]] = True
    used = used.reshape(-1, P)
    at = np.broadcast_to(used[:, None, None, :, None], codes.shape)
    g, w = got[at], want[at]
    nan = (w & 0x7f) == 0x7f
    assert np.array_equal((g & 0x7f) == 0x7f, nan)
    assert np.array_equal(g[~nan], w[~nan])


def rows_of(R, H, D, seed, spread=4):
    r = np.random.default_rng(seed)
    return bf16(r.standard_normal((R, H, D)) * 2.0 ** r.uniform(-spread, spread, (R, H, 1)))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("P", [16, 32, 64])
@pytest.mark.parametrize("first,n", [(0, 1), (0, 64), (1, 1), (5, 16), (13, 150), (0, 300), (63, 2)])
def test_append_runs(D, P, first, n):
    """A run of n tokens from position `first`, in shuffled pages; started pages go on."""
    H = 3
    pages = -(-(first + n) // P) + 2
    perm = np.random.default_rng(first * 31 + n).permutation(pages)
    pos = first + np.arange(n)
    slots = perm[pos // P] * P + pos % P
    codes, scale = filled(pages, H, P, D, seed=n)
    check_append(rows_of(n, H, D, 1), rows_of(n, H, D, 2), slots, codes, scale)


def test_append_batch_of_blocks_with_skipped_rows():
    """Blocks of several sequences; refused sequences have negative slots."""
    P, H, D, G = 16, 8, 128, 16
    r = np.random.default_rng(0)
    pages, slots, page = 64, [], 0
    for b in range(20):
        ctx = int(r.integers(0, 16))
        pos = ctx + np.arange(G)
        s = (page + pos // P) * P + pos % P
        page += 2
        slots.append(np.full(G, -1) if b % 5 == 3 else s)
    codes, scale = filled(pages, H, P, D, seed=4)
    check_append(rows_of(20 * G, H, D, 5), rows_of(20 * G, H, D, 6), np.concatenate(slots), codes, scale)


def test_append_accepted_path_of_a_tree():
    """Rows of a page with gaps between them: the path's nodes, the others skipped."""
    P, H, D = 16, 2, 64
    slots = np.full(48, -1)
    slots[[0, 3, 9, 20, 41, 47]] = 14 + np.arange(6)  # positions 14 .. 19: pages 0 and 1
    codes, scale = filled(4, H, P, D, seed=7)
    check_append(rows_of(48, H, D, 8), rows_of(48, H, D, 9), slots, codes, scale)


def test_append_interleaved_pages():
    """Rows of two pages taking turns within the window."""
    P, H, D = 64, 1, 128
    slots = np.stack([np.arange(60) + 2, np.arange(60) + 64 + 1], 1).reshape(-1)
    codes, scale = filled(2, H, P, D, seed=10)
    check_append(rows_of(120, H, D, 11), rows_of(120, H, D, 12), slots, codes, scale)


def test_append_edges_of_the_type():
    """Exact halves and the scale's boundary, zeros, infinities, NaN, subnormal and huge values."""
    P, H, D = 16, 1, 64
    x = np.zeros((16, 1, 64), np.float32)
    x[0, 0, :8] = [448, 447, 432, 416, 1.0625, 1.1875, 2 ** -9, 2 ** -10]
    x[1, 0, :4] = [np.inf, -np.inf, np.nan, 3.5]
    x[2, 0, :3] = [1e-40, -1e-30, 2 ** -33]
    x[3, 0, :2] = [0.0, -0.0]
    for row in range(4):
        k = bf16(x[row:row + 1])
        for place in (0, 5):
            codes, scale = filled(1, H, P, D, seed=row, garbage=False)
            check_append(k, k, [place], codes, scale)
    big = np.full((1, 1, 64), 3e38, np.float32)
    big[0, 0, 1] = 1.0
    codes, scale = filled(1, H, P, D, seed=2)
    check_append(bf16(big), bf16(-big), [0], codes, scale)
    allnan = np.full((1, 1, 64), np.nan, np.float32)
    check_append(bf16(allnan), bf16(allnan), [0], codes, scale)


@pytest.mark.parametrize("old", [0.0, -1.0, np.nan, np.inf, 0.75])
def test_append_foreign_scales(old):
    """Scales that no call wrote are read clamped; non-powers of two keep working."""
    P, H, D = 16, 1, 64
    codes, scale = filled(1, H, P, D, seed=3)
    scale[:] = old
    k = rows_of(2, H, D, 13, spread=0)
    got, gs = run_append(k, k, [4, 5], codes, scale)
    eff = np.float32(np.fmin(np.fmax(np.float32(old), 2.0 ** -32), 2.0 ** 32))
    want, ws = ref.append(as_np(k), as_np(k), np.array([4, 5]), codes, np.full_like(scale, eff), P)
    assert np.array_equal(gs.astype(np.float64), ws)
    same = got == want
    if old == 0.75:  # old / new is not a power of two: one fp32 rounding before the e4m3 one
        near = np.abs(ref.decode(got) - ref.decode(want)) <= np.abs(ref.decode(want)) / 8 + 2.0 ** -9
        assert same.mean() > 0.999 and near.all()
    else:
        assert same.all()


def test_append_strided_rows_and_streams():
    """Column ranges of a wider projection, on a stream of their own."""
    P, H, D, n = 32, 4, 128, 50
    wide = rows_of(n, 3 * H, D, 14)
    codes, scale = filled(4, H, P, D, seed=5)
    slots = np.arange(n) + 3
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        check_append(wide[:, H:2 * H], wide[:, 2 * H:], slots, codes, scale)


def test_append_repeated_call_changes_nothing():
    P, H, D = 16, 2, 128
    codes, scale = filled(3, H, P, D, seed=6)
    k, v, slots = rows_of(20, H, D, 15), rows_of(20, H, D, 16), np.arange(20) + 9
    c1, s1 = run_append(k, v, slots, codes, scale)
    c2, s2 = run_append(k, v, slots, c1, s1)
    assert np.array_equal(c1, c2) and np.array_equal(s1, s2)


def test_append_bad_slots_are_skipped_and_reported():
    from paper_2609_04010_gb300 import binding as b
    P, H, D = 16, 2, 64
    codes, scale = filled(2, H, P, D, seed=8)
    ws = b.new_workspace(256)
    check_append(rows_of(4, H, D, 1), rows_of(4, H, D, 2), [3, 32, 4, 2 ** 31 - 1], codes, scale, ws)
    assert b.read_device_status(ws) == (5, b.FLAG_BAD_PAGE)
    check_append(rows_of(4, H, D, 1), rows_of(4, H, D, 2), [3, -1, 4, -7], codes, scale, ws)
    assert b.read_device_status(ws) == (0, 0)


def test_append_no_rows():
    codes, scale = filled(1, 1, 16, 64, seed=1)
    check_append(rows_of(0, 1, 64, 1), rows_of(0, 1, 64, 2), np.zeros(0, np.int32), codes, scale)


def test_append_far_page():
    """A page whose bytes start past 2^32."""
    from paper_2609_04010_gb300 import binding as b
    P, H, D = 64, 8, 128
    pages = 2 ** 32 // (H * 2 * P * D) + 40
    cache = torch.empty(pages, H, 2, P, D, dtype=torch.uint8, device="cuda")
    scale = torch.ones(pages, H, 2, device="cuda")
    cache[-1] = 0x38
    k, v = rows_of(5, H, D, 3), rows_of(5, H, D, 4)
    slots = (pages - 1) * P + 7 + np.arange(5)
    b.append_kv_fp8(k, v, i32(slots), cache.view(torch.float8_e4m3fn), scale)
    want, ws = ref.append(as_np(k), as_np(v), slots - (pages - 1) * P, np.full((1, H, 2, P, D), 0x38, np.uint8),
                          np.ones((1, H, 2)), P)
    assert np.array_equal(cache[-1].cpu().numpy(), want[0])
    assert np.array_equal(scale[-1].cpu().numpy(), ws[0])


def test_slots_feed_the_append():
    """map_slots, append and commit over steps: the cache holds every kept token."""
    from paper_2609_04010_gb300 import binding as b
    B, G, P, H, D, MP = 3, 8, 16, 2, 64, 12
    r = np.random.default_rng(20)
    pages = 40
    cache, scale = b.new_kv_cache_fp8(pages, H, P, D)
    table, kv = i32(np.full((B, MP), -1)), i32(np.zeros(B))
    free, count = i32(r.permutation(pages)), i32([pages])
    kept = [[] for _ in range(B)]
    new = i32([37, 5, 16])
    for step in range(6):
        n = new.cpu().numpy()
        R = int(n.sum())
        m = b.map_slots(new, kv, table, P, pages, free, count, R, reserved=0 if step < 2 else G)
        assert int(m["flags"].sum()) == 0
        k = rows_of(R, H, D, 100 + step, spread=1)
        b.append_kv_fp8(k, k, m["slots"], cache, scale)
        rows = as_np(k)
        for s in range(B):
            part = rows[int(m["row_start"][s]):int(m["row_start"][s + 1])]
            kept[s].extend(part)
        if step > 0:
            acc = i32(r.integers(0, G, B))
            b.commit_kv(kv, acc, table, P, G, free, count, reserve=True)
            for s in range(B):
                kept[s] = kept[s][:len(kept[s]) - G + int(acc[s]) + 1]
        new = i32([G] * B)
    codes, sc, tb = cache.view(torch.uint8).cpu().numpy(), scale.cpu().numpy(), table.cpu().numpy()
    for s in range(B):
        assert int(kv[s]) == len(kept[s])
        for pos, x in enumerate(kept[s]):
            page = tb[s, pos // P]
            for kind in (0, 1):
                got = ref.decode(codes[page, :, kind, pos % P]) * sc[page, :, kind][:, None]
                # within half a step of e4m3 at the scale's range, twice (the page may have grown)
                tol = np.abs(x) * 2.0 ** -4 + sc[page, :, kind][:, None] * 2.0 ** -9
                assert (np.abs(got - x) <= 2 * tol).all()
