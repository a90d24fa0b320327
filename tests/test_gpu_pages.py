"""Forked and ended sequences, and page copies, against plain loops: whole numbers, equal."""

import numpy as np
import pytest
import torch

import serving_reference as ref

pytestmark = pytest.mark.gpu


def i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def fork_case(B, P, seed, hi=300, reserved=0, spare=1.0, kind="mixed", group=4):
    """A consistent state: sequences of a group hold a common prefix together."""
    r = np.random.default_rng(seed)
    MP = -(-(hi + reserved) // P) + 2
    lens = r.integers(0, hi + 1, B)
    held = -(-(lens + reserved) // P)
    N = int(held.sum()) + B * (2 + reserved // P)
    pool = r.permutation(N)
    table, shares, at = np.full((B, MP), -1), np.zeros(N, np.int64), 0
    for b in range(B):
        lead = b // group * group
        skip = 0 if b == lead else min(lens[lead], lens[b]) // 2 // P
        table[b, :skip] = table[lead, :skip]
        shares[table[b, :skip]] += 1
        table[b, skip:held[b]] = pool[at:at + held[b] - skip]
        at += held[b] - skip
    free = np.concatenate([pool[at:], np.full(at + 3, -7)])
    parent = np.arange(B)
    if kind == "mixed":
        u = r.random(B)
        parent = np.where(u < 0.25, -1, np.where(u < 0.6, r.integers(0, B, B), parent))
    elif kind == "beams":
        parent = np.arange(B) // group * group + r.integers(0, group, B)
        parent = np.minimum(parent, B - 1)
    elif kind == "end":
        parent = np.full(B, -1)
    elif kind == "one":
        parent = np.zeros(B, np.int64)
    return dict(parent=parent, kv_len=lens, table=table, shares=shares, free=free,
                count=int((N - at) * spare), page=P, reserved=reserved)


def run(c, in_place):
    from paper_2609_04010_gb300 import binding as b
    t = {k: i32(np.atleast_1d(c[k])) for k in ("parent", "kv_len", "table", "shares", "free", "count")}
    if in_place:
        res = b.fork_sequences(t["parent"], t["kv_len"], t["table"], t["shares"], t["free"], t["count"],
                               c["page"], c["reserved"])
        new = t
    else:
        new = {k: torch.full_like(v, -9) for k, v in t.items()}
        res = dict(copies=torch.full((len(c["parent"]), 2), -9, dtype=torch.int32, device="cuda"),
                   flags=torch.full((len(c["parent"]),), -9, dtype=torch.int32, device="cuda"))
        a = b.fork_args(t["parent"], t["kv_len"], new["kv_len"], t["table"], new["table"], t["shares"],
                        new["shares"], t["free"], new["free"], t["count"], new["count"], c["page"],
                        res["copies"], res["flags"], c["reserved"])
        ws = b.new_workspace(b.fork_workspace_size(a))
        for _ in range(3):  # nothing read is changed: every call gives the same
            b.fork_sequences_args(a, ws)
        for k, v in t.items():
            assert np.array_equal(v.cpu().numpy(), np.atleast_1d(c[k]))
    out = dict(new_kv_len=new["kv_len"], new_table=new["table"], new_shares=new["shares"],
               new_free=new["free"], new_count=new["count"], **res)
    return {k: v.cpu().numpy() for k, v in out.items()}


def check(c, in_place):
    want = ref.fork(c["parent"], c["kv_len"], c["table"], c["shares"], c["free"], c["count"], c["page"],
                    c["reserved"])
    got = run(c, in_place)
    for k in want:
        assert np.array_equal(got[k], want[k]), k
    return want


def check_state(c, w):
    """Every page has its holders counted, and is either held or free."""
    N, P, res = len(c["shares"]), c["page"], c["reserved"]
    holders = np.zeros(N, int)
    for b, n in enumerate(w["new_kv_len"]):
        if c["parent"][b] >= 0 and w["flags"][b] == 0:
            np.add.at(holders, w["new_table"][b, :-(-(n + res) // P)], 1)
    top = w["new_count"][0]
    assert np.array_equal(np.maximum(holders - 1, 0), w["new_shares"])
    listed = w["new_free"][:top]
    assert len(set(listed)) == top and not holders[listed].any()


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("kind", ["mixed", "beams", "end", "one"])
@pytest.mark.parametrize("B,P,reserved", [(1, 16, 0), (2, 5, 3), (33, 16, 16), (300, 64, 1), (1025, 16, 0)])
def test_forks(B, P, reserved, kind, in_place):
    c = fork_case(B, P, seed=B + P, reserved=reserved, kind=kind, hi=120 if kind == "one" and B > 100 else 300)
    check_state(c, check(c, in_place))


@pytest.mark.parametrize("spare", [0.0, 0.05, 0.3])
def test_refused_forks(spare):
    c = fork_case(200, 16, seed=3, spare=spare, reserved=4)
    w = check(c, False)
    assert (w["flags"] == 2).any() == (spare < 0.3)
    check(c, True)


def test_long_rows_many_blocks():
    c = fork_case(512, 16, seed=4, hi=8192, reserved=16)
    check_state(c, check(c, False))
    check(c, True)


def test_odd_requests_and_lengths():
    c = fork_case(40, 16, seed=5)
    c["parent"][[3, 9, 11]] = -2, 40, 2 ** 31 - 1
    c["kv_len"][[5, 20]] = -1, 2 ** 31 - 1
    c["parent"][6], c["parent"][7], c["parent"][20] = 5, 20, 1
    w = check(c, False)
    assert set(np.nonzero(w["flags"] == 1)[0]) >= {3, 5, 6, 7, 9, 11, 20}
    check(c, True)


def test_page_ids_out_of_range_are_handed_on():
    c = fork_case(16, 16, seed=6, hi=200)
    rows = np.nonzero(c["kv_len"] > 40)[0][:4]
    c["table"][rows[:2], 1] = -5, len(c["shares"]) + 9
    c["table"][rows[2:], 0] = 2 ** 31 - 1
    check(c, False)
    check(c, True)


def test_a_page_twice_in_one_sequence():
    """A state that cannot arise: the page is freed once, nothing is written out of range."""
    c = fork_case(8, 16, seed=7, kind="end", hi=100)
    b = int(np.argmax(c["kv_len"]))
    c["table"][b, 1] = c["table"][b, 0]
    w = check(c, False)
    assert len(set(w["new_free"][:w["new_count"][0]])) == w["new_count"][0]


def test_state_runs_on():
    """Forks, ends and forks again: the state stays consistent."""
    c = fork_case(64, 16, seed=8, hi=200)
    for step in range(6):
        w = check(c, step % 2 == 0)
        check_state(c, w)
        r = np.random.default_rng(step)
        c.update(kv_len=w["new_kv_len"], table=w["new_table"], shares=w["new_shares"], free=w["new_free"],
                 count=int(w["new_count"][0]), parent=np.where(r.random(64) < 0.2, -1, r.integers(0, 64, 64)))
        c["parent"] = np.where(r.random(64) < 0.4, np.arange(64), c["parent"])


def test_fork_in_a_graph():
    from paper_2609_04010_gb300 import binding as b
    c = fork_case(48, 16, seed=9, kind="beams")
    want = ref.fork(c["parent"], c["kv_len"], c["table"], c["shares"], c["free"], c["count"], 16, 0)
    t = {k: i32(np.atleast_1d(c[k])) for k in ("parent", "kv_len", "table", "shares", "free", "count")}
    first = {k: v.clone() for k, v in t.items()}
    copies = torch.empty(48, 2, dtype=torch.int32, device="cuda")
    a = b.fork_args(t["parent"], t["kv_len"], t["kv_len"], t["table"], t["table"], t["shares"], t["shares"],
                    t["free"], t["free"], t["count"], t["count"], 16, copies)
    ws = b.new_workspace(b.fork_workspace_size(a))
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        b.fork_sequences_args(a, ws)
    for _ in range(2):
        for k, v in t.items():
            v.copy_(first[k])
        g.replay()
        torch.cuda.synchronize()
        assert np.array_equal(t["table"].cpu(), want["new_table"]) and np.array_equal(copies.cpu(), want["copies"])
        assert np.array_equal(t["free"].cpu(), want["new_free"]) and np.array_equal(t["shares"].cpu(), want["new_shares"])


# ----------------------------------------------------------------------------------
# Copies
# ----------------------------------------------------------------------------------
@pytest.mark.parametrize("pages,pairs,shapes", [
    (4, 1, [(1,)]), (9, 4, [(8, 16, 128), (8, 2)]), (64, 20, [(3, 16, 64), (3, 2), (5,), (1, 64, 64)]),
    (40, 17, [(8, 64, 128)] * 6), (7, 3, [(70000,), (70001,)])])
def test_copies(pages, pairs, shapes):
    from paper_2609_04010_gb300 import binding as b
    r = np.random.default_rng(pages)
    g = torch.Generator(device="cuda").manual_seed(pages)
    buffers = [torch.randn(pages, *s, generator=g, device="cuda") for s in shapes]
    buffers += [x.bfloat16() for x in buffers if x[0].numel() % 2 == 0]
    want = [x.clone() for x in buffers]
    at = r.permutation(pages)
    half = pages // 2
    p = np.stack([r.choice(at[:half], pairs), at[half:half + pairs] if pairs <= pages - half else at[-pairs:]], 1)
    for x in want:
        x[torch.from_numpy(p[:, 1]).cuda()] = x[torch.from_numpy(p[:, 0]).cuda()]
    listed = np.insert(p, 1, [-1, -1], 0)
    b.copy_pages(i32(listed), buffers)
    for x, w in zip(buffers, want):
        assert torch.equal(x, w)


def test_copies_of_many_layers_and_bytes():
    from paper_2609_04010_gb300 import binding as b
    caches = [torch.randint(0, 255, (12, 2, 2, 16, 64), dtype=torch.uint8, device="cuda") for _ in range(200)]
    want = [x.clone() for x in caches]
    for x in want:
        x[[7, 3]] = x[[1, 1]]
    b.copy_pages(i32([[1, 7], [1, 3]]), [x.view(torch.float8_e4m3fn) for x in caches])
    assert all(torch.equal(x, w) for x, w in zip(caches, want))


def test_unaligned_buffers():
    from paper_2609_04010_gb300 import binding as b
    store = torch.arange(4 * 1000 + 1, dtype=torch.int32, device="cuda")
    x = store[1:].view(4, 1000)
    want = x.clone()
    want[2] = want[0]
    b.copy_pages(i32([[0, 2]]), [x])
    assert torch.equal(x, want) and int(store[0]) == 0


def test_pairs_out_of_range_are_flagged():
    from paper_2609_04010_gb300 import binding as b
    x = torch.arange(40, dtype=torch.int32, device="cuda").view(5, 8)
    want = x.clone()
    want[3] = want[0]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    b.copy_pages(i32([[-1, -1], [0, 3], [-7, -2]]), [x], status)
    assert int(status) == 0
    b.copy_pages(i32([[0, 3], [-1, 2], [5, 1], [1, 5], [0, -1], [2 ** 31 - 1, 4]]), [x], status)
    assert int(status) == b.FLAG_BAD_PAGE and torch.equal(x, want)
    b.copy_pages(torch.empty(0, 2, dtype=torch.int32, device="cuda"), [x], status)
    assert torch.equal(x, want)
