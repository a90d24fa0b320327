"""Rotary positions and the write into the bf16 cache against a 64-bit reference.

Tolerance: the angle is off by at most 2^-25 of a turn (2 pi 2^-25) plus the rounding of the sine,
products and sum, together below 2^-20 of |x1| + |x2|; the result is rounded once: 2^-8 of it."""

import numpy as np
import pytest
import torch

import serving_reference as ref

pytestmark = pytest.mark.gpu


def i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def check(got, x, positions, freq, interleaved, factor=1.0):
    want = ref.rope(x, positions, freq, interleaved, factor)
    size = factor * ref.rope(x.double().abs(), torch.zeros_like(positions), freq, interleaved)
    mate = size.clone()
    h = freq.numel()
    i = torch.arange(h, device=x.device)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + h)
    mate[..., a] += size[..., b]
    mate[..., b] += size[..., a]
    err = (got.double() - want).abs()
    turned = (positions >= 0)[:, None, None]
    assert bool((torch.where(turned, err - 2.0 ** -8 * want.abs() - 2.0 ** -20 * mate, 0) <= 0).all())


def inputs(R, Hq, Hkv, D, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rows = torch.randn(R, Hq + 2 * Hkv, D, generator=g, device="cuda").bfloat16()
    return rows, *rows.split([Hq, Hkv, Hkv], 1)


@pytest.mark.parametrize("R,Hq,Hkv,D,rot,P", [
    (1, 1, 1, 64, 64, 16), (1, 32, 8, 128, 128, 16), (7, 12, 3, 64, 48, 32), (33, 16, 2, 128, 16, 64),
    (300, 5, 5, 128, 112, 16), (1000, 32, 8, 128, 64, 64), (2500, 8, 1, 64, 32, 32)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_and_cache(R, Hq, Hkv, D, rot, P, interleaved):
    from paper_2609_04010_gb300 import binding as b
    r = np.random.default_rng(R)
    _, q, k, v = inputs(R, Hq, Hkv, D)
    pages = -(-R // P) + 3
    positions = r.integers(0, 200000, R)
    slots = r.permutation(pages * P)[:R]
    positions[r.random(R) < 0.1] = -1
    slots[r.random(R) < 0.1] = -1
    freq, factor = b.rope_frequencies(rot, 500000.0, "yarn", 4.0, original_max=8192)
    assert factor > 1
    kc, vc = (torch.full((pages, Hkv, P, D), 7.0, device="cuda").bfloat16() for _ in range(2))
    positions_t, slots_t = i32(positions), i32(slots)
    q_out, k_out = b.rope_kv(q, k, v, positions_t, b.rope_turns(freq), slots_t, kc, vc, interleaved, factor)
    check(q_out, q, positions_t, freq, interleaved, factor)
    check(k_out, k, positions_t, freq, interleaved, factor)
    assert not q_out[positions_t < 0].any() and not k_out[positions_t < 0].any()
    # the cache holds what came out, and elsewhere what it held
    want_k, want_v = torch.full_like(kc, 7.0), torch.full_like(vc, 7.0)
    put = (positions_t >= 0) & (slots_t >= 0)
    at = slots_t[put].long()
    want_k[at // P, :, at % P], want_v[at // P, :, at % P] = k_out[put], v[put]
    assert torch.equal(kc, want_k) and torch.equal(vc, want_v)


@pytest.mark.parametrize("interleaved", [False, True])
def test_far_positions(interleaved):
    """Frequencies of a turn and positions up to the last one: no whole turn costs precision."""
    from paper_2609_04010_gb300 import binding as b
    _, q, k, v = inputs(64, 2, 1, 64, 1)
    positions = i32(np.linspace(0, 2 ** 31 - 1, 64).astype(np.int64))
    freq, _ = b.rope_frequencies(64, 10000.0)
    q_out, k_out = b.rope_kv(q, k, None, positions, b.rope_turns(freq), interleaved=interleaved)
    # the reference's own angle: frequency * 2^31 in 64 bits is off by 2^-52 * 2^31, far below a bf16 step
    check(q_out, q, positions, freq, interleaved)
    check(k_out, k, positions, freq, interleaved)


def test_in_place_on_the_projection():
    from paper_2609_04010_gb300 import binding as b
    rows, q, k, v = inputs(50, 4, 2, 128, 2)
    before = rows.clone()
    positions = i32(np.arange(50) - 3)
    freq, _ = b.rope_frequencies(128)
    t = b.rope_turns(freq)
    want_q, want_k = b.rope_kv(q, k, None, positions, t)
    b.rope_kv(q, k, None, positions, t, in_place=True)
    assert torch.equal(rows[3:, :4], want_q[3:]) and torch.equal(rows[3:, 4:6], want_k[3:])
    assert torch.equal(rows[:3], before[:3]) and torch.equal(rows[:, 6:], before[:, 6:])


def test_queries_alone_and_keys_alone():
    from paper_2609_04010_gb300 import binding as b
    _, q, k, v = inputs(9, 3, 3, 64, 3)
    positions, t = i32(np.arange(9)), b.rope_turns(b.rope_frequencies(32)[0])
    both = b.rope_kv(q, k, None, positions, t)
    assert torch.equal(b.rope_kv(q, None, None, positions, t)[0], both[0])
    assert torch.equal(b.rope_kv(None, k, None, positions, t)[1], both[1])
    empty = b.rope_kv(q[:0], k[:0], None, positions[:0], t)
    assert empty[0].shape == (0, 3, 64)


def test_special_values_stay_in_their_pair():
    from paper_2609_04010_gb300 import binding as b
    q = torch.ones(2, 1, 64, dtype=torch.bfloat16, device="cuda")
    q[0, 0, 3], q[0, 0, 40], q[1, 0, 63] = float("nan"), float("inf"), float("-inf")
    out, _ = b.rope_kv(q, None, None, i32([5, 0]), b.rope_turns(b.rope_frequencies(32)[0]))
    assert torch.isnan(out[0, 0, [3, 19]]).all() and out[0, 0, 40] == float("inf")
    assert int(torch.isnan(out).sum()) == 2 and out[1, 0, 63] == float("-inf")


def test_slots_past_the_cache_are_flagged():
    from paper_2609_04010_gb300 import binding as b
    _, q, k, v = inputs(4, 1, 1, 64, 4)
    kc, vc = (torch.zeros(2, 1, 16, 64, device="cuda").bfloat16() for _ in range(2))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    t = b.rope_turns(b.rope_frequencies(64)[0])
    b.rope_kv(q, k, v, i32([1, 2, 3, 4]), t, i32([0, 32, 2 ** 31 - 1, -5]), kc, vc, status_ws=status)
    assert int(status) == b.FLAG_BAD_PAGE
    assert torch.equal(vc[0, 0, 0], v[0, 0]) and int((vc != 0).any(-1).sum()) == 1


def test_other_stream_and_graph():
    from paper_2609_04010_gb300 import binding as b
    _, q, k, v = inputs(40, 4, 2, 128, 5)
    positions, t = i32(np.arange(40)), b.rope_turns(b.rope_frequencies(128)[0])
    want = b.rope_kv(q, k, None, positions, t)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = b.rope_kv(q, k, None, positions, t, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(got[0], want[0])
    q_out, k_out = torch.zeros_like(want[0]), torch.zeros_like(want[1])
    a = b.rope_args(q, k, None, positions, t, q_out, k_out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        b.rope_kv_args(a)
    for _ in range(2):
        q_out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(q_out, want[0]) and torch.equal(k_out, want[1])
