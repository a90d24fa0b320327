"""Rotary positions of as many rows as take several a block (8 from 64 rows an SM on), the last block of
which is not full: each row as where it is rotated alone."""

import numpy as np
import pytest
import torch

from test_gpu_rope import check, i32, inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Hq,Hkv,D,rot,P", [(4, 1, 64, 64, 16), (5, 2, 64, 16, 32), (8, 2, 128, 128, 64), (3, 3, 128, 80, 16)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("extra", [0, 1, 7])
def test_rope_of_long_prompts(Hq, Hkv, D, rot, P, interleaved, extra):
    from paper_2609_04010_gb300 import binding as b
    R = 64 * torch.cuda.get_device_properties(0).multi_processor_count + extra
    r = np.random.default_rng(R)
    _, q, k, v = inputs(R, Hq, Hkv, D, seed=extra)
    pages = -(-R // P) + 3
    positions, slots = r.integers(0, 200000, R), r.permutation(pages * P)[:R]
    positions[r.random(R) < 0.1] = -1
    slots[r.random(R) < 0.1] = -1
    slots[R - 1], positions[R - 1] = pages * P, 5  # past the cache
    freq, factor = b.rope_frequencies(rot, 500000.0, "yarn", 4.0, original_max=8192)
    kc, vc = (torch.full((pages, Hkv, P, D), 7.0, device="cuda").bfloat16() for _ in range(2))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    pos, at, turns = i32(positions), i32(slots), b.rope_turns(freq)
    q_out, k_out = b.rope_kv(q, k, v, pos, turns, at, kc, vc, interleaved, factor, status_ws=status)
    assert int(status) == b.FLAG_BAD_PAGE
    check(q_out, q, pos, freq, interleaved, factor)
    check(k_out, k, pos, freq, interleaved, factor)
    want_k, want_v = torch.full_like(kc, 7.0), torch.full_like(vc, 7.0)
    put = (pos >= 0) & (at >= 0) & (at < pages * P)
    to = at[put].long()
    want_k[to // P, :, to % P], want_v[to // P, :, to % P] = k_out[put], v[put]
    assert torch.equal(kc, want_k) and torch.equal(vc, want_v)
    # in parts that take a row a block
    parts = [b.rope_kv(q[i:i + 1000], k[i:i + 1000], None, pos[i:i + 1000], turns, interleaved=interleaved, factor=factor)
             for i in range(0, R, 1000)]
    assert torch.equal(torch.cat([p[0] for p in parts]), q_out) and torch.equal(torch.cat([p[1] for p in parts]), k_out)
    # and in place, on the projection itself
    b.rope_kv(q, k, None, pos, turns, interleaved=interleaved, factor=factor, in_place=True)
    turned = pos >= 0
    assert torch.equal(q[turned], q_out[turned]) and torch.equal(k[turned], k_out[turned])
