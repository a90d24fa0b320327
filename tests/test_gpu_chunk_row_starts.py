"""Sequences whose rows lie in [0, rows) in order are served beside others that are left out, whatever the
other entries of row_start are."""

import pytest
import torch

import chunk_reference as ref
from test_gpu_chunk import make, run

pytestmark = pytest.mark.gpu
AUTO, CUDA_CORES = 0, 1


@pytest.mark.parametrize("path", [CUDA_CORES, AUTO])
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("starts,good", [
    ([0, 5, -1, 25, 30], [0, 3]), ([0, 5, 1000, 25, 30], [0, 3]), ([0, 100, 0, 5, 9], [2, 3]),
    ([7, 9, 2 ** 31 - 1, 0, 5], [0, 3]), ([-2 ** 31, 20, 30, 2 ** 31 - 1, 3], [1]), ([30, 31, 0, 1, 17], [2, 3]),
    ([0, 1, 2, 31, 30], [0, 1]), ([0, 0, 30, 30, 30], [1])])
def test_good_sequences_beside_bad_ones(path, fp8, starts, good):
    from paper_2609_04010_gb300 import binding as b
    c = make([10, 10, 5, 5], [300, 40, 700, 0], Hq=8, Hkv=4, D=64, fp8=fp8, seed=51)
    assert c["rows"] == 30
    c["starts"] = starts
    c["lens"] = [300, 50, 705, 30]
    c["table"][:] = c["table"][2]  # (pages enough for every length)
    out, lse, code, flags = run(c, path)
    want = [torch.full_like(out, 5.0, dtype=torch.float64), torch.full_like(lse, 5.0, dtype=torch.float64)]
    want += [torch.zeros_like(want[0]), torch.zeros_like(want[1]), torch.zeros_like(want[0])]
    for i in good:
        r0, r1 = starts[i], starts[i + 1]
        one = dict(c, q=c["q"][r0:r1], table=c["table"][i:i + 1], starts=[0, r1 - r0], lens=[c["lens"][i]])
        for w, x in zip(want, ref.attend(one)):
            w[r0:r1] = x
    ref.check((out, lse), want, c, path == CUDA_CORES)
    bad = any(not (0 <= starts[i] <= starts[i + 1] <= 30) for i in range(4))
    assert (code, flags) == ((5, b.FLAG_BAD_KV_LEN) if bad else (0, 0))


@pytest.mark.parametrize("path", [CUDA_CORES, AUTO])
def test_many_short_sequences_between_empty_ones(path):
    """One to three tokens each, groups that fill no block, empty sequences at both ends and between."""
    new = [0, 0] + [i % 4 for i in range(400)] + [0]
    c = make(new, [(7 * i) % 90 + (n == 0) for i, n in enumerate(new)], Hq=6, Hkv=2, D=64, seed=52, extra_rows=3)
    out, lse, code, _ = run(c, path)
    used = c["starts"][-1]
    assert code == 0 and bool((out[used:] == 5).all())
    ref.check((out[:used], lse[:used]), [x[:used] for x in ref.attend(c)], c, path == CUDA_CORES)
