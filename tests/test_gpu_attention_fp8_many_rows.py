"""The attention over the 8-bit KV cache with 33 and more query rows a KV head (a kernel of its
own on the tensor cores), where it can go wrong: against the 64-bit host reference with the bounds
of test_gpu_attention_fp8.py, and against the call's own result without the disturbance."""

import numpy as np
import pytest

from test_gpu_attention_fp8 import Case, TENSOR_CORES

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
