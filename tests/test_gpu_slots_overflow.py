"""Pages and slots behind requests whose size is wrong, and of rows past max_rows: the requests
that are served have their pages in the table, whatever the others ask for."""

import numpy as np
import pytest

from test_gpu_kv_fp8 import run_slots, slot_case

pytestmark = pytest.mark.gpu

INT32_MAX = 2 ** 31 - 1


def expected(c, max_rows):
    """As fp8_reference.map_slots, without a list of rows (here they are up to 2^31)."""
    P, table = c["page_size"], c["table"].copy()
    B, MP = table.shape
    new_len, flags, start = c["kv_len"].copy(), np.zeros(B, int), [0]
    rows = {k: np.full(max_rows, -1) for k in ("slots", "positions", "row_seq")}
    asked = taken = 0
    for b in range(B):
        n, held = int(c["num_new"][b]), int(c["kv_len"][b])
        if n < 0 or held < 0 or held + n > MP * P:
            flags[b] = 1
        else:
            first = -(-(held + c["reserved"]) // P)
            need = max(0, -(-(held + n) // P) - first)
            if need and asked + need > c["count"]:
                flags[b] = 2
            else:
                table[b, first:first + need] = c["free"][:c["count"]][::-1][asked:asked + need]
                taken, new_len[b] = asked + need if need else taken, held + n
            asked += need
        at = np.arange(start[-1], min(start[-1] + max(n, 0), max_rows))
        pos = held + at - start[-1]
        rows["positions"][at], rows["row_seq"][at] = pos, b
        if flags[b] == 0:
            rows["slots"][at] = table[b, pos // P] * P + pos % P
        start.append(min(start[-1] + max(n, 0), INT32_MAX))
    return dict(rows, table=table, new_len=new_len, flags=flags, row_start=np.array(start),
                count=c["count"] - taken)


def check(c, max_rows):
    want, got = expected(c, max_rows), run_slots(c, max_rows)
    for k in want:
        assert np.array_equal(np.ravel(got[k]), np.ravel(want[k])), k


@pytest.mark.parametrize("bad", [(0,), (0, 1), (3,), (2, 5, 6)])
@pytest.mark.parametrize("size", [INT32_MAX, INT32_MAX // 2, 2 ** 30 + 7])
@pytest.mark.parametrize("max_rows", [1, 300, 5000])
def test_requests_of_a_wrong_size(bad, size, max_rows):
    c = slot_case(9, 16, seed=len(bad), hi_new=200)
    c["num_new"][list(bad)] = size
    check(c, max_rows)


@pytest.mark.parametrize("B,P", [(7, 16), (600, 5), (40, 64)])
@pytest.mark.parametrize("spare,reserved", [(1.0, 0), (0.6, 0), (0.8, 16)])
def test_rows_past_max_rows(B, P, spare, reserved):
    c = slot_case(B, P, seed=B + P, spare=spare, reserved=reserved, hi_new=300)
    for max_rows in (1, 2, int(c["num_new"].sum()) // 2, int(c["num_new"].sum())):
        check(c, max_rows)


def test_a_refused_request_larger_than_the_cache():
    """Refused for its pages (flag 2) between two that are served."""
    c = slot_case(3, 16, seed=4, hi_new=200)
    c["table"] = np.pad(c["table"], ((0, 0), (0, 2 ** 20)), constant_values=-1)
    c["num_new"][:] = [5, 2 ** 24, 0]
    check(c, 64)
