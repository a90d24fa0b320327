"""What the binding of the 8-bit cache takes and refuses before any call: tensors that say they
are on a GPU, whose addresses are never read."""

import pytest
import torch

from paper_2609_04010_gb300 import binding


class OnGpu(torch.Tensor):
    is_cuda = True


def gpu(t):
    return t.as_subclass(OnGpu)


def append_args(k, v=None, pages=4, P=16, **kw):
    R, H, D = k.shape
    cache = torch.zeros(pages, H, 2, P, D, dtype=torch.uint8).view(torch.float8_e4m3fn)
    return binding.append_fp8_args(gpu(k), gpu(k if v is None else v), gpu(torch.zeros(R, dtype=torch.int32)),
                                   gpu(cache), gpu(torch.zeros(pages, H, 2)), **kw)


def rows(R, H, D):
    return torch.zeros(R, H, D, dtype=torch.bfloat16)


def test_append_takes_rows_of_any_stride_that_do_not_overlap():
    a = append_args(rows(5, 2, 64))
    assert (a.rows, a.k_row_stride, a.v_row_stride) == (5, 128, 128)
    wide = torch.zeros(5, 1024, dtype=torch.bfloat16)
    a = append_args(wide[:, 128:256].unflatten(1, (2, 64)), rows(5, 2, 64))
    assert (a.k_row_stride, a.v_row_stride) == (1024, 128)
    assert append_args(rows(1, 2, 64).expand(1, 2, 64)).k_row_stride == 0


@pytest.mark.parametrize("R", [2, 700])
def test_append_refuses_broadcast_rows(R):
    """A row stride of 0 would read as dense rows, past the one row that there is."""
    one = rows(1, 2, 64).expand(R, 2, 64)
    with pytest.raises(ValueError):
        append_args(one)
    with pytest.raises(ValueError):
        append_args(rows(R, 2, 64), one)
    half = torch.zeros(R * 64 + 64, dtype=torch.bfloat16).as_strided((R, 2, 64), (64, 64, 1))
    with pytest.raises(ValueError):
        append_args(half)
