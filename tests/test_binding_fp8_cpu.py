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


@pytest.mark.parametrize("R", [2, 200])
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


def test_append_checks_the_status_word():
    k = rows(3, 2, 64)
    for ok in (torch.zeros(256, dtype=torch.uint8), torch.zeros(1, dtype=torch.int32)):
        assert append_args(k, status_ws=gpu(ok)).status == ok.data_ptr()
    for bad, error in ((torch.zeros(256, dtype=torch.uint8), ValueError),             # a host tensor
                       (gpu(torch.zeros(3, dtype=torch.uint8)), ValueError),          # too short
                       (gpu(torch.zeros(512, dtype=torch.uint8)[::2]), ValueError),   # not contiguous
                       (gpu(torch.zeros(4, dtype=torch.float64)), TypeError)):
        with pytest.raises(error):
            append_args(k, status_ws=bad)


def test_append_call_refuses_an_unaligned_status_word():
    import ctypes
    a = append_args(rows(3, 2, 64), status_ws=gpu(torch.zeros(64, dtype=torch.uint8)))
    for p in ("k", "v", "kv_cache", "kv_scale", "slots"):
        setattr(a, p, 1 << 20)
    a.status = (1 << 20) + 2
    assert binding.lib().spec_append_kv_fp8(ctypes.byref(a), None) == 1


def test_append_takes_one_head_whatever_its_stride():
    """[heads][rows][D] with one head: the head's stride is that of all its rows."""
    k = torch.zeros(1, 5, 64, dtype=torch.bfloat16).transpose(0, 1)
    assert k.stride() == (64, 320, 1)
    assert append_args(k).k_row_stride == 64
    wide = torch.zeros(3, 5, 256, dtype=torch.bfloat16)[1:2, :, 64:128].transpose(0, 1)
    assert append_args(wide).k_row_stride == 256
    with pytest.raises(ValueError):
        append_args(torch.zeros(2, 5, 64, dtype=torch.bfloat16).transpose(0, 1))
    with pytest.raises(ValueError):
        append_args(torch.zeros(5, 1, 128, dtype=torch.bfloat16)[..., ::2])
