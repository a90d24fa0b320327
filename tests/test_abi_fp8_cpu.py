"""Host-side refusals of the 8-bit KV cache calls and of the logit constraints: nothing
here touches a device (the addresses are made up and never read)."""

import ctypes

import pytest
import torch

from paper_2609_04010_gb300 import binding, build

OK_ADDRESS = 1 << 20


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.lib()


def fill(a, values, pointers):
    for k, v in values.items():
        setattr(a, k, v)
    for k in pointers:
        setattr(a, k, OK_ADDRESS)
    return a


def slots(**kw):
    a = fill(binding.SlotArgs(), dict(batch=4, page_size=16, max_pages_per_seq=10, num_pages=40,
                                      reserved=0, max_rows=64, free_capacity=40),
             ("num_new", "kv_len", "new_len", "page_table", "free_pages", "free_count",
              "new_free_count", "row_start", "slots", "positions", "row_seq", "flags"))
    return fill(a, kw, ())


def append(**kw):
    a = fill(binding.AppendFp8Args(), dict(rows=4, num_kv_heads=8, head_dim=128, page_size=16,
                                           num_pages=40),
             ("k", "v", "slots", "kv_cache", "kv_scale"))
    return fill(a, kw, ())


def attn(**kw):
    a = fill(binding.AttnFp8Args(), dict(batch=2, gamma=4, num_q_heads=32, num_kv_heads=8,
                                         head_dim=128, page_size=16, max_pages_per_seq=10,
                                         num_pages=20, softmax_scale=0.0, path=0),
             ("q", "kv_cache", "kv_scale", "page_table", "kv_len", "out", "lse"))
    return fill(a, kw, ())


def adjust(**kw):
    a = fill(binding.AdjustArgs(), dict(batch=2, gamma=4, vocab=1000, logits_dtype=1,
                                        block_shift=0, max_history=5, max_bias=3),
             ("logits", "out", "history", "history_len", "bias_tokens", "bias_values"))
    return fill(a, kw, ())


@pytest.mark.parametrize("bad,code", [
    (dict(batch=0), 1), (dict(page_size=0), 1), (dict(max_pages_per_seq=0), 1), (dict(num_pages=0), 1),
    (dict(reserved=-1), 1), (dict(max_rows=0), 1), (dict(free_capacity=-1), 1), (dict(num_new=None), 1),
    (dict(kv_len=None), 1), (dict(new_len=None), 1), (dict(page_table=None), 1), (dict(free_pages=None), 1),
    (dict(free_count=None), 1), (dict(new_free_count=None), 1), (dict(row_start=None), 1),
    (dict(slots=None), 1), (dict(batch=8193), 2), (dict(max_pages_per_seq=1 << 27), 2),
    (dict(num_pages=1 << 28), 2), (dict(reserved=(1 << 30) + 1), 2)])
def test_map_slots_refuses(lib, bad, code):
    a = slots(**bad)
    assert lib.spec_map_slots(ctypes.byref(a), OK_ADDRESS, 1 << 20, None) == code
    assert lib.spec_slot_workspace_size(ctypes.byref(a)) == 0


def test_map_slots_workspace(lib):
    a = slots()
    n = lib.spec_slot_workspace_size(ctypes.byref(a))
    assert n > 0
    assert lib.spec_map_slots(None, OK_ADDRESS, n, None) == 1
    assert lib.spec_map_slots(ctypes.byref(a), None, n, None) == 1
    assert lib.spec_map_slots(ctypes.byref(a), OK_ADDRESS + 16, n, None) == 1
    assert lib.spec_map_slots(ctypes.byref(a), OK_ADDRESS, n - 1, None) == 3


@pytest.mark.parametrize("bad,code", [
    (dict(rows=-1), 1), (dict(num_kv_heads=0), 1), (dict(num_pages=0), 1), (dict(head_dim=0), 1),
    (dict(k=None), 1), (dict(v=None), 1), (dict(slots=None), 1), (dict(kv_cache=None), 1),
    (dict(kv_scale=None), 1), (dict(k=OK_ADDRESS + 2), 1), (dict(v=OK_ADDRESS + 8), 1),
    (dict(kv_cache=OK_ADDRESS + 8), 1), (dict(kv_scale=OK_ADDRESS + 2), 1),
    (dict(k_row_stride=1023), 1), (dict(v_row_stride=1028), 1), (dict(k_row_stride=512), 1),
    (dict(head_dim=96), 2), (dict(page_size=8), 2), (dict(page_size=128), 2),
    (dict(num_kv_heads=65536), 2), (dict(num_pages=1 << 28), 2)])
def test_append_refuses(lib, bad, code):
    assert lib.spec_append_kv_fp8(ctypes.byref(append(**bad)), None) == code
    assert lib.spec_append_kv_fp8(None, None) == 1


def test_append_without_rows_reads_nothing(lib):
    assert lib.spec_append_kv_fp8(ctypes.byref(append(rows=0, k=None, v=None, slots=None)), None) == 0


@pytest.mark.parametrize("bad,code", [
    (dict(batch=0), 1), (dict(gamma=0), 1), (dict(num_kv_heads=5), 1), (dict(head_dim=0), 1),
    (dict(q=None), 1), (dict(kv_cache=None), 1), (dict(kv_scale=None), 1), (dict(page_table=None), 1),
    (dict(kv_len=None), 1), (dict(out=None), 1), (dict(q=OK_ADDRESS + 8), 1),
    (dict(kv_cache=OK_ADDRESS + 8), 1), (dict(out=OK_ADDRESS + 8), 1), (dict(kv_scale=OK_ADDRESS + 4), 1),
    (dict(softmax_scale=-1.0), 1), (dict(softmax_scale=float("nan")), 1), (dict(path=3), 1),
    (dict(path=-1), 1), (dict(gamma=65), 2), (dict(head_dim=96), 2), (dict(page_size=8), 2),
    (dict(max_pages_per_seq=1 << 27), 2), (dict(num_pages=1 << 28), 2)])
def test_attention_refuses(lib, bad, code):
    a = attn(**bad)
    assert lib.spec_verify_attention_fp8(ctypes.byref(a), OK_ADDRESS, 1 << 40, None) == code
    assert lib.spec_attn_fp8_workspace_size(ctypes.byref(a)) == 0


def test_attention_workspace(lib):
    a = attn()
    assert lib.spec_attn_fp8_workspace_size(ctypes.byref(a)) > 0
    assert lib.spec_verify_attention_fp8(None, OK_ADDRESS, 1 << 40, None) == 1
    assert lib.spec_verify_attention_fp8(ctypes.byref(a), None, 1 << 40, None) == 1
    assert lib.spec_verify_attention_fp8(ctypes.byref(a), OK_ADDRESS + 128, 1 << 40, None) == 1


def test_attention_workspace_does_not_grow_with_the_batch(lib):
    """On the tensor cores only units that are split between blocks have partial results: two a
    block, of 64 rows of two heads here (fp32 outputs and 8 bytes more), on up to 256 SMs."""
    a = attn(batch=100000, gamma=16, num_q_heads=32, num_kv_heads=8, head_dim=128)
    counters = 100000 * 8 * 4 * 4  # the other path's
    assert lib.spec_attn_fp8_workspace_size(ctypes.byref(a)) <= 2 * 256 * 128 * (128 * 4 + 8) + counters + 65536


@pytest.mark.parametrize("bad,code", [
    (dict(batch=0), 1), (dict(gamma=0), 1), (dict(vocab=0), 1), (dict(logits_dtype=2), 1),
    (dict(block_shift=2), 1), (dict(max_history=-1), 1), (dict(max_bias=-1), 1), (dict(logits=None), 1),
    (dict(out=None), 1), (dict(history=None), 1), (dict(history_len=None), 1),
    (dict(bias_tokens=None), 1), (dict(bias_values=None), 1), (dict(logits=OK_ADDRESS + 1), 1),
    (dict(logits_dtype=0, out=OK_ADDRESS + 2), 1), (dict(gamma=65), 2), (dict(batch=65536), 2)])
def test_adjust_refuses(lib, bad, code):
    assert lib.spec_adjust_logits(ctypes.byref(adjust(**bad)), None) == code
    assert lib.spec_adjust_logits(None, None) == 1


def test_binding_refuses_wrong_tensors():
    f8 = torch.zeros(4, 2, 2, 16, 64, dtype=torch.uint8).view(torch.float8_e4m3fn)
    sc, s = torch.zeros(4, 2, 2), torch.zeros(3, dtype=torch.int32)
    k = torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):  # host tensors
        binding.append_fp8_args(k, k, s, f8, sc)
    with pytest.raises(TypeError):
        binding.append_fp8_args(k, k, s, f8.view(torch.uint8), sc)
    with pytest.raises(ValueError):
        binding.attn_fp8_args(k.view(1, 3, 2, 64), f8, sc, s.view(1, 3), s[:1], k.view(1, 3, 2, 64))
    with pytest.raises(ValueError):
        binding.adjust_args(sc, sc)
    with pytest.raises(TypeError):
        binding.adjust_args(sc.half(), sc.half())
    with pytest.raises(ValueError):
        binding.slot_args(s, s, s, s.view(1, 3), 16, 4, s, s[:1], s[:1], s, s)
