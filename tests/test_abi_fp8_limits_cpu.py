"""Sizes past the 32-bit counts of the 8-bit cache's kernels and the logit constraints are refused
on the host, before anything is launched (the addresses are made up and never read)."""

import ctypes

import pytest

from test_abi_fp8_cpu import OK_ADDRESS, adjust, attn, lib  # noqa: F401


@pytest.mark.parametrize("path", [0, 1, 2])
@pytest.mark.parametrize("heads,gamma", [(1 << 26, 64), (1 << 30, 2), (1 << 30, 4), ((1 << 31) - 255, 1)])
def test_attention_refuses_more_rows_than_it_counts(lib, path, heads, gamma):  # noqa: F811
    a = attn(num_q_heads=heads, num_kv_heads=1, gamma=gamma, path=path)
    assert lib.spec_attn_fp8_workspace_size(ctypes.byref(a)) == 0
    assert lib.spec_verify_attention_fp8(ctypes.byref(a), OK_ADDRESS, 1 << 40, None) == 2


@pytest.mark.parametrize("vocab", [65535 * 2048 + 1, 2 ** 31 - 1])
def test_adjust_refuses_vocabularies_past_the_grid(lib, vocab):  # noqa: F811
    assert lib.spec_adjust_logits(ctypes.byref(adjust(vocab=vocab)), None) == 2
