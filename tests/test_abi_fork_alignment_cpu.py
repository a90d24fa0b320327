"""Every array of a fork is checked for its alignment before anything is launched (the addresses are made
up and never read)."""

import ctypes

import pytest

from paper_2609_04010_gb300 import binding
from test_abi_chunk_cpu import OK_ADDRESS, fork, lib  # noqa: F401

ARRAYS = [n for n, t in binding.ForkArgs._fields_ if t is ctypes.c_void_p]


@pytest.mark.parametrize("name", ARRAYS)
@pytest.mark.parametrize("off", [1, 2, 3])
def test_fork_refuses_misaligned(lib, name, off):  # noqa: F811
    a = fork(**{name: OK_ADDRESS + off})
    assert lib.spec_fork_workspace_size(ctypes.byref(a)) == 0
    assert lib.spec_fork_sequences(ctypes.byref(a), OK_ADDRESS, 1 << 40, None) == 1


def test_all_arrays_are_there():
    assert len(ARRAYS) == 13 and "new_free_count" in ARRAYS and "flags" in ARRAYS
