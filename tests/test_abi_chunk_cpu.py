"""Host-side refusals of the calls that serve ragged batches: nothing here touches a device (the
addresses are made up and never read)."""

import ctypes

import pytest

from paper_2609_04010_gb300 import binding, build

OK_ADDRESS = 1 << 20
BIG = 2 ** 31 - 1


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


def rope(**kw):
    a = fill(binding.RopeArgs(), dict(rows=4, num_q_heads=32, num_kv_heads=8, head_dim=128, rot_dim=64,
                                      page_size=16, num_pages=40),
             ("q", "k", "v", "positions", "turns", "q_out", "slots", "k_cache", "v_cache"))
    return fill(a, kw, ())


def chunk(**kw):
    a = fill(binding.ChunkAttnArgs(), dict(batch=2, rows=9, num_q_heads=32, num_kv_heads=8, head_dim=128,
                                           page_size=16, max_pages_per_seq=10, num_pages=20, causal=1),
             ("q", "k_cache", "v_cache", "page_table", "row_start", "kv_len", "out", "lse"))
    return fill(a, kw, ())


def fork(**kw):
    a = fill(binding.ForkArgs(), dict(batch=4, page_size=16, max_pages_per_seq=10, num_pages=40,
                                      free_capacity=40),
             ("parent", "kv_len", "new_kv_len", "page_table", "new_table", "shares", "new_shares",
              "free_pages", "new_free_pages", "free_count", "new_free_count", "copies", "flags"))
    return fill(a, kw, ())


def copy(pages=(4096, 64), bases=(OK_ADDRESS, OK_ADDRESS), **kw):
    n = len(pages)
    b, s = (ctypes.c_void_p * n)(*bases), (ctypes.c_int64 * n)(*pages)
    a = fill(binding.CopyArgs(), dict(num_pairs=3, num_pages=40, num_buffers=n), ("pairs",))
    a.buffers, a.page_bytes = ctypes.cast(b, ctypes.c_void_p), ctypes.cast(s, ctypes.c_void_p)
    a.arrays = b, s
    return fill(a, kw, ())


@pytest.mark.parametrize("bad,code", [
    (dict(rows=-1), 1), (dict(num_q_heads=-1), 1), (dict(num_kv_heads=-1), 1), (dict(head_dim=0), 1),
    (dict(rot_dim=0), 1), (dict(rot_dim=144), 1), (dict(interleaved=2), 1), (dict(factor=-1.0), 1),
    (dict(factor=float("nan")), 1), (dict(factor=float("inf")), 1), (dict(positions=None), 1),
    (dict(turns=None), 1), (dict(q=None), 1), (dict(q_out=None), 1), (dict(k=None), 1), (dict(v=None), 1),
    (dict(slots=None), 1), (dict(k_cache=None), 1), (dict(v_cache=None), 1), (dict(num_pages=0), 1),
    (dict(page_size=0), 1), (dict(q=OK_ADDRESS + 8), 1), (dict(k=OK_ADDRESS + 2), 1),
    (dict(v=OK_ADDRESS + 4), 1), (dict(q_out=OK_ADDRESS + 8), 1), (dict(k_out=OK_ADDRESS + 8), 1),
    (dict(k_cache=OK_ADDRESS + 8), 1), (dict(turns=OK_ADDRESS + 4), 1), (dict(positions=OK_ADDRESS + 2), 1),
    (dict(slots=OK_ADDRESS + 1), 1), (dict(status=OK_ADDRESS + 2), 1), (dict(q_row_stride=4095), 1),
    (dict(q_row_stride=4088), 1), (dict(k_row_stride=1028), 1), (dict(v_row_stride=8), 1),
    (dict(q_out_row_stride=-8), 1), (dict(k_out_row_stride=1016), 1), (dict(num_q_heads=0), 1),
    (dict(head_dim=96), 2), (dict(rot_dim=24), 2), (dict(rot_dim=8), 2), (dict(page_size=8), 2),
    (dict(num_pages=1 << 28), 2), (dict(num_q_heads=1 << 18), 2), (dict(num_q_heads=BIG, num_kv_heads=BIG), 2)])
def test_rope_refuses(lib, bad, code):
    assert lib.spec_rope_kv(ctypes.byref(rope(**bad)), None) == code
    assert lib.spec_rope_kv(None, None) == 1


def test_rope_without_rows_reads_nothing(lib):
    a = rope(rows=0, q=None, k=None, v=None, positions=None, turns=None, q_out=None)
    assert lib.spec_rope_kv(ctypes.byref(a), None) == 0


@pytest.mark.parametrize("bad,code", [
    (dict(batch=0), 1), (dict(rows=-1), 1), (dict(num_kv_heads=5), 1), (dict(num_q_heads=0), 1),
    (dict(head_dim=0), 1), (dict(causal=2), 1), (dict(causal=-1), 1), (dict(window=-1), 1), (dict(q=None), 1),
    (dict(k_cache=None), 1), (dict(v_cache=None), 1), (dict(kv_cache=OK_ADDRESS), 1),
    (dict(kv_scale=OK_ADDRESS), 1), (dict(k_cache=None, v_cache=None, kv_cache=OK_ADDRESS), 1),
    (dict(k_cache=None, v_cache=None, kv_cache=OK_ADDRESS, kv_scale=OK_ADDRESS + 4), 1),
    (dict(k_cache=None, v_cache=None), 1), (dict(page_table=None), 1), (dict(row_start=None), 1),
    (dict(kv_len=None), 1), (dict(out=None), 1), (dict(q=OK_ADDRESS + 8), 1), (dict(k_cache=OK_ADDRESS + 8), 1),
    (dict(out=OK_ADDRESS + 8), 1), (dict(lse=OK_ADDRESS + 2), 1), (dict(softmax_scale=-1.0), 1),
    (dict(softmax_scale=float("nan")), 1), (dict(path=3), 1), (dict(path=-1), 1), (dict(q_row_stride=4095), 1),
    (dict(q_row_stride=2048), 1), (dict(row_start=OK_ADDRESS + 2), 1), (dict(head_dim=96), 2),
    (dict(page_size=8), 2), (dict(max_pages_per_seq=1 << 27), 2), (dict(num_pages=1 << 28), 2),
    (dict(rows=BIG), 2), (dict(rows=BIG // 4), 2), (dict(num_q_heads=65536, num_kv_heads=65536), 2)])
def test_chunk_refuses(lib, bad, code):
    a = chunk(**bad)
    assert lib.spec_chunk_attention(ctypes.byref(a), OK_ADDRESS, 1 << 40, None) == code
    assert lib.spec_chunk_attn_workspace_size(ctypes.byref(a)) == 0


def test_chunk_workspace(lib):
    a = chunk()
    n = lib.spec_chunk_attn_workspace_size(ctypes.byref(a))
    assert n > 0
    assert lib.spec_chunk_attention(None, OK_ADDRESS, n, None) == 1
    assert lib.spec_chunk_attention(ctypes.byref(a), None, n, None) == 1
    assert lib.spec_chunk_attention(ctypes.byref(a), OK_ADDRESS + 16, n, None) == 1
    assert lib.spec_chunk_attention(ctypes.byref(a), OK_ADDRESS, 255, None) == 3
    empty = chunk(rows=0, q=None, out=None, lse=None)
    assert lib.spec_chunk_attention(ctypes.byref(empty), OK_ADDRESS, n, None) == 0


@pytest.mark.parametrize("bad,code", [
    (dict(batch=0), 1), (dict(page_size=0), 1), (dict(max_pages_per_seq=0), 1), (dict(num_pages=0), 1),
    (dict(reserved=-1), 1), (dict(free_capacity=39), 1), (dict(parent=None), 1), (dict(kv_len=None), 1),
    (dict(new_kv_len=None), 1), (dict(page_table=None), 1), (dict(new_table=None), 1), (dict(shares=None), 1),
    (dict(new_shares=None), 1), (dict(free_pages=None), 1), (dict(new_free_pages=None), 1),
    (dict(free_count=None), 1), (dict(new_free_count=None), 1), (dict(copies=None), 1),
    (dict(parent=OK_ADDRESS + 2), 1), (dict(batch=8193), 2), (dict(max_pages_per_seq=1 << 27), 2),
    (dict(batch=8192, max_pages_per_seq=(1 << 17) + 1, page_size=1), 2), (dict(num_pages=1 << 28, free_capacity=1 << 28), 2),
    (dict(reserved=(1 << 30) + 1), 2)])
def test_fork_refuses(lib, bad, code):
    a = fork(**bad)
    assert lib.spec_fork_sequences(ctypes.byref(a), OK_ADDRESS, 1 << 40, None) == code
    assert lib.spec_fork_workspace_size(ctypes.byref(a)) == 0


def test_fork_workspace(lib):
    a, b = fork(), fork(new_table=OK_ADDRESS + 4096)
    n = lib.spec_fork_workspace_size(ctypes.byref(a))
    assert n > lib.spec_fork_workspace_size(ctypes.byref(b)) > 0  # in place a copy of the table is kept
    assert lib.spec_fork_sequences(None, OK_ADDRESS, n, None) == 1
    assert lib.spec_fork_sequences(ctypes.byref(a), None, n, None) == 1
    assert lib.spec_fork_sequences(ctypes.byref(a), OK_ADDRESS + 16, n, None) == 1
    assert lib.spec_fork_sequences(ctypes.byref(a), OK_ADDRESS, n - 1, None) == 3


@pytest.mark.parametrize("bad,code", [
    (dict(num_pairs=-1), 1), (dict(num_pages=0), 1), (dict(num_buffers=0), 1), (dict(pairs=None), 1),
    (dict(buffers=None), 1), (dict(page_bytes=None), 1), (dict(pairs=OK_ADDRESS + 2), 1),
    (dict(status=OK_ADDRESS + 2), 1), (dict(pages=(4096, 6)), 1), (dict(pages=(0, 4)), 1),
    (dict(bases=(OK_ADDRESS, OK_ADDRESS + 2)), 1), (dict(bases=(None, OK_ADDRESS)), 1),
    (dict(num_buffers=129), 2), (dict(pages=(4, (1 << 40) + 4)), 2)])
def test_copy_refuses(lib, bad, code):
    assert lib.spec_copy_pages(ctypes.byref(copy(**bad)), None) == code
    assert lib.spec_copy_pages(None, None) == 1


def test_copy_without_pairs_reads_nothing(lib):
    assert lib.spec_copy_pages(ctypes.byref(copy(num_pairs=0, pairs=None)), None) == 0
