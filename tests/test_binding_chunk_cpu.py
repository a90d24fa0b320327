"""What the binding of the ragged-batch calls takes and refuses before any call: tensors that say
they are on a GPU, whose addresses are never read; and the tables of rotary frequencies."""

import math

import pytest
import torch

from paper_2609_04010_gb300 import binding as b


class OnGpu(torch.Tensor):
    is_cuda = True


def gpu(t):
    return t.as_subclass(OnGpu)


def i32(*shape):
    return gpu(torch.zeros(shape, dtype=torch.int32))


def bf16(*shape):
    return gpu(torch.zeros(shape, dtype=torch.bfloat16))


def turns(n=32):
    return gpu(torch.zeros(n, dtype=torch.int64))


def rope(R=5, **kw):
    a = dict(q=bf16(R, 4, 64), k=bf16(R, 2, 64), v=bf16(R, 2, 64), positions=i32(R), turns=turns(),
             q_out=bf16(R, 4, 64), slots=i32(R), k_cache=bf16(7, 2, 16, 64), v_cache=bf16(7, 2, 16, 64))
    a.update(kw)
    return b.rope_args(**a)


def test_rope_takes_column_ranges():
    wide = gpu(torch.zeros(5, 8, 64, dtype=torch.bfloat16))
    a = rope(q=wide[:, :4], k=wide[:, 4:6], v=wide[:, 6:], q_out=wide[:, :4])
    assert (a.q_row_stride, a.k_row_stride, a.v_row_stride, a.q_out_row_stride) == (512,) * 4
    assert (a.rows, a.num_q_heads, a.num_kv_heads, a.rot_dim, a.num_pages, a.page_size) == (5, 4, 2, 64, 7, 16)
    assert a.q == a.q_out and a.k_out is None
    assert rope(q=None, q_out=None).num_q_heads == 0
    only_q = rope(k=None, v=None, slots=None, k_cache=None, v_cache=None)
    assert only_q.num_kv_heads == 0 and only_q.k is None


@pytest.mark.parametrize("bad,error", [
    (dict(q=torch.zeros(5, 4, 64, dtype=torch.bfloat16)), ValueError), (dict(k=bf16(4, 2, 64)), ValueError),
    (dict(q=gpu(torch.zeros(5, 4, 64))), TypeError), (dict(q_out=None), ValueError),
    (dict(k_cache=None), ValueError), (dict(slots=None), ValueError), (dict(v=None), ValueError),
    (dict(k=None), ValueError), (dict(positions=i32(4)), ValueError), (dict(slots=i32(6)), ValueError),
    (dict(turns=gpu(torch.zeros(32))), TypeError), (dict(turns=gpu(torch.zeros(4, 8, dtype=torch.int64))), ValueError),
    (dict(k_cache=bf16(7, 3, 16, 64)), ValueError), (dict(v_cache=bf16(7, 2, 32, 64)), ValueError),
    (dict(q=gpu(torch.zeros(1, 4, 64, dtype=torch.bfloat16).expand(5, 4, 64))), ValueError),
    (dict(q=gpu(torch.zeros(5, 4, 128, dtype=torch.bfloat16)[..., ::2])), ValueError),
    (dict(factor=0.0), ValueError), (dict(status_ws=gpu(torch.zeros(3, dtype=torch.uint8))), ValueError)])
def test_rope_refuses(bad, error):
    with pytest.raises(error):
        rope(**bad)


def chunk(R=6, **kw):
    a = dict(q=bf16(R, 4, 64), cache=(bf16(7, 2, 16, 64), bf16(7, 2, 16, 64)), page_table=i32(3, 5),
             row_start=i32(4), kv_len=i32(3), out=bf16(R, 4, 64), lse=gpu(torch.zeros(R, 4)))
    a.update(kw)
    return b.chunk_attn_args(**a)


def cache8(pages=7, H=2, P=16, D=64):
    return (gpu(torch.zeros(pages, H, 2, P, D, dtype=torch.uint8).view(torch.float8_e4m3fn)),
            gpu(torch.zeros(pages, H, 2)))


def test_chunk_takes_both_caches_and_column_ranges():
    a = chunk(q=gpu(torch.zeros(6, 8, 64, dtype=torch.bfloat16))[:, :4])
    assert (a.batch, a.rows, a.q_row_stride, a.kv_cache, a.kv_scale, a.causal) == (3, 6, 512, None, None, 1)
    a = chunk(cache=cache8(), causal=False, window=9, lse=None)
    assert a.k_cache is None and a.kv_cache and a.kv_scale and (a.causal, a.window, a.lse) == (0, 9, None)


@pytest.mark.parametrize("bad,error", [
    (dict(cache=(bf16(7, 2, 16, 64), bf16(7, 2, 32, 64))), ValueError), (dict(cache=cache8(D=128)), ValueError),
    (dict(cache=(cache8()[0], gpu(torch.zeros(7, 2)))), ValueError), (dict(row_start=i32(3)), ValueError),
    (dict(page_table=i32(2, 5)), ValueError), (dict(out=bf16(5, 4, 64)), ValueError),
    (dict(lse=gpu(torch.zeros(6, 2))), ValueError), (dict(kv_len=gpu(torch.zeros(3))), TypeError),
    (dict(q=gpu(torch.zeros(6, 4, 64))), TypeError), (dict(cache=(bf16(7, 2, 16), bf16(7, 2, 16))), ValueError)])
def test_chunk_refuses(bad, error):
    with pytest.raises(error):
        chunk(**bad)


def test_fork_and_copy_refuse():
    i = [i32(3), i32(3), i32(3), i32(3, 5), i32(3, 5), i32(9), i32(9), i32(9), i32(9), i32(1), i32(1)]
    assert b.fork_args(*i, 16, i32(3, 2)).num_pages == 9
    for at, bad in ((0, i32(4)), (4, i32(3, 6)), (6, i32(8)), (8, i32(10)), (9, i32(2)),
                    (1, torch.zeros(3, dtype=torch.int32))):
        with pytest.raises(ValueError):
            b.fork_args(*i[:at], bad, *i[at + 1:], 16, i32(3, 2))
    with pytest.raises(ValueError):
        b.fork_args(*i, 16, i32(3, 3))
    a = b.copy_args(i32(4, 2), [bf16(7, 2, 16, 64), cache8()[1]])
    assert (a.num_pairs, a.num_pages, a.num_buffers, list(a.arrays[1])) == (4, 7, 2, [4096, 16])
    for bad in ([], [bf16(7, 64), bf16(6, 64)], [bf16(7, 64)[:, ::2]], [torch.zeros(7, 4)]):
        with pytest.raises(ValueError):
            b.copy_args(i32(4, 2), bad)
    with pytest.raises(ValueError):
        b.copy_args(i32(8), [bf16(7, 64)])


def test_tensors_of_two_devices_are_refused():
    class Elsewhere(torch.Tensor):
        is_cuda = True
        device = torch.device("cuda", 1)
    with pytest.raises(ValueError, match="one device"):
        chunk(kv_len=torch.zeros(3, dtype=torch.int32).as_subclass(Elsewhere))


def test_turns_are_frequencies_modulo_a_turn():
    f = torch.tensor([1.0, 0.25, 1e-6, 2 * math.pi, 7.0, 0.0], dtype=torch.float64)
    t = b.rope_turns(f)
    for x, w in zip(f.tolist(), t.tolist()):
        turn = x / (2 * math.pi)
        assert abs((w % 2 ** 64) / 2.0 ** 64 - turn % 1.0) < 2.0 ** -52
    # a far position: the product overflows by whole turns and keeps the fraction
    pos = 2 ** 31 - 1
    w = t[0].item() * pos % 2 ** 64 / 2.0 ** 64
    assert abs(math.remainder(2 * math.pi * w - math.fmod(pos * 1.0, 2 * math.pi), 2 * math.pi)) < 1e-5
    with pytest.raises(ValueError):
        b.rope_turns(torch.zeros(4, dtype=torch.int64))


def test_frequency_tables():
    plain, one = b.rope_frequencies(64, 10000.0, device="cpu")
    assert plain.numel() == 32 and one == 1.0
    assert plain[0] == 1.0 and abs(plain[16].item() - 0.01) < 1e-15
    linear, one = b.rope_frequencies(64, scaling="linear", factor=4.0, device="cpu")
    assert torch.equal(linear, plain / 4) and one == 1.0
    ntk, _ = b.rope_frequencies(64, scaling="ntk", factor=4.0, device="cpu")
    assert ntk[0] == 1.0 and abs(ntk[31].item() / (plain[31].item() / 4) - 1) < 1e-12
    for name, mult in (("yarn", 0.1 * math.log(8.0) + 1), ("bands", 1.0)):
        got, factor = b.rope_frequencies(128, 500000.0, name, 8.0, original_max=8192, device="cpu")
        base, _ = b.rope_frequencies(128, 500000.0, device="cpu")
        share = base / got
        assert abs(factor - mult) < 1e-12
        assert torch.equal(got[:5], base[:5]) and torch.allclose(got[-5:], base[-5:] / 8, rtol=1e-14)
        assert bool((share.diff() >= -1e-12).all()) and bool(((share >= 1 - 1e-12) & (share <= 8 + 1e-12)).all())
    for bad in (dict(scaling="other"), dict(scaling="yarn", factor=2.0), dict(factor=0.5), dict(base=1.0),
                dict(scaling="bands", original_max=5, low=4.0, high=1.0)):
        with pytest.raises(ValueError):
            b.rope_frequencies(64, device="cpu", **bad)
    with pytest.raises(ValueError):
        b.rope_frequencies(63, device="cpu")
