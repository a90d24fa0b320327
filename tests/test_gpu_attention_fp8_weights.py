"""Rows of the attention over the 8-bit KV cache that one key dominates: what the other keys
add to the output, which is most of it where the dominating key's value is small.

Tolerance. A weight enters the tensor-core products as three e5m2 terms of its fp16 value:
two cut off after three bits, the last rounded, so it is off by at most
2^-9 + 2^-11 = 1.25 * 2^-9 of itself, or, where it is small, by 2^-28 of the row's largest
weighted value scale. Queries, keys and scores as in test_gpu_attention_fp8.py, whose
ds bounds a score's error. So with a value scale that all pages share
  |do| <= (1.25 * 2^-9 + 2 |ds|) * sum_t p_t |v_t| + 2^-28 * max_t p_t * sum_t |v_t| + 2^-9 |o|,
and as a whole, where the weights' errors are independent, 2^-8 of the output's norm.
"""

import numpy as np
import pytest
import torch

import fp8_reference as ref
from test_gpu_attention_fp8 import CUDA_CORES, TENSOR_CORES, i32

pytestmark = pytest.mark.gpu

# (gamma, Hq, Hkv): rows of a KV head of 4, 16, 32 (few: the keys on the MMA's M side) and of 48,
# 256 (many: the rows), two heads a block and one
LAYOUTS = [(1, 8, 2), (4, 4, 1), (8, 8, 2), (12, 8, 2), (16, 16, 1)]


def dominated(B, G, Hq, H, D, n, share, mean, seed):
    """B sequences that share the n keys of one page table. The first key has about `share` of
    every row's weight and values of a hundredth of the others', whose mean is `mean` of their
    deviation; the scores of the others are normal."""
    r = np.random.default_rng(seed)
    P, pages = 64, -(-n // 64)
    k = r.standard_normal((n, H, D))
    k[:, :, 0] = 0.0
    k[0] = 0.0
    k[0, :, 0] = np.log(share / (1 - share) * n * np.exp(0.5)) * D ** 0.5 / 16
    v = r.standard_normal((n, H, D)) + mean
    v[0] *= 0.01
    codes = np.zeros((pages, H, 2, P, D), np.uint8)
    scale = np.full((pages, H, 2), 2.0 ** -6, np.float32)
    scale[0, :, 0] = 2.0 ** -4  # the first key is larger than the others
    for kind, x in ((0, k), (1, v)):
        x = np.pad(x, ((0, pages * P - n), (0, 0), (0, 0))).reshape(pages, P, H, D).transpose(0, 2, 1, 3)
        codes[:, :, kind] = ref.encode(x / scale[:, :, kind, None, None])
    q = r.standard_normal((B, G, Hq, D)).astype(np.float32)
    q[..., 0] = 16.0
    table = np.broadcast_to(np.arange(pages), (B, pages))
    return torch.from_numpy(q).bfloat16(), codes, scale, table, np.full(B, n)


def attention(q, codes, scale, n):
    """One sequence's causal attention over pages 0, 1, ..: out, lse, sum_t p_t |v_t|, sum_t |v_t|,
    max_t sum_d |k_td|."""
    G, Hq, D = q.shape
    H = codes.shape[1]
    x = (ref.decode(codes) * scale.astype(np.float64)[..., None, None]).transpose(1, 2, 0, 3, 4).reshape(H, 2, -1, D)[:, :, :n]
    out, lse, mass = np.zeros(q.shape), np.zeros((G, Hq)), np.zeros(q.shape)
    vsum, kmax = np.zeros((Hq, D)), np.zeros(Hq)
    hidden = np.arange(n)[None] > n - G + np.arange(G)[:, None]
    for h in range(Hq):
        k, v = x[h * H // Hq]
        s = np.where(hidden, -np.inf, q[:, h] @ k.T * D ** -0.5)
        w = np.exp(s - s.max(1, keepdims=True))
        lse[:, h] = s.max(1) + np.log(w.sum(1))
        w /= w.sum(1, keepdims=True)
        out[:, h], mass[:, h] = w @ v, w @ np.abs(v)
        vsum[h], kmax[h] = np.abs(v).sum(0), np.abs(k).sum(1).max()
    return out, lse, mass, vsum, kmax


def check(case, path, at):
    from paper_2609_04010_gb300 import binding as b
    q, codes, scale, table, kv_len = case
    o, l = b.verify_attention_fp8(q.cuda(), torch.from_numpy(codes).cuda().view(torch.float8_e4m3fn),
                                  torch.from_numpy(scale).cuda(), i32(table), i32(kv_len), path=path)
    G, Hq, D = q.shape[1:]
    H = codes.shape[1]
    for s in at:
        x = q[s].double().numpy()
        ro, rl, mass, vsum, kmax = attention(x, codes, scale, int(kv_len[s]))
        qmax = np.repeat(np.abs(x).reshape(G, H, -1).max((0, 2)), Hq // H)
        ds = D ** -0.5 * kmax * (2.0 ** -18 + 128 * 2.0 ** -24) * qmax
        tol = (1.25 * 2.0 ** -9 + 2 * ds[:, None]) * mass + 2.0 ** -28 * vsum + 2.0 ** -9 * np.abs(ro)
        err = np.abs(o[s].float().cpu().numpy() - ro)
        whole = np.linalg.norm(err) / np.linalg.norm(ro)
        assert (err / tol).max() <= 1 and whole <= 2.0 ** -8, ((err / tol).max(), whole)
        assert (np.abs(l[s].cpu().numpy() - rl) / (ds + 2.0 ** -20 * (1 + np.abs(rl)))).max() <= 1


@pytest.mark.parametrize("G,Hq,H", LAYOUTS)
@pytest.mark.parametrize("D,n", [(128, 8192), (64, 8200), (128, 32768)])
@pytest.mark.parametrize("share", [0.5, 0.9])
@pytest.mark.parametrize("mean", [0.0, 0.5])
def test_one_key_dominates_whole_units(G, Hq, H, D, n, share, mean):
    """So many sequences that a unit's keys are (nearly) all in one block's part of it."""
    check(dominated(160 if H == 1 else 170, G, Hq, H, D, n, share, mean, seed=n + G), TENSOR_CORES, [0, 77])


@pytest.mark.parametrize("path", [CUDA_CORES, TENSOR_CORES])
@pytest.mark.parametrize("G,Hq,H", LAYOUTS)
def test_one_key_dominates_split_units(path, G, Hq, H):
    check(dominated(1, G, Hq, H, 128, 8192, 0.9, 0.5, seed=G), path, [0])


@pytest.mark.parametrize("G,Hq,H", LAYOUTS)
@pytest.mark.parametrize("share", [0.99, 0.999])
def test_one_key_has_nearly_all_the_weight(G, Hq, H, share):
    check(dominated(160, G, Hq, H, 128, 8192, share, 0.5, seed=G + 1), TENSOR_CORES, [0, 159])


@pytest.mark.parametrize("path", [CUDA_CORES, TENSOR_CORES])
@pytest.mark.parametrize("G,Hq,H", LAYOUTS)
@pytest.mark.parametrize("apart", [8, 16, 20, 24])
def test_value_scales_far_apart(path, G, Hq, H, apart):
    """Every second page has a value scale 2^apart times the others', and values of 0 in half of
    the dims, which the other pages alone fill. What enters the product of a key is its weight
    times its page's value scale, so its error is at most 1.25 * 2^-9 of itself or 2^-28 of the
    row's largest: |do| <= 1.25 * 2^-9 sum_t p_t |v_t| + 2^-28 * max_t (p_t sv_t) * sum_t |v8_t| +
    2^-9 |o|, v8 the e4m3 values. All scores are 0."""
    r = np.random.default_rng(apart)
    n, P, D = 1500, 32, 128
    pages = -(-n // P)
    codes = ref.encode(r.standard_normal((pages, H, 2, P, D)) * 60 + 30)
    scale = np.ones((pages, H, 2), np.float32)
    scale[1::2, :, 1] = 2.0 ** -apart
    codes[::2, :, 1, :, D // 2:] = 0
    q = torch.zeros(2, G, Hq, D, dtype=torch.bfloat16)
    from paper_2609_04010_gb300 import binding as b
    o, _ = b.verify_attention_fp8(q.cuda(), torch.from_numpy(codes).cuda().view(torch.float8_e4m3fn),
                                  torch.from_numpy(scale).cuda(), i32(np.broadcast_to(np.arange(pages), (2, pages))),
                                  i32([n, n]), path=path)
    for s in range(2):
        ro, _, mass, _, _ = attention(q[s].double().numpy(), codes, scale, n)
        seen = n - G + 1 + np.arange(G)[:, None, None]
        v8 = np.abs(ref.decode(codes[:, :, 1])).transpose(1, 0, 2, 3).reshape(H, -1, D)[:, :n].sum(1)
        tol = 1.25 * 2.0 ** -9 * mass + 2.0 ** -28 / seen * np.repeat(v8, Hq // H, 0)[None] + 2.0 ** -9 * np.abs(ro)
        err = np.abs(o[s].float().cpu().numpy() - ro)
        assert (err / tol).max() <= 1, (err / tol).max()
