"""Query rows far larger or smaller than the others of their KV group: a row's precision is that
of its own largest element, whatever the other rows hold. Bounds as in
test_gpu_attention_fp8_weights.py, with each row's own largest |q|."""

import numpy as np
import pytest
import torch

import fp8_reference as ref
from test_gpu_attention_fp8 import CUDA_CORES, TENSOR_CORES, i32
from test_gpu_attention_fp8_weights import LAYOUTS, attention

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("path", [CUDA_CORES, TENSOR_CORES])
@pytest.mark.parametrize("G,Hq,H", LAYOUTS)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("factor", [2.0 ** 12, 2.0 ** 24, 2.0 ** -24])
def test_rows_of_other_magnitudes(path, G, Hq, H, D, factor):
    from paper_2609_04010_gb300 import binding as b
    r = np.random.default_rng(G)
    n, P = 700, 32
    pages = -(-n // P)
    codes = ref.encode(r.standard_normal((pages, H, 2, P, D)) * 64)
    scale = np.full((pages, H, 2), 2.0 ** -6, np.float32)
    x = r.standard_normal((2, G, Hq, D))
    x[:, ::3, ::2] *= factor
    q = torch.from_numpy(x).bfloat16()
    o, l = b.verify_attention_fp8(q.cuda(), torch.from_numpy(codes).cuda().view(torch.float8_e4m3fn),
                                  torch.from_numpy(scale).cuda(), i32(np.broadcast_to(np.arange(pages), (2, pages))),
                                  i32([n, n - 100]), path=path)
    for s, keys in enumerate((n, n - 100)):
        y = q[s].double().numpy()
        ro, rl, mass, vsum, kmax = attention(y, codes, scale, keys)
        ds = D ** -0.5 * kmax * (2.0 ** -18 + 128 * 2.0 ** -24) * np.abs(y).max(2)
        # rows whose scores are thousands of times one are decided by one key or by a tie
        plain = ds < 2.0 ** -6
        tol = (1.25 * 2.0 ** -9 + 2 * ds[..., None]) * mass + 2.0 ** -28 * vsum + 2.0 ** -9 * np.abs(ro)
        err = np.abs(o[s].float().cpu().numpy() - ro) / tol
        lerr = np.abs(l[s].cpu().numpy() - rl) / (ds + 2.0 ** -20 * (1 + np.abs(rl)))
        assert plain.any() and err[plain].max() <= 1 and lerr[plain].max() <= 1, (err[plain].max(), lerr[plain].max())


@pytest.mark.parametrize("path", [CUDA_CORES, TENSOR_CORES])
@pytest.mark.parametrize("G,Hq,H", LAYOUTS)
@pytest.mark.parametrize("power", range(16, 46, 3))
def test_scores_far_past_one(path, G, Hq, H, power):
    """Scores of 2^power, whose steps in fp32 are larger than the softmax's whole range: a row whose
    largest score is clear of the others by four times its error and 64 steps is the value of that
    key, and no finite input gives a NaN or an infinity."""
    from paper_2609_04010_gb300 import binding as b
    r = np.random.default_rng(power)
    n, P, D = 600, 16, 128
    pages = -(-n // P)
    codes = ref.encode(r.standard_normal((pages, H, 2, P, D)) * 64)
    scale = np.full((pages, H, 2), 2.0 ** -6, np.float32)
    q = torch.from_numpy(r.standard_normal((1, G, Hq, D)) * 2.0 ** power).bfloat16()
    o, l = b.verify_attention_fp8(q.cuda(), torch.from_numpy(codes).cuda().view(torch.float8_e4m3fn),
                                  torch.from_numpy(scale).cuda(), i32(np.arange(pages)[None]), i32([n]), path=path)
    o, l = o[0].float().cpu().numpy(), l[0].cpu().numpy()
    assert np.isfinite(o).all() and np.isfinite(l).all()
    y = q[0].double().numpy()
    x = (ref.decode(codes) * 2.0 ** -6).transpose(1, 2, 0, 3, 4).reshape(H, 2, -1, D)[:, :, :n]
    clear = 0
    for h in range(Hq):
        k, v = x[h * H // Hq]
        for j in range(G):
            s = k[:n - G + 1 + j] @ y[j, h] * D ** -0.5
            order = np.argsort(s)[::-1]
            ds = D ** -0.5 * np.abs(k).sum(1).max() * (2.0 ** -18 + 128 * 2.0 ** -24) * np.abs(y[j, h]).max()
            if s[order[0]] - s[order[1]] > 4 * ds + 64 * 2.0 ** -23 * abs(s[order[0]]):
                clear += 1
                assert np.all(np.abs(o[j, h] - v[order[0]]) <= 2.0 ** -7 * np.abs(v[order[0]]))
                assert abs(l[j, h] - s[order[0]]) <= ds + 2.0 ** -20 * abs(s[order[0]])
    assert clear > 0
