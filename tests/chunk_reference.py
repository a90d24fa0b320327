"""Attention of chunks in 64 bits where values may be NaN, and the tolerance that the 8-bit cache's
tensor-core path promises."""

import math

import torch

import serving_reference as ref


def attend(c, softmax_scale=0.0, causal=True, window=0):
    """What serving_reference.chunk_attention gives for a case, for any number of NaN values, and per output
    the sum of |stored value| of the seen keys times the row's largest weight * value scale ("steps").
    A NaN value makes the outputs NaN of the rows that see it, in its column, however small its weight."""
    q, cache, table, starts, lens, eight = c["q"], c["cache"], c["table"], c["starts"], c["lens"], c["fp8"]
    R, Hq, D = q.shape
    H, P = cache[0].shape[1], cache[0].shape[3 if eight else 2]
    softmax_scale = softmax_scale or 1 / math.sqrt(D)
    f = dict(dtype=torch.float64, device=q.device)
    out, spread, steps = (torch.zeros(R, Hq, D, **f) for _ in range(3))
    lse, reach = torch.full((R, Hq), -math.inf, **f), torch.zeros(R, Hq, **f)
    for b in range(len(lens)):
        r0, r1, n = starts[b], starts[b + 1], lens[b]
        if r1 == r0:
            continue
        at = torch.arange(n - (r1 - r0), n, device=q.device)[:, None]
        key = torch.arange(n, device=q.device)[None]
        see = (key <= at) if causal else torch.ones(r1 - r0, n, dtype=torch.bool, device=q.device)
        if window:
            see = see & (key > at - window)
        pages = table[b, :-(-n // P)].long().clone()
        if window:
            pages[:max(0, n - (r1 - r0) - window + 1) // P] = 0  # no row looks at them
        for h in range(Hq):
            g = h // (Hq // H)
            k, v = (ref.keys(cache, pages, g, i, n) for i in (0, 1))
            nan, v0 = torch.isnan(v).double(), v.nan_to_num(0.0)
            x = q[r0:r1, h].double() @ k.T * softmax_scale
            x = torch.where(see, x, -math.inf)
            w = torch.softmax(x, -1)
            out[r0:r1, h] = torch.where(see.double() @ nan > 0, math.nan, w @ v0)
            spread[r0:r1, h] = w @ v0.abs()
            lse[r0:r1, h] = torch.logsumexp(x, -1)
            mag = (q[r0:r1, h].double().abs() @ k.abs().T * softmax_scale).masked_fill(~see, 0)
            reach[r0:r1, h] = mag.nan_to_num(0, 0, 0).amax(-1)
            if eight:
                scale = cache[1][pages, g, 1].double().clamp(2.0 ** -32, 2.0 ** 32).repeat_interleave(P)[:n]
                steps[r0:r1, h] = (w * scale).nan_to_num(0).amax(-1, keepdim=True) * (see.double() @ (v0 / scale[:, None]).abs())
    return out, lse, spread, reach, steps


# Over the 8-bit cache the tensor cores' weights are rounded to fp16 together with the value scale: off by
# 2^-11 of themselves, or by 2^-33 of the row's largest (steps). Queries and values enter exactly. Scores are
# fp32 sums of D products, off by D 2^-24 of their magnitudes (reach); their scales, the softmax's and the
# exponent's sum are five more roundings of 2^-24 of the exponent, whose part that is not a score (the value
# scale's logarithm and the reference) is at most 2^6 in these tests: 2^-17, the sums of weights included.
# A weight enters twice, with its value and through the sum. The output is rounded once: 2^-8 of itself.
def check_8_bit(got, want, dim):
    (o, l), (out, lse, spread, reach, steps) = got, want
    score = (dim + 5) * 2.0 ** -24 * reach + 2.0 ** -17
    tol = 2.0 ** -8 * out.abs() + (2 * score + 2.0 ** -11)[..., None] * spread + 2.0 ** -33 * steps + 1e-30
    assert torch.equal(torch.isnan(o), torch.isnan(out)), "NaN in other places"
    fin = torch.isfinite(out)
    worst = ((o.double() - out).abs() / tol)[fin]
    assert worst.numel() == 0 or float(worst.max()) <= 1 + 2.0 ** -7, f"out: {float(worst.max()):.2f} of the tolerance"
    check_lse(l, lse, score)


def check_lse(l, lse, score):
    if l is None:
        return
    fin = torch.isfinite(lse)
    assert torch.equal(torch.isfinite(l), fin)
    assert torch.equal(l[~fin].double().nan_to_num(7.0), lse[~fin].nan_to_num(7.0))
    err = ((l.double() - lse).abs() - 2.0 ** -22 * lse.abs() - score)[fin]
    assert err.numel() == 0 or float(err.max()) <= 0, f"lse off by {float(err.max()):.2e} more than allowed"


def check(got, want, c, cuda_cores=False):
    """Either cache, either path."""
    if c["fp8"] and not cuda_cores:
        check_8_bit(got, want, c["D"])
    else:
        ref.check_chunk(got, want[:4], c["D"], not cuda_cores)
