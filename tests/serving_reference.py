"""Plain 64-bit implementations of rotary positions, attention of chunks, forks and page copies."""

import math

import numpy as np
import torch


def rope(x, positions, freq, interleaved, factor=1.0):
    """x [rows][heads][D] (any float type), positions [rows], freq radians [rot / 2]: float64."""
    y = x.double().clone()
    h = freq.numel()
    a = positions.double()[:, None, None] * freq.double()
    c, s = factor * torch.cos(a), factor * torch.sin(a)
    i = torch.arange(h, device=x.device)
    first, second = (2 * i, 2 * i + 1) if interleaved else (i, i + h)
    x1, x2 = x[..., first].double(), x[..., second].double()
    y[..., first], y[..., second] = x1 * c - x2 * s, x2 * c + x1 * s
    y[positions < 0] = x[positions < 0].double()
    return y


def keys(cache, pages, head, kind, n):
    """The first n keys (kind 0) or values (1) behind these pages, float64."""
    first, second = cache
    if first.dtype == torch.float8_e4m3fn:
        scale = second[pages, head, kind].double()
        if kind:
            scale = scale.clamp(2.0 ** -32, 2.0 ** 32)
        x = first[pages, head, kind].double() * scale[:, None, None]
    else:
        x = cache[kind][pages, head].double()
    return x.reshape(-1, x.shape[-1])[:n]


def chunk_attention(q, cache, table, starts, lens, scale=0.0, causal=True, window=0):
    """out, lse, and per output what bounds its error: sum of weight * |value| ("spread") and, per
    row, the largest scale * sum |q_d k_d| ("reach"). Host lists starts and lens. All float64."""
    R, Hq, D = q.shape
    eight = cache[0].dtype == torch.float8_e4m3fn
    H, P = cache[0].shape[1], cache[0].shape[3 if eight else 2]
    scale = scale or 1 / math.sqrt(D)
    f = dict(dtype=torch.float64, device=q.device)
    out, spread = torch.zeros(R, Hq, D, **f), torch.zeros(R, Hq, D, **f)
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
        lowest = int(max(0, n - (r1 - r0) - window + 1)) if window else 0
        pages = table[b, :-(-n // P)].long().clone()
        pages[:lowest // P] = 0  # no row looks at them
        for h in range(Hq):
            k, v = (keys(cache, pages, h // (Hq // H), i, n) for i in (0, 1))
            seen_v = torch.where(see.any(0)[:, None], v, 0.0)
            x = q[r0:r1, h].double() @ k.T * scale
            x = torch.where(see, x, -math.inf)
            w = torch.softmax(x, -1)
            out[r0:r1, h] = _product(w, seen_v, see)
            spread[r0:r1, h] = _product(w, seen_v.abs(), see)
            lse[r0:r1, h] = torch.logsumexp(x, -1)
            mag = (q[r0:r1, h].double().abs() @ k.abs().T * scale).masked_fill(~see, 0)
            reach[r0:r1, h] = mag.nan_to_num(0, 0, 0).amax(-1)
    return out, lse, spread, reach


def _product(w, v, see):
    if bool(torch.isfinite(v).all()):
        return w @ v
    # a hidden key's value, whatever it is, adds nothing
    return torch.stack([torch.where(see[r][:, None], w[r][:, None] * v, 0.0).sum(0) for r in range(len(w))])


# One rounding of a bf16 output or weight is off by at most 2^-8 of it. A score is an fp32 sum of D
# products: off by at most D * 2^-24 of the sum of their magnitudes (reach), in natural units; 2^x and
# the sums of weights add less than 2^-18. So a weight is off by 2 (D 2^-24 reach) + 2^-18, relative
# (once in the numerator, once through the sum), plus 2^-8 where it is rounded to bf16; an output by
# that much of sum w |v| plus its own rounding.
def tolerance(out, spread, reach, dim, rounded_weights):
    rel = 2 * dim * 2.0 ** -24 * reach + 2.0 ** -18 + (2.0 ** -8 if rounded_weights else 0.0)
    return 2.0 ** -8 * out.abs() + rel[..., None] * spread + 1e-30, dim * 2.0 ** -24 * reach + 2.0 ** -18


def check_chunk(got, want, dim, rounded_weights):
    (o, l), (out, lse, spread, reach) = got, want
    t_out, t_lse = tolerance(out, spread, reach, dim, rounded_weights)
    same_nan = torch.isnan(o) == torch.isnan(out)
    assert bool(same_nan.all()), "NaN in other places"
    bad = ((o.double() - out).abs() > t_out * (1 + 2.0 ** -7)) & ~torch.isnan(out) & (o.double() != out)
    worst = ((o.double() - out).abs() / t_out).nan_to_num(0).max()
    assert not bool(bad.any()), f"out: {int(bad.sum())} of {bad.numel()} off, worst {float(worst):.2f} of the tolerance"
    if l is not None:
        fin = torch.isfinite(lse)
        assert torch.equal(torch.isfinite(l), fin)
        assert torch.equal(l[~fin].double().nan_to_num(7.0), lse[~fin].nan_to_num(7.0))
        err = ((l.double() - lse).abs() - 2.0 ** -22 * lse.abs() - t_lse)[fin]
        assert err.numel() == 0 or float(err.max()) <= 0, f"lse off by {float(err.max()):.2e} more than allowed"


def fork(parent, kv_len, table, shares, free, count, page, reserved):
    """Everything that spec_fork_sequences writes, in plain loops. numpy int arrays."""
    B, MP = table.shape
    N = len(shares)

    def len_ok(b):
        return 0 <= kv_len[b] and kv_len[b] + reserved <= MP * page

    def held(n):
        return -(-(n + reserved) // page)
    src, flags = [], np.zeros(B, np.int32)
    for b in range(B):
        ok = -1 <= parent[b] < B and len_ok(b) and (parent[b] < 0 or len_ok(parent[b]))
        src.append(int(parent[b]) if ok else b)
        flags[b] = 0 if ok else 1
    keeper = {}
    for b in range(B):
        if src[b] >= 0 and src[b] not in keeper:
            keeper[src[b]] = src[b] if src[src[b]] == src[b] else b
    new_len, new_table = np.array(kv_len), np.array(table)
    new_shares, new_free = np.array(shares), np.array(free)
    copies = np.full((B, 2), -1, np.int32)
    total = taken = 0
    for b in range(B):
        q = src[b]
        if q == b:
            continue
        new_table[b] = -1
        new_len[b] = 0
        if q < 0:
            continue
        n = int(kv_len[q])
        if keeper[q] == b:
            new_len[b] = n
            new_table[b, :held(n)] = table[q, :held(n)]
            continue
        whole = n // page
        need = held(n) - whole
        start = total
        total += need
        if need and total > count:
            flags[b] = 2
            continue
        new_len[b] = n
        if need:
            taken = max(taken, total)
        for i in range(whole):
            new_table[b, i] = table[q, i]
            if 0 <= table[q, i] < N:
                new_shares[table[q, i]] += 1
        for i in range(need):
            new_table[b, whole + i] = free[count - 1 - start - i]
        if n % page:
            copies[b] = table[q, whole], new_table[b, whole]
    gone = [(b, i) for b in range(B) if len_ok(b) and b not in keeper for i in range(held(kv_len[b]))]
    last = {}
    for b, i in gone:
        if 0 <= table[b, i] < N:
            new_shares[table[b, i]] -= 1
            last[table[b, i]] = (b, i)
    top = count - taken
    for b, i in gone:
        pg = table[b, i]
        if 0 <= pg < N and last[pg] == (b, i) and new_shares[pg] < 0:
            new_free[top] = pg
            top += 1
    new_shares = np.maximum(new_shares, 0)
    return dict(new_kv_len=new_len, new_table=new_table, new_shares=new_shares, new_free=new_free,
                new_count=np.array([top]), copies=copies, flags=flags)
