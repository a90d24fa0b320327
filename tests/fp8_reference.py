"""Plain 64-bit (and whole-number) references of the 8-bit KV cache operators and of the
logit constraints, with loops, on the host. They share no code with the CUDA path."""

import numpy as np


def _decode_table():
    t = np.zeros(256)
    for c in range(256):
        e, m = c >> 3 & 15, c & 7
        x = m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        if c & 0x7f == 0x7f:
            x = np.nan
        t[c] = -x if c & 0x80 else x
    return t


E4M3 = _decode_table()
_POSITIVE = E4M3[:0x7f]  # 0 .. 448, ascending


def decode(codes):
    return E4M3[np.asarray(codes, np.uint8)]


def encode(x):
    """The nearest e4m3 code (ties to the even code), saturated at +-448, NaN to NaN."""
    x = np.asarray(x, np.float64)
    a = np.minimum(np.abs(x), 448.0)
    hi = np.clip(np.searchsorted(_POSITIVE, a), 0, len(_POSITIVE) - 1)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - _POSITIVE[lo], _POSITIVE[hi] - a
    code = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi).astype(np.uint8)
    code = np.where(np.isnan(x), 0x7f, code)
    return (code | np.where(np.signbit(x), 0x80, 0)).astype(np.uint8)


def scale_of(amax):
    """The smallest power of two in [2^-32, 2^32] with amax <= 448 * scale."""
    k = -32
    while k < 32 and amax > 448.0 * 2.0 ** k:
        k += 1
    return 2.0 ** k


def append(k, v, slots, codes, scale, page_size):
    """codes [pages][H][2][P][D] and scale [pages][H][2] after the call (copies)."""
    codes, scale = codes.copy(), scale.astype(np.float64).copy()
    pages, H = scale.shape[:2]
    rows_of = {}
    for r, s in enumerate(slots):
        if 0 <= s < pages * page_size:
            rows_of.setdefault(int(s) // page_size, []).append(r)
    for page, rows in rows_of.items():
        places = [int(slots[r]) % page_size for r in rows]
        for h in range(H):
            for kind, x in ((0, k), (1, v)):
                new = x[rows, h].astype(np.float64)
                finite = np.abs(new[np.isfinite(new)])
                need = scale_of(finite.max() if finite.size else 0.0)
                if 0 not in places:
                    old = min(max(float(scale[page, h, kind]), 2.0 ** -32), 2.0 ** 32)
                    if old >= need:
                        need = old
                    else:
                        held = decode(codes[page, h, kind]) * (old / need)
                        codes[page, h, kind] = encode(held)
                scale[page, h, kind] = need
                codes[page, h, kind, places] = encode(np.clip(new, -1e300, 1e300) / need)
    return codes, scale


def map_slots(num_new, kv_len, table, page_size, num_pages, free, count, max_rows, reserved=0):
    table, kv_len = table.copy(), kv_len.astype(np.int64)
    B, MP = table.shape
    count = min(max(int(count), 0), len(free))
    new_len, flags = kv_len.copy(), np.zeros(B, np.int32)
    row_start = [0]
    slots, positions, row_seq = [], [], []
    asked = taken = 0
    for b in range(B):
        n, held = int(num_new[b]), int(kv_len[b])
        if n < 0 or held < 0 or held + n > MP * page_size:
            flags[b] = 1
        else:
            first = -(-(held + reserved) // page_size)
            need = max(0, -(-(held + n) // page_size) - first)
            if need and asked + need > count:
                flags[b] = 2
            else:
                for i in range(need):
                    table[b, first + i] = free[count - 1 - asked - i]
                if need:
                    taken = asked + need
                new_len[b] = held + n
            asked += need
        for i in range(max(n, 0)):
            pos = held + i
            page = table[b, pos // page_size] if flags[b] == 0 else -1
            ok = flags[b] == 0 and 0 <= page < num_pages
            slots.append(page * page_size + pos % page_size if ok else -1)
            positions.append(pos)
            row_seq.append(b)
        row_start.append(row_start[-1] + max(n, 0))

    def rows(x):
        return np.array((x + [-1] * max_rows)[:max_rows], np.int32)
    return dict(new_len=new_len.astype(np.int32), flags=flags, table=table, count=count - taken,
                row_start=np.array(row_start, np.int32), slots=rows(slots),
                positions=rows(positions), row_seq=rows(row_seq))


def attention(q, codes, scale, table, kv_len, gamma, page_size, softmax_scale=0.0, tree=None):
    """out, lse, and the bounds' parts: mass = sum_t p_t |v_t| and kmax = max_t sum_d |k_td|."""
    B, G, Hq, D = q.shape
    H = codes.shape[1]
    group = Hq // H
    sc = softmax_scale or D ** -0.5
    out, lse = np.zeros(q.shape), np.full(q.shape[:3], -np.inf)
    mass, kmax = np.zeros(q.shape), np.zeros(q.shape[:3])
    for b in range(B):
        n = int(kv_len[b])
        ctx = n - gamma
        pages = table[b, :-(-n // page_size)]
        for h in range(H):
            k = (decode(codes[pages, h, 0]) * scale[pages, h, 0].astype(np.float64)[:, None, None]).reshape(-1, D)[:n]
            v = (decode(codes[pages, h, 1]) * np.clip(scale[pages, h, 1].astype(np.float64), 2.0 ** -32, 2.0 ** 32)[:, None, None]).reshape(-1, D)[:n]
            for j in range(G):
                if tree is None:
                    see = np.arange(n) <= ctx + j
                else:
                    bits = [bool(int(tree[b, j]) >> i & 1) for i in range(gamma)]
                    see = np.concatenate([np.ones(ctx, bool), np.array(bits, bool)])
                if not see.any():
                    continue
                kk, vv = k[see], v[see]
                for g in range(group):
                    x = kk @ q[b, j, h * group + g] * sc
                    top = x.max()
                    w = np.exp(x - top)
                    i = (b, j, h * group + g)
                    lse[i] = top + np.log(w.sum())
                    out[i] = w @ vv / w.sum()
                    mass[i] = w @ np.abs(vv) / w.sum()
                    kmax[i] = np.abs(kk).sum(1).max()
    return out, lse, mass, kmax


def adjust(x, block=None, history=None, history_len=None, prompt_len=None, repetition=None,
           frequency=None, presence=None, bias_tokens=None, bias_values=None, allowed=None,
           block_shift=0):
    x = x.astype(np.float64).copy()
    B, G, V = x.shape
    for b in range(B):
        r = 1.0 if repetition is None else float(repetition[b])
        f = 0.0 if frequency is None else float(frequency[b])
        p = 0.0 if presence is None else float(presence[b])
        held = [] if history is None else list(history[b, :min(max(int(history_len[b]), 0), history.shape[1])])
        cut = 0 if prompt_len is None else min(max(int(prompt_len[b]), 0), len(held))
        for j in range(G):
            spoken = list(held[cut:])
            if block is not None:
                spoken += list(block[b, :j + 1 - block_shift])
            count = {}
            for t in spoken:
                count[int(t)] = count.get(int(t), 0) + 1
            for t in set(int(t) for t in held[:cut]) | set(count):
                if 0 <= t < V:
                    x[b, j, t] = x[b, j, t] / r if x[b, j, t] > 0 else x[b, j, t] * r
            for t, c in count.items():
                if 0 <= t < V:
                    x[b, j, t] -= f * c + p
            if bias_tokens is not None:
                done = set()
                for t, w in zip(bias_tokens[b], bias_values[b]):
                    if 0 <= t < V and int(t) not in done:
                        x[b, j, t] += float(w)
                    done.add(int(t))
            if allowed is not None:
                bits = np.unpackbits(allowed[b, j].view(np.uint8), bitorder="little")[:V]
                x[b, j, bits == 0] = -np.inf
    return x
