"""Cases of the operators that serve prompts and forked sequences over the paged KV caches.

Four operators that run together when prompts of any length, single tokens and draft blocks
share a batch:

* ``rope``: rotary positions of queries and keys, and the write of keys and values into the
  paged bf16 cache;
* ``chunk``: attention of a ragged batch of new tokens (one token to whole prompts) over the
  paged cache, bf16 or 8-bit: causal, or with the chunk seen from both sides, with or without a
  sliding window;
* ``fork``: sequences that go on from others (parallel samples, beams), end or stay: their page
  tables, the holders of shared pages, the free list, and the pages to copy;
* ``copy``: those copies, in the caches of all layers.

``run`` computes a case in plain torch operations, or, with ``own`` set, through the
package's binding. ``exact`` computes it in 64 bits from the definitions.
"""

import math

import numpy as np
import torch

own = False

E4M3_MAX = 448.0


# ----------------------------------------------------------------------------------
# Cases
# ----------------------------------------------------------------------------------
def listed():
    return [
        # a verify step's blocks of 16 for 64 requests, whole heads, halves rotated
        dict(name="rope_serve64", op="rope", batch=64, new=16, hq=32, hkv=8, dim=128, page=16,
             rot=128, pairs=False, lo=512, hi=4096),
        # a chunk of prompts far into long contexts, half of each head in interleaved pairs
        dict(name="rope_prefill", op="rope", batch=8, new=4093, hq=32, hkv=8, dim=128, page=64,
             rot=64, pairs=True, lo=0, hi=1000000),
        # one request's next token over a short context, one query head per KV head
        dict(name="chunk_tiny", op="chunk", batch=1, ones=1, new=1, hq=8, hkv=8, dim=64, page=16,
             lo=512, hi=512, causal=True, window=0, fp8=False),
        # a serving batch: 60 requests decode, four more bring a chunk of their prompts
        dict(name="chunk_mixed64", op="chunk", batch=64, ones=60, new=1021, hq=32, hkv=8, dim=128,
             page=16, lo=256, hi=16384, causal=True, window=0, fp8=False),
        # a drafter's pass: blocks of 16 whose tokens see each other in both directions
        dict(name="chunk_draft64", op="chunk", batch=64, ones=0, new=16, hq=32, hkv=8, dim=128,
             page=16, lo=512, hi=4096, causal=False, window=0, fp8=False),
        # whole prompts from the first token
        dict(name="chunk_prompts4", op="chunk", batch=4, ones=0, new=4093, hq=32, hkv=8, dim=128,
             page=16, lo=0, hi=0, causal=True, window=0, fp8=False),
        # chunks of two prompts over the 8-bit cache
        dict(name="chunk_fp8", op="chunk", batch=2, ones=0, new=2048, hq=32, hkv=8, dim=128,
             page=16, lo=4001, hi=12288, causal=True, window=0, fp8=True),
        # the last chunk of a long document, 64-token pages
        dict(name="chunk_long", op="chunk", batch=1, ones=0, new=4096, hq=32, hkv=8, dim=128,
             page=64, lo=28672, hi=28672, causal=True, window=0, fp8=False),
        # eight requests of four beams, each beam from a random one of its request
        dict(name="fork_beams32", op="fork", batch=32, group=4, beams=True, page=16, lo=500,
             hi=2000, reserved=0),
        # a large batch: one in eight ends, one in eight starts as another sample of a request
        dict(name="fork_serve512", op="fork", batch=512, group=4, beams=False, page=16, lo=0,
             hi=8192, reserved=16),
        # eight pages of one layer
        dict(name="copy_small", op="copy", pairs=8, layers=1, pages=64, hkv=8, dim=128, page=16,
             fp8=False),
        # 64 forked requests, 32 layers
        dict(name="copy_layers32", op="copy", pairs=64, layers=32, pages=160, hkv=8, dim=128,
             page=16, fp8=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["chunk", "chunk", "chunk", "rope", "fork", "copy"])
    if op == "rope":
        dim = rng.choice([64, 128])
        hq, hkv = rng.choice([(8, 8), (32, 8), (12, 3), (16, 2), (10, 2)])
        new = _log_int(rng, 1, 4093)
        return dict(op="rope", batch=_log_int(rng, 1, max(1, min(128, 8 * 4093 // new))), new=new,
                    hq=hq, hkv=hkv, dim=dim, page=rng.choice([16, 32, 64]),
                    rot=rng.choice([16, 32, 48, 64, dim]), pairs=rng.random() < 0.5,
                    lo=rng.randint(0, 500), hi=500 + _log_int(rng, 1, 1000000))
    if op == "chunk":
        hq, hkv = rng.choice([(8, 8), (32, 8), (64, 8), (12, 3), (16, 2), (8, 1), (10, 2)])
        dim = rng.choice([64, 128])
        new, hi = _log_int(rng, 1, 4096), _log_int(rng, 64, 32768)
        # at most the work and the cache of the largest listed case
        most = min(32 * 4096 * 30720 // (hq * new * (hi + new)), 8 * 32768 // (hkv * (hi + new)))
        batch = _log_int(rng, 1, max(1, min(96, most)))
        return dict(op="chunk", batch=batch, ones=rng.choice([0, batch // 2, batch - 1]), new=new,
                    hq=hq, hkv=hkv, dim=dim, page=rng.choice([16, 32, 64]), lo=rng.randint(0, hi),
                    hi=hi, causal=rng.random() < 0.7,
                    window=rng.choice([0, 0, _log_int(rng, 1, 8192)]), fp8=rng.random() < 0.4)
    if op == "fork":
        group = rng.choice([1, 2, 4, 8])
        return dict(op="fork", batch=group * _log_int(rng, 1, 512 // group), group=group,
                    beams=rng.random() < 0.5, page=rng.choice([16, 32, 64]), lo=0,
                    hi=_log_int(rng, 1, 8192), reserved=rng.choice([0, 0, 1, 16, 40]))
    pages = _log_int(rng, 16, 512)
    layers = _log_int(rng, 1, 32)
    return dict(op="copy", pairs=_log_int(rng, 1, min(64, pages // 2)), layers=layers, pages=pages,
                hkv=rng.choice([1, 3, 8]), dim=rng.choice([64, 128]), page=16, fp8=rng.random() < 0.5)


# ----------------------------------------------------------------------------------
# Inputs
# ----------------------------------------------------------------------------------
def _spread(lo, hi, n, seed):
    """n whole numbers spread evenly over lo..hi, in an order of the seed's."""
    at = np.array([(lo + hi) // 2]) if n == 1 else lo + (hi - lo) * np.arange(n) // (n - 1)
    return np.random.default_rng([seed, 1]).permutation(at).astype(np.int64)


def _gen(seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1000 + stream)
    return g


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a).astype(np.int32)).cuda()


def _pages(lens, page, seed):
    """A page table for sequences of these lengths over a shuffled pool, and the pool's size."""
    need = -(-lens // page)
    total = int(need.sum())
    pool = np.random.default_rng([seed, 2]).permutation(total)
    table = np.full((len(lens), max(1, int(need.max()))), -1, np.int64)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = pool[at:at + n]
        at += n
    return table, max(1, total)


def _chunk_sizes(case, seed):
    """New tokens and contexts of the sequences: `ones` of them bring one token."""
    B = case["batch"]
    new = np.full(B, case["new"], np.int64)
    new[:case["ones"]] = 1
    new = np.random.default_rng([seed, 3]).permutation(new)
    return new, _spread(case["lo"], case["hi"], B, seed)


def _caches(case, pages, seed):
    """A filled cache: bf16 K and V, or the 8-bit one with its scales."""
    shape = (pages, case["hkv"], case["page"], case["dim"])
    g = _gen(seed, 4)
    if not case["fp8"]:
        return tuple(torch.randn(shape, generator=g, device="cuda").bfloat16() for _ in range(2))
    pages, H, P, D = shape
    values = torch.empty(pages, H, 2, P, D, dtype=torch.uint8, device="cuda")
    scale = torch.empty(pages, H, 2, dtype=torch.float32, device="cuda")
    for p0 in range(0, pages, 4096):
        n = min(4096, pages - p0)
        x = torch.randn(n, H, 2, P, D, generator=g, device="cuda")
        x *= torch.exp2(torch.rand(n, H, 2, 1, 1, generator=g, device="cuda") * 2 - 1)
        _, e = torch.frexp(x.abs().amax((3, 4)) / E4M3_MAX)
        scale[p0:p0 + n] = torch.exp2(e.float())
        values[p0:p0 + n] = (x / scale[p0:p0 + n, ..., None, None]).to(torch.float8_e4m3fn).view(torch.uint8)
    return values.view(torch.float8_e4m3fn), scale


def _held(lens, reserved, page):
    return -(-(lens + reserved) // page)


def prepare(case, seed):
    s = dict(case)
    r = np.random.default_rng([seed, 5])
    if case["op"] == "rope":
        B, N, H, D, P = (case[k] for k in ("batch", "new", "hkv", "dim", "page"))
        start = _spread(case["lo"], case["hi"], B, seed)
        # a cache that holds the new tokens alone: positions run on from contexts held elsewhere
        table, pages = _pages(start % P + N, P, seed)
        at = (start % P)[:, None] + np.arange(N)
        s["slots"] = _i32((np.take_along_axis(table, at // P, 1) * P + at % P).reshape(-1))
        s["positions"] = _i32((start[:, None] + np.arange(N)).reshape(-1))
        # q, k and v as the projection leaves them: column ranges of one row
        rows = torch.randn(B * N, case["hq"] + 2 * H, D, generator=_gen(seed, 6), device="cuda").bfloat16()
        s["q"], s["k"], s["v"] = rows.split([case["hq"], H, H], 1)
        s["cache"] = tuple(torch.zeros(pages, H, P, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        i = torch.arange(case["rot"] // 2, dtype=torch.float64)
        s["freq"] = (500000.0 ** (-2 * i / case["rot"])).cuda()
        s["q_out"] = torch.empty(B * N, case["hq"], D, dtype=torch.bfloat16, device="cuda")
    elif case["op"] == "chunk":
        new, ctx = _chunk_sizes(case, seed)
        lens = ctx + new
        table, pages = _pages(lens, case["page"], seed)
        s["cache"] = _caches(case, pages, seed)
        s["table"], s["kv_len"] = _i32(table), _i32(lens)
        s["starts"] = [0] + np.cumsum(new).tolist()
        s["lens"] = lens.tolist()
        s["row_start"] = _i32(s["starts"])
        rows = s["starts"][-1]
        # queries are a column range of the projection's rows
        wide = torch.randn(rows, case["hq"] + 2 * case["hkv"], case["dim"], generator=_gen(seed, 7),
                           device="cuda").bfloat16()
        s["q"] = wide[:, :case["hq"]]
        s["out"] = torch.empty(rows, case["hq"], case["dim"], dtype=torch.bfloat16, device="cuda")
        s["lse"] = torch.empty(rows, case["hq"], device="cuda")
    elif case["op"] == "fork":
        B, G, P = case["batch"], case["group"], case["page"]
        lens = np.repeat(_spread(case["lo"], case["hi"], B // G, seed), G)
        # a pool for the sequences with nothing shared, and room for forks
        pages = int(_held(lens, case["reserved"], P).sum()) + B * (2 + case["reserved"] // P)
        lens = np.clip(lens + r.integers(-min(100, case["hi"] // 2), 1, B), 0, None)
        held = _held(lens, case["reserved"], P)
        table = np.full((B, int(_held(case["hi"], case["reserved"], P)) + 3), -1, np.int64)
        # sequences of a group hold the whole pages of a common prefix together
        common = np.array([lens[b // G * G:b // G * G + G].min() // 2 // P for b in range(B)])
        pool = r.permutation(pages)
        shares = np.zeros(pages, np.int64)
        at = 0
        for b in range(B):
            lead = b // G * G
            skip = 0 if b == lead else common[b]
            table[b, :skip] = table[lead, :skip]
            shares[table[b, :skip]] += 1
            n = held[b] - skip
            table[b, skip:held[b]] = pool[at:at + n]
            at += n
        free = np.concatenate([pool[at:], np.full(at, -1, np.int64)])
        lead = np.arange(B) // G * G
        if case["beams"]:
            parent = lead + r.integers(0, G, B)
        else:
            parent = np.arange(B)
            kind = r.random(B)
            parent[kind < 0.125] = -1
            forked = (kind >= 0.125) & (kind < 0.25)
            parent[forked] = (lead + r.integers(0, G, B))[forked]
        s["parent"], s["kv_len"], s["table"] = _i32(parent), _i32(lens), _i32(table)
        s["shares"], s["free"], s["count"] = _i32(shares), _i32(free), _i32([pages - at])
        for k in ("kv_len", "table", "shares", "free", "count"):
            s["new_" + k] = torch.empty_like(s[k])
        s["pairs"] = torch.empty(B, 2, dtype=torch.int32, device="cuda")
        s["flags"] = torch.empty(B, dtype=torch.int32, device="cuda")
    else:
        g = _gen(seed, 8)
        shape = (case["pages"], case["hkv"], case["page"], case["dim"])
        s["buffers"] = []
        for _ in range(case["layers"]):
            if case["fp8"]:
                x = torch.randint(0, 127, (shape[0], shape[1], 2) + shape[2:], generator=g, device="cuda",
                                  dtype=torch.uint8)
                s["buffers"] += [x.view(torch.float8_e4m3fn),
                                 torch.rand(case["pages"], case["hkv"], 2, generator=g, device="cuda")]
            else:
                s["buffers"] += [torch.randn(shape, generator=g, device="cuda").bfloat16() for _ in range(2)]
        at = r.permutation(case["pages"])
        # sources repeat (several samples of one request); destinations do not
        half = case["pages"] // 2
        s["pair_list"] = _i32(np.stack([r.choice(at[:half], case["pairs"]), at[half:half + case["pairs"]]], 1))
    if own:
        _plan(s)
    return s


def _plan(s):
    """The argument structures and the workspace that a program keeps over its steps."""
    from paper_2609_04010_gb300 import binding as b
    if s["op"] == "rope":
        s["args"] = b.rope_args(s["q"], s["k"], s["v"], s["positions"], b.rope_turns(s["freq"]),
                                q_out=s["q_out"], slots=s["slots"], k_cache=s["cache"][0],
                                v_cache=s["cache"][1], interleaved=s["pairs"])
    elif s["op"] == "chunk":
        s["args"] = b.chunk_attn_args(s["q"], s["cache"], s["table"], s["row_start"], s["kv_len"],
                                      s["out"], s["lse"], causal=s["causal"], window=s["window"])
        s["ws"] = b.new_workspace(b.chunk_attn_workspace_size(s["args"]))
    elif s["op"] == "fork":
        s["args"] = b.fork_args(s["parent"], s["kv_len"], s["new_kv_len"], s["table"], s["new_table"],
                                s["shares"], s["new_shares"], s["free"], s["new_free"], s["count"],
                                s["new_count"], s["page"], s["pairs"], s["flags"], s["reserved"])
        s["ws"] = b.new_workspace(b.fork_workspace_size(s["args"]))
    else:
        s["args"] = b.copy_args(s["pair_list"], s["buffers"])


# ----------------------------------------------------------------------------------
# One pass
# ----------------------------------------------------------------------------------
def run(s):
    if own:
        from paper_2609_04010_gb300 import binding as b
        if s["op"] == "rope":
            b.rope_kv_args(s["args"])
            return dict(q=s["q_out"], k=s["cache"][0], v=s["cache"][1])
        if s["op"] == "chunk":
            b.chunk_attention_args(s["args"], s["ws"])
            return dict(out=s["out"], lse=s["lse"])
        if s["op"] == "fork":
            b.fork_sequences_args(s["args"], s["ws"])
            return {k: s[k] for k in ("new_kv_len", "new_table", "new_shares", "new_free", "new_count",
                                      "pairs", "flags")}
        b.copy_pages_args(s["args"])
        return list(s["buffers"])
    return dict(rope=_plain_rope, chunk=_plain_chunk, fork=_plain_fork, copy=_plain_copy)[s["op"]](s)


def _plain_rope(s):
    P, h = s["page"], s["rot"] // 2
    angle = s["positions"].double()[:, None] * s["freq"]
    cos, sin = (f(angle).float()[:, None] for f in (torch.cos, torch.sin))

    def turned(x):
        x = x.float()
        a, b = (x[..., 0:2 * h:2], x[..., 1:2 * h:2]) if s["pairs"] else (x[..., :h], x[..., h:2 * h])
        a, b = a * cos - b * sin, b * cos + a * sin
        front = torch.stack([a, b], -1).flatten(-2) if s["pairs"] else torch.cat([a, b], -1)
        return torch.cat([front, x[..., 2 * h:]], -1).bfloat16()
    slots = s["slots"].long()
    page, place = slots // P, slots % P
    s["cache"][0][page, :, place] = turned(s["k"])
    s["cache"][1][page, :, place] = s["v"]
    return dict(q=turned(s["q"]), k=s["cache"][0], v=s["cache"][1])


def _keys(s, b, kind, heads, dtype):
    """Keys (kind 0) or values (1) of sequence b and some KV heads: [heads][len][dim]."""
    n, P = s["lens"][b], s["page"]
    pages = s["table"][b, :-(-n // P)].long()
    if s["fp8"]:
        values, scale = s["cache"]
        x = values[pages, heads, kind].to(dtype) * scale[pages, heads, kind].to(dtype)[..., None, None]
    else:
        x = s["cache"][kind][pages, heads].to(dtype)
    return x.transpose(0, 1).flatten(1, 2)[:, :n]


def _visible(s, b):
    """[new][len]: which keys each new token of sequence b sees."""
    n, r = s["lens"][b], s["starts"][b + 1] - s["starts"][b]
    at = torch.arange(n - r, n, device="cuda")[:, None]
    key = torch.arange(n, device="cuda")[None]
    see = key <= at if s["causal"] else torch.ones(r, n, dtype=torch.bool, device="cuda")
    return see & (key > at - s["window"]) if s["window"] else see


def _plain_chunk(s):
    R, Hq, D = s["q"].shape
    H, group = s["hkv"], Hq // s["hkv"]
    out = torch.empty(R, Hq, D, dtype=torch.bfloat16, device="cuda")
    lse = torch.empty(R, Hq, device="cuda")
    for b in range(s["batch"]):
        r0, r1 = s["starts"][b], s["starts"][b + 1]
        see = _visible(s, b)
        step = min(H, max(1, 2 ** 28 // (group * see.numel())))    # KV heads at a time
        for h in range(0, H, step):
            heads = slice(h * group, min(h + step, H) * group)
            k, v = (_keys(s, b, i, slice(h, h + step), torch.float32)[:, None] for i in (0, 1))
            q = s["q"][r0:r1, heads].float().transpose(0, 1).unflatten(0, (-1, group))
            x = torch.matmul(q, k.transpose(2, 3)) / math.sqrt(D)
            x = torch.where(see, x, -math.inf)
            top = x.amax(-1, keepdim=True)
            w = torch.exp(x - top)
            total = w.sum(-1, keepdim=True)
            o = torch.matmul(w, v) / total
            out[r0:r1, heads] = o.flatten(0, 1).transpose(0, 1).bfloat16()
            lse[r0:r1, heads] = (top + torch.log(total)).flatten(0, 1)[..., 0].T
    return dict(out=out, lse=lse)


def _plain_fork(s):
    P, res, N = s["page"], s["reserved"], s["shares"].numel()
    parent, lens, table, count = s["parent"].long(), s["kv_len"].long(), s["table"].long(), s["count"].long()
    B, MP = table.shape
    at, col = torch.arange(B, device="cuda"), torch.arange(MP, device="cuda")
    held = (lens + res + P - 1) // P
    # of the sequences with one parent, the parent itself or else the first goes on with its pages
    big = B + 1
    keeper = torch.full((B + 1,), big, device="cuda").scatter_reduce_(
        0, torch.where(parent < 0, B, parent), torch.where(parent == at, -1, at), "amin")[:B]
    keeper = torch.where(keeper == -1, at, keeper)
    src = parent.clamp_min(0)
    alive = parent >= 0
    keeps = alive & (keeper[src] == at)
    child = alive & ~keeps
    full = lens[src] // P
    need = torch.where(child, held[src] - full, 0)
    upto = need.cumsum(0)
    served = ~child | (need == 0) | (upto <= count)
    fresh = (s["free"].long()[(count - 1 - (upto - need)[:, None] - (col - full[:, None])).clamp(0, N - 1)])
    rows = table[src]
    rows = torch.where(child[:, None] & (col >= full[:, None]), fresh, rows)
    rows = torch.where((col < held[src][:, None]) & (alive & served)[:, None], rows, -1)
    rows = torch.where((parent == at)[:, None], table, rows)
    taken = torch.where(child & served & (need > 0), upto, 0).amax()
    copies = child & served & (lens[src] % P > 0)
    pairs = torch.stack([table[at * 0 + src, full.clamp_max(MP - 1)], rows[at, full.clamp_max(MP - 1)]], 1)
    # holders of pages: children more, sequences that nobody goes on from fewer
    more = (child & served)[:, None] & (col < full[:, None])
    gone = (keeper == big)[:, None] & (col < held[:, None])
    shares = torch.cat([s["shares"].long(), torch.zeros(1, dtype=torch.int64, device="cuda")])
    shares.scatter_add_(0, torch.where(more, table[src], N).flatten(), more.long().flatten())
    shares.scatter_add_(0, torch.where(gone, table, N).flatten(), -gone.long().flatten())
    # freed pages, in the order of the last place that held them
    place = torch.arange(B * MP, device="cuda").view(B, MP)
    owner = torch.full((N + 1,), -1, device="cuda").scatter_reduce_(
        0, torch.where(gone, table, N).flatten(), place.flatten(), "amax")
    freed = gone & (shares[table.clamp_min(0)] < 0) & (owner[table.clamp_min(0)] == place)
    rank = freed.flatten().cumsum(0)
    to = torch.where(freed.flatten(), count - taken + rank - 1, N)
    free = torch.cat([s["free"].long(), torch.zeros(1, dtype=torch.int64, device="cuda")])
    free.scatter_(0, to, torch.where(freed, table, 0).flatten())
    return dict(new_kv_len=torch.where(alive & served, lens[src], 0).int(), new_table=rows.int(),
                new_shares=shares[:N].clamp_min(0).int(), new_free=free[:N].int(),
                new_count=(count - taken + rank[-1:]).int(),
                pairs=torch.where(copies[:, None], pairs, -1).int(), flags=torch.where(served, 0, 2).int())


def _plain_copy(s):
    src, dst = s["pair_list"].long().unbind(1)
    for x in s["buffers"]:
        x = x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x
        x[dst] = x[src]
    return list(s["buffers"])


# ----------------------------------------------------------------------------------
# What a pass cannot do without
# ----------------------------------------------------------------------------------
def work(case):
    if case["op"] == "rope":
        rows = case["batch"] * case["new"]
        heads = case["hq"] + 2 * case["hkv"]
        return dict(bytes=rows * (4 * heads * case["dim"] + 8) + 4 * case["rot"],
                    flops=rows * 3 * (case["hq"] + case["hkv"]) * case["rot"])
    if case["op"] == "chunk":
        new, ctx = _chunk_sizes(case, 0)
        D, H, Hq, P = (case[k] for k in ("dim", "hkv", "hq", "page"))
        keys = pairs = 0
        for r, c in zip(new.tolist(), ctx.tolist()):
            at = np.arange(c, c + r, dtype=np.int64)
            low = np.maximum(0, at - case["window"] + 1) if case["window"] else 0 * at
            high = at if case["causal"] else 0 * at + c + r - 1
            pairs += int((high - low + 1).sum())
            keys += c + r - int(low[0])
        per_key = 2 * H * D * (1 if case["fp8"] else 2)
        scales = keys // P * H * 8 if case["fp8"] else 0
        rows = int(new.sum())
        return dict(bytes=keys * per_key + scales + keys // P * 4 + rows * Hq * (4 * D + 4),
                    flops=4 * D * Hq * pairs)
    if case["op"] == "fork":
        B = case["batch"]
        held = _held(_spread(case["lo"], case["hi"], B, 0), case["reserved"], case["page"])
        row = int(held.max()) + 3
        # tables, holders of pages and the free list, each once in and out
        return dict(bytes=8 * B * row + 16 * int(held.sum()) + 28 * B, flops=0)
    page = 2 * case["hkv"] * case["page"] * case["dim"] * (1 if case["fp8"] else 2)
    page += case["hkv"] * 8 if case["fp8"] else 0
    return dict(bytes=2 * case["pairs"] * case["layers"] * page, flops=0)


# ----------------------------------------------------------------------------------
# The definitions in 64 bits
# ----------------------------------------------------------------------------------
def exact(case, seed):
    global own
    was, own = own, False
    s = prepare(case, seed)
    own = was
    return dict(rope=_exact_rope, chunk=_exact_chunk, fork=lambda s: None, copy=lambda s: None)[case["op"]](s)


def _exact_rope(s):
    """Each pair as a complex number times e^(i angle)."""
    P, h = s["page"], s["rot"] // 2
    turn = torch.polar(torch.ones_like(s["freq"]), torch.zeros_like(s["freq"]))
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                       s["positions"].double()[:, None] * s["freq"]) * turn

    def turned(x):
        y = x.double().clone()
        if s["pairs"]:
            z = torch.view_as_complex(y[..., :2 * h].unflatten(-1, (h, 2)).contiguous())
            y[..., :2 * h] = torch.view_as_real(z * turn[:, None]).flatten(-2)
        else:
            z = torch.complex(y[..., :h].contiguous(), y[..., h:2 * h].contiguous()) * turn[:, None]
            y[..., :h], y[..., h:2 * h] = z.real, z.imag
        return y
    flat = s["slots"].long()
    k, v = (c.double().permute(0, 2, 1, 3).flatten(0, 1) for c in s["cache"])
    k[flat] = turned(s["k"])
    v[flat] = s["v"].double()
    k, v = (c.unflatten(0, (-1, P)).permute(0, 2, 1, 3) for c in (k, v))
    return dict(q=turned(s["q"]), k=k, v=v)


def _exact_chunk(s):
    """Sequence by sequence and query head by query head."""
    R, Hq, D = s["q"].shape
    out = torch.zeros(R, Hq, D, dtype=torch.float64, device="cuda")
    lse = torch.zeros(R, Hq, dtype=torch.float64, device="cuda")
    for b in range(s["batch"]):
        rows = slice(s["starts"][b], s["starts"][b + 1])
        hidden = ~_visible(s, b)
        for h in range(Hq):
            g = h // (Hq // s["hkv"])
            if h % (Hq // s["hkv"]) == 0:
                k, v = (_keys(s, b, i, slice(g, g + 1), torch.float64)[0] for i in (0, 1))
            x = torch.einsum("rd,kd->rk", s["q"][rows, h].double(), k) * D ** -0.5
            x = x.masked_fill_(hidden, -math.inf)
            lse[rows, h] = torch.logsumexp(x, 1)
            out[rows, h] = torch.einsum("rk,kd->rd", torch.softmax(x, 1), v)
    return dict(out=out, lse=lse)
