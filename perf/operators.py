"""Cases of the 8-bit KV cache operators and of the logit constraints.

Four operators of a verify step whose KV cache is held in 8 bits:

* ``slots``: pages and cache slots for the new tokens of a ragged batch, from its lengths;
* ``append``: new keys and values written into the 8-bit cache (e4m3, one power-of-two
  scale per page, KV head, and K or V);
* ``attn``: block-causal or tree attention of the block queries over that cache;
* ``logits``: penalties for repeated tokens, biases and grammar masks on logits rows.

``run`` computes a case in plain torch operations, or, with ``own`` set, through the
package's binding. ``exact`` computes it in 64 bits from the definitions.
"""

import math

import numpy as np
import torch

own = False

E4M3_MAX = 448.0
MIN_EXP, MAX_EXP = -32, 32  # the range of a scale's exponent


# ----------------------------------------------------------------------------------
# Cases
# ----------------------------------------------------------------------------------
def listed():
    return [
        # one short request: a block of 4 over 512 tokens, one query head per KV head
        dict(name="attn_tiny", op="attn", batch=1, gamma=4, hq=8, hkv=8, dim=64, page=16,
             lo=512, hi=512, tree=False),
        # single-token decoding of a mid-size batch at ragged contexts (the sweep's range)
        dict(name="attn_decode32", op="attn", batch=32, gamma=1, hq=32, hkv=8, dim=128, page=16,
             lo=256, hi=16384, tree=False),
        # a candidate tree of 31 nodes per request, odd context
        dict(name="attn_tree8", op="attn", batch=8, gamma=31, hq=32, hkv=8, dim=128, page=16,
             lo=4001, hi=4096, tree=True),
        # high-batch serving: blocks of 16, ragged contexts, 16-token pages
        dict(name="attn_serve64", op="attn", batch=64, gamma=16, hq=32, hkv=8, dim=128, page=16,
             lo=512, hi=4096, tree=False),
        # long contexts, 256 query rows per KV head, 64-token pages
        dict(name="attn_long4", op="attn", batch=4, gamma=32, hq=64, hkv=8, dim=128, page=64,
             lo=32768, hi=32768, tree=False),
        # the block keys of a serving batch, written at ragged places of started pages
        dict(name="append_serve64", op="append", batch=64, new=16, hkv=8, dim=128, page=16,
             lo=33, hi=96),
        # a chunk of prompts: 8 requests of 4,093 tokens into new 64-token pages
        dict(name="append_prefill", op="append", batch=8, new=4093, hkv=8, dim=128, page=64,
             lo=0, hi=0),
        # a verify step's blocks of 16 for 64 requests
        dict(name="slots_serve64", op="slots", batch=64, new_lo=16, new_hi=16, page=16, lo=512,
             hi=4096, spare=1.0),
        # a mixed batch of decoding requests and prompts, some of which do not get pages
        dict(name="slots_mixed512", op="slots", batch=512, new_lo=1, new_hi=4096, page=16, lo=0,
             hi=4096, spare=0.9),
        # one request, fp32 rows of a small vocabulary
        dict(name="logits_tiny", op="logits", batch=1, gamma=4, vocab=32000, f32=True, hist=600,
             bias=8, mask=True),
        # blocks of 8 for 8 requests with penalties and biases, no grammar
        dict(name="logits_llama8b", op="logits", batch=8, gamma=8, vocab=128256, f32=False,
             hist=4096, bias=64, mask=False),
        # a serving batch, half of it under a grammar
        dict(name="logits_serve64", op="logits", batch=64, gamma=16, vocab=128256, f32=False,
             hist=2000, bias=16, mask=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attn", "attn", "append", "slots", "logits"])
    if op == "attn":
        hq, hkv = rng.choice([(8, 8), (32, 8), (64, 8), (12, 3), (16, 2), (8, 1)])
        gamma = _log_int(rng, 1, 32)
        hi = _log_int(rng, 64, 32768)
        # at most the rows x keys of the largest listed case, and a cache of its size
        most = min(4 * 64 * 32 * 32768 // (hq * gamma * (hi + gamma)),
                   4 * 8 * 32768 // (hkv * (hi + gamma)))
        batch = _log_int(rng, 1, max(1, min(128, most)))
        return dict(op="attn", batch=batch, gamma=gamma, hq=hq, hkv=hkv,
                    dim=rng.choice([64, 128]), page=rng.choice([16, 32, 64]),
                    lo=rng.randint(0, hi), hi=hi, tree=rng.random() < 0.3)
    if op == "append":
        new = _log_int(rng, 1, 4093)
        batch = _log_int(rng, 1, max(1, min(128, 8 * 4093 // new)))
        lo = rng.choice([0, rng.randint(1, 500)])
        return dict(op="append", batch=batch, new=new, hkv=rng.choice([1, 3, 8]),
                    dim=rng.choice([64, 128]), page=rng.choice([16, 32, 64]), lo=lo,
                    hi=lo + rng.randint(0, 300))
    if op == "slots":
        batch = _log_int(rng, 1, 512)
        new_lo = rng.choice([0, 1, 7]) if batch > 1 else 1
        return dict(op="slots", batch=batch, new_lo=new_lo,
                    new_hi=new_lo + _log_int(rng, 1, 4000), page=rng.choice([16, 32, 64]), lo=0,
                    hi=_log_int(rng, 1, 4096), spare=rng.choice([0.5, 0.9, 1.0]))
    gamma = _log_int(rng, 1, 16)
    vocab = _log_int(rng, 1000, 151936)
    batch = _log_int(rng, 1, max(1, min(64, 64 * 16 * 128256 // (2 * gamma * vocab))))
    return dict(op="logits", batch=batch, gamma=gamma, vocab=vocab, f32=rng.random() < 0.4,
                hist=_log_int(rng, 1, 16384), bias=rng.choice([0, 1, 33, 300]),
                mask=rng.random() < 0.6)


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


def _pages(lens, page, extra, seed):
    """A page table for sequences of these lengths over a shuffled pool with `extra` pages more."""
    need = -(-lens // page)
    total = int(need.sum())
    pool = np.random.default_rng([seed, 2]).permutation(total + extra)
    table = np.full((len(lens), max(1, int(need.max()))), -1, np.int64)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = pool[at:at + n]
        at += n
    return table, pool[total:], total + extra


def _filled_cache(pages, hkv, page, dim, seed):
    """A cache of normal keys and values whose magnitude differs by page and head."""
    g = _gen(seed, 3)
    values = torch.empty(pages, hkv, 2, page, dim, dtype=torch.uint8, device="cuda")
    scale = torch.empty(pages, hkv, 2, dtype=torch.float32, device="cuda")
    for p0 in range(0, pages, 4096):
        n = min(4096, pages - p0)
        x = torch.randn(n, hkv, 2, page, dim, generator=g, device="cuda")
        x *= torch.exp2(torch.rand(n, hkv, 2, 1, 1, generator=g, device="cuda") * 2 - 1)
        _, e = torch.frexp(x.abs().amax((3, 4)) / E4M3_MAX)
        s = torch.exp2(e.float())
        scale[p0:p0 + n] = s
        values[p0:p0 + n] = (x / s[..., None, None]).to(torch.float8_e4m3fn).view(torch.uint8)
    return values.view(torch.float8_e4m3fn), scale


def prepare(case, seed):
    s = dict(case)
    if case["op"] == "attn":
        B, G, D, P = case["batch"], case["gamma"], case["dim"], case["page"]
        lens = _spread(case["lo"], case["hi"], B, seed) + G
        table, _, pages = _pages(lens, P, 0, seed)
        s["cache"], s["scale"] = _filled_cache(pages, case["hkv"], P, D, seed)
        s["table"], s["kv_len"] = _i32(table), _i32(lens)
        s["q"] = torch.randn(B, G, case["hq"], D, generator=_gen(seed, 4), device="cuda").bfloat16()
        s["tree_mask"] = None
        if case["tree"]:
            r = np.random.default_rng([seed, 5])
            bits = np.zeros((B, G), np.uint64)
            bits[:, 0] = 1
            for c in range(1, G):
                parent = r.integers(max(0, c - 6), c, B)
                bits[:, c] = bits[np.arange(B), parent] | np.uint64(1 << c)
            s["tree_mask"] = torch.from_numpy(bits.view(np.int64)).cuda()
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(B, G, case["hq"], device="cuda")
    elif case["op"] == "append":
        B, N, H, D, P = (case[k] for k in ("batch", "new", "hkv", "dim", "page"))
        lens = _spread(case["lo"], case["hi"], B, seed)
        table, _, pages = _pages(lens + N, P, 0, seed)
        s["cache"], s["scale"] = _filled_cache(pages, H, P, D, seed)
        at = lens[:, None] + np.arange(N)
        s["slots"] = _i32((np.take_along_axis(table, at // P, 1) * P + at % P).reshape(-1))
        # keys and values as the projection leaves them: column ranges of one row
        g = _gen(seed, 6)
        rows = torch.randn(B * N, 3 * H, D, generator=g, device="cuda")
        rows *= torch.exp2(torch.rand(B * N, 3 * H, 1, generator=g, device="cuda") * 2)
        rows = rows.bfloat16()
        s["k"], s["v"] = rows[:, H:2 * H], rows[:, 2 * H:]
    elif case["op"] == "slots":
        B, P = case["batch"], case["page"]
        lens = _spread(case["lo"], case["hi"], B, seed)
        new = np.random.default_rng([seed, 7]).permutation(
            _spread(case["new_lo"], case["new_hi"], B, seed))
        table, rest, held = _pages(lens, P, 1000, seed)
        need = -(-(lens + new) // P) - -(-lens // P)
        total, first = int(need.sum()), int(need[np.argmax(need > 0)])
        free = np.concatenate([held + np.arange(total), rest])
        free = np.random.default_rng([seed, 8]).permutation(free)[:max(1, total)]
        wide = np.full((B, -(-(case["hi"] + case["new_hi"]) // P) + 1), -1, np.int64)
        wide[:, :table.shape[1]] = table[:, :wide.shape[1]]
        s["pages"] = held + total
        s["rows"] = max(1, int(new.sum()) + 3)
        s["kv_len"], s["num_new"], s["table"] = _i32(lens), _i32(new), _i32(wide)
        s["free"], s["count"] = _i32(free), _i32([max(first, int(total * case["spare"]))])
        i32 = dict(dtype=torch.int32, device="cuda")
        s["new_len"], s["new_count"] = torch.empty(B, **i32), torch.empty(1, **i32)
        s["row_start"], s["flags"] = torch.empty(B + 1, **i32), torch.empty(B, **i32)
        for k in ("slots", "positions", "row_seq"):
            s[k] = torch.empty(s["rows"], **i32)
    else:
        B, G, V, L = case["batch"], case["gamma"], case["vocab"], case["hist"]
        g = _gen(seed, 9)
        x = torch.randn(B, G, V, generator=g, device="cuda") * 3
        s["x"] = x if case["f32"] else x.bfloat16()
        del x
        r = np.random.default_rng([seed, 10])
        # text repeats itself: tokens of a skewed distribution
        def tokens(*shape):
            return np.minimum(V * r.random(shape) ** 4, V - 1).astype(np.int64)
        length = _spread(max(1, L // 2), L, B, seed)
        s["history"], s["block"] = _i32(tokens(B, L)), _i32(tokens(B, G))
        s["history_len"], s["prompt_len"] = _i32(length), _i32(length * r.random(B))

        def f32(a):
            return torch.from_numpy(a.astype(np.float32)).cuda()
        s["repetition"] = f32(1 + 0.3 * r.random(B))
        s["frequency"], s["presence"] = f32(r.random(B)), f32(r.random(B))
        s["bias_tokens"] = s["bias_values"] = s["mask"] = None
        if case["bias"]:
            n = min(case["bias"], V)
            t = np.stack([r.choice(V, n, replace=False) for _ in range(B)])
            s["bias_tokens"], s["bias_values"] = _i32(t), f32(r.normal(0, 4, (B, n)))
        if case["mask"]:
            # a grammar allows few tokens between values and most of them inside a text;
            # every second request has none
            W = -(-V // 32)
            bits = torch.empty(B, G, W, dtype=torch.int32, device="cuda")
            keep = torch.from_numpy(np.where(r.random((B, G, 1)) < 0.5, 0.002, 0.95)).cuda()
            keep[::2] = 2
            weight = 2 ** torch.arange(32, device="cuda", dtype=torch.int64)
            for b in range(B):
                u = torch.rand(G, W * 32, generator=g, device="cuda") < keep[b]
                w = (u.view(G, W, 32).long() * weight).sum(-1)
                bits[b] = torch.where(w >= 2 ** 31, w - 2 ** 32, w).int()
            s["mask"] = bits
        s["out"] = torch.empty_like(s["x"])
    if own:
        _plan(s)
    return s


def _plan(s):
    """The argument structures and the workspace that a program keeps over its steps."""
    from paper_2609_04010_gb300 import binding as b
    if s["op"] == "attn":
        s["args"] = b.attn_fp8_args(s["q"], s["cache"], s["scale"], s["table"], s["kv_len"],
                                    s["out"], s["lse"], tree_mask=s["tree_mask"])
        s["ws"] = b.new_workspace(b.attn_fp8_workspace_size(s["args"]))
    elif s["op"] == "append":
        s["args"] = b.append_fp8_args(s["k"], s["v"], s["slots"], s["cache"], s["scale"])
    elif s["op"] == "slots":
        s["args"] = b.slot_args(s["num_new"], s["kv_len"], s["new_len"], s["table"], s["page"],
                                s["pages"], s["free"], s["count"], s["new_count"], s["row_start"],
                                s["slots"], s["positions"], s["row_seq"], s["flags"])
        s["ws"] = b.new_workspace(b.slot_workspace_size(s["args"]))
    else:
        s["args"] = b.adjust_args(s["x"], s["out"], s["block"], s["history"], s["history_len"],
                                  s["prompt_len"], s["repetition"], s["frequency"], s["presence"],
                                  s["bias_tokens"], s["bias_values"], s["mask"])


# ----------------------------------------------------------------------------------
# One pass
# ----------------------------------------------------------------------------------
def run(s):
    if own:
        from paper_2609_04010_gb300 import binding as b
        if s["op"] == "attn":
            b.verify_attention_fp8_args(s["args"], s["ws"])
            return dict(out=s["out"], lse=s["lse"])
        if s["op"] == "append":
            b.append_kv_fp8_args(s["args"])
            return dict(cache=s["cache"], scale=s["scale"])
        if s["op"] == "slots":
            b.map_slots_args(s["args"], s["ws"])
            return _slots_out(s)
        b.adjust_logits_args(s["args"])
        return dict(out=s["out"])
    return dict(attn=_plain_attn, append=_plain_append, slots=_plain_slots,
                logits=_plain_logits)[s["op"]](s)


def _slots_out(s):
    return {k: s[k] for k in ("new_len", "new_count", "row_start", "flags", "slots", "positions",
                              "row_seq", "table")}


def _plain_attn(s):
    B, G, Hq, D = s["q"].shape
    H, P = s["hkv"], s["page"]
    table = s["table"].long().clamp_min(0)
    kv = s["cache"][table].float() * s["scale"][table][..., None, None]
    L = table.shape[1] * P                                  # [B][pages][H][2][P][D]
    kv = kv.permute(3, 0, 2, 1, 4, 5).reshape(2, B, H, L, D)
    q = s["q"].float().view(B, G, H, Hq // H, D).permute(0, 2, 1, 3, 4).reshape(B, H, -1, D)
    x = torch.matmul(q, kv[0].transpose(2, 3)) / math.sqrt(D)
    rel = torch.arange(L, device="cuda") - (s["kv_len"].long()[:, None] - G)
    j = torch.arange(G, device="cuda")
    if s["tree_mask"] is None:
        see = rel[:, None, :] <= j[:, None]
    else:
        bit = (s["tree_mask"][:, :, None] >> rel[:, None, :].clamp(0, 63)) & 1
        see = (rel[:, None, :] < 0) | ((rel[:, None, :] < G) & (bit == 1))
    see = see[:, None, :, None, :].expand(B, H, G, Hq // H, L).reshape(B, H, -1, L)
    x = torch.where(see, x, -math.inf)
    top = x.amax(-1, keepdim=True)
    w = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
    total = w.sum(-1, keepdim=True)
    out = torch.matmul(w, kv[1]) / torch.where(total == 0, 1.0, total)
    lse = top + torch.log(total)

    def rows(t):
        return t.view(B, H, G, Hq // H, -1).permute(0, 2, 1, 3, 4).reshape(B, G, Hq, -1)
    return dict(out=rows(out).bfloat16(), lse=rows(lse)[..., 0])


def _plain_append(s):
    cache, scale, P = s["cache"].view(torch.uint8), s["scale"], s["page"]
    slots = s["slots"].long()
    page, place = slots // P, slots % P
    new = torch.stack([s["k"], s["v"]], 2).float()          # [rows][H][2][D]
    top = torch.zeros_like(scale).scatter_reduce_(
        0, page[:, None, None].expand(-1, *scale.shape[1:]), new.abs().amax(3), "amax")
    m, e = torch.frexp(top)
    e = torch.where(top == 0, MIN_EXP, e - 9 + (m > 0.875).int()).clamp(MIN_EXP, MAX_EXP)
    touched = torch.zeros(len(scale), dtype=torch.bool, device="cuda")
    touched[page] = True
    starts = torch.zeros_like(touched)
    starts[page[place == 0]] = True
    goes_on = (touched & ~starts)[:, None, None]
    now = torch.where(touched[:, None, None], torch.exp2(e.float()), scale)
    now = torch.where(goes_on, torch.maximum(now, scale), now)
    at = torch.nonzero(touched & ~starts)[:, 0]
    held = s["cache"][at].float() * (scale[at] / now[at])[..., None, None]
    cache[at] = held.to(torch.float8_e4m3fn).view(torch.uint8)
    x = (new / now[page][..., None]).clamp(-E4M3_MAX, E4M3_MAX)
    cache[page, :, :, place] = x.to(torch.float8_e4m3fn).view(torch.uint8)
    scale.copy_(now)
    return dict(cache=s["cache"], scale=scale)


def _plain_slots(s):
    P, MP, rows = s["page"], s["table"].shape[1], s["rows"]
    have, n = s["kv_len"].long(), s["num_new"].long()
    count = s["count"].long()
    fits = (have >= 0) & (n >= 0) & (have + n <= MP * P)
    first = (have + P - 1) // P
    need = torch.where(fits, (have + n + P - 1) // P - first, 0)
    upto = need.cumsum(0)
    gets = fits & ((need == 0) | (upto <= count))
    flags = torch.where(fits, torch.where(gets, 0, 2), 1)
    n = n.clamp_min(0)
    start = torch.cat([n.new_zeros(1), n.cumsum(0)])
    r = torch.arange(rows, device="cuda")
    b = torch.searchsorted(start, r, right=True) - 1
    used = b < len(have)
    b = b.clamp_max(len(have) - 1)
    pos = have[b] + r - start[b]
    good = used & gets[b]
    index = torch.where(good, pos // P, 0)
    order = count - 1 - (upto[b] - need[b]) - (index - first[b])
    fresh = good & (index >= first[b])
    table = s["table"].long()
    page = torch.where(fresh, s["free"].long()[order.clamp(0, len(s["free"]) - 1)],
                       table[b, index])
    opens = fresh & (pos % P == 0)
    table.index_put_((torch.where(opens, b, 0), torch.where(opens, index, 0)),
                     torch.where(opens, page, table[0, 0]))
    # the first entry of the table again, where a fresh page belongs there
    head = opens & (b == 0) & (index == 0)
    table[0, 0] = torch.where(head.any(), (page * head).sum(), s["table"][0, 0].long())
    s["table"].copy_(table)
    taken = torch.where(gets & (need > 0), upto, 0).amax()
    return dict(new_len=torch.where(gets, have + n, have).int(), new_count=(count - taken).int(),
                row_start=start.int(), flags=flags.int(),
                slots=torch.where(good, page * P + pos % P, -1).int(),
                positions=torch.where(used, pos, -1).int(),
                row_seq=torch.where(used, b, -1).int(), table=s["table"])


def _plain_logits(s):
    x = s["x"].float()
    B, G, V = x.shape
    at = torch.arange(s["history"].shape[1], device="cuda")
    live = at < s["history_len"][:, None]
    prompt = at < s["prompt_len"][:, None]
    zero = torch.zeros(B, V, device="cuda")
    tokens = s["history"].long()
    in_prompt = zero.scatter_add(1, tokens, (live & prompt).float()) > 0
    spoken = zero.scatter_add(1, tokens, (live & ~prompt).float())
    block = torch.zeros(B, G, V, device="cuda").scatter_add_(
        2, s["block"].long()[..., None], torch.ones(B, G, 1, device="cuda"))
    times = spoken[:, None] + block.cumsum(1)
    seen = in_prompt[:, None] | (times > 0)
    r = s["repetition"][:, None, None]
    x = torch.where(seen, torch.where(x > 0, x / r, x * r), x)
    x = x - s["frequency"][:, None, None] * times
    x = x - s["presence"][:, None, None] * (times > 0)
    if s["bias_tokens"] is not None:
        x = x + zero.scatter_add(1, s["bias_tokens"].long(), s["bias_values"])[:, None]
    if s["mask"] is not None:
        bit = (s["mask"][..., None] >> torch.arange(32, device="cuda", dtype=torch.int32)) & 1
        x = torch.where(bit.view(B, G, -1)[..., :V] == 1, x, -math.inf)
    return dict(out=x.to(s["x"].dtype))


# ----------------------------------------------------------------------------------
# What a pass cannot do without
# ----------------------------------------------------------------------------------
def work(case):
    if case["op"] == "attn":
        B, G, Hq, H, D, P = (case[k] for k in ("batch", "gamma", "hq", "hkv", "dim", "page"))
        ctx = _spread(case["lo"], case["hi"], B, 0)
        keys, pages = int((ctx + G).sum()), int((-(-(ctx + G) // P)).sum())
        per_key = H * 2 * D
        io = B * G * Hq * (2 * D + 2 * D + 4)
        pairs = int((ctx * G).sum()) + B * G * (G + 1) // 2
        return dict(bytes=keys * per_key + pages * (H * 8 + 4) + io + 4 * B,
                    flops=4 * D * Hq * pairs)
    if case["op"] == "append":
        rows = case["batch"] * case["new"]
        values = rows * case["hkv"] * case["dim"] * 2
        pages = case["batch"] * (case["new"] // case["page"] + 1)
        return dict(bytes=3 * values + 4 * rows + 8 * case["hkv"] * pages, flops=2 * values)
    if case["op"] == "slots":
        B = case["batch"]
        rows = int(_spread(case["new_lo"], case["new_hi"], B, 0).sum())
        return dict(bytes=12 * rows + 8 * rows // case["page"] + 24 * B, flops=0)
    n = case["batch"] * case["gamma"] * case["vocab"]
    return dict(bytes=2 * n * (4 if case["f32"] else 2) + (n // 8 if case["mask"] else 0)
                + 4 * case["batch"] * (case["hist"] + 2 * case["bias"]), flops=4 * n)


# ----------------------------------------------------------------------------------
# The definitions in 64 bits
# ----------------------------------------------------------------------------------
def exact(case, seed):
    global own
    was, own = own, False
    s = prepare(case, seed)
    own = was
    return dict(attn=_exact_attn, append=_exact_append, logits=_exact_logits,
                slots=lambda s: None)[case["op"]](s)


def _exact_attn(s):
    """Sequence by sequence and KV head by KV head."""
    B, G, Hq, D = s["q"].shape
    H, P = s["hkv"], s["page"]
    out = torch.zeros(B, G, Hq, D, dtype=torch.float64, device="cuda")
    lse = torch.zeros(B, G, Hq, dtype=torch.float64, device="cuda")
    lens, group = s["kv_len"].tolist(), Hq // H
    for b in range(B):
        n = lens[b]
        pages = s["table"][b, :-(-n // P)].long()
        see = torch.ones(G, n, dtype=torch.bool, device="cuda")
        for j in range(G):
            if s["tree_mask"] is None:
                see[j, n - G + j + 1:] = False
            else:
                bits = int(s["tree_mask"][b, j])
                see[j, n - G:] = torch.tensor([bits >> i & 1 for i in range(G)], device="cuda") == 1
        for h in range(H):
            k, v = ((s["cache"][pages, h, i].double() * s["scale"][pages, h, i].double()[:, None, None])
                    .reshape(-1, D)[:n] for i in (0, 1))
            q = s["q"][b, :, h * group:(h + 1) * group].double()
            x = torch.einsum("jgd,td->gjt", q, k) / D ** 0.5
            x = x.masked_fill(~see, -math.inf)
            lse[b, :, h * group:(h + 1) * group] = torch.logsumexp(x, -1).T
            p = torch.softmax(x, -1).nan_to_num(0.0)
            out[b, :, h * group:(h + 1) * group] = torch.einsum("gjt,td->jgd", p, v)
    return dict(out=out, lse=lse)


def _to_e4m3(x):
    """The nearest e4m3 values (ties to even), by their spacing: 2^(e - 3), at least 2^-9."""
    _, e = torch.frexp(x)
    step = torch.exp2((e - 4).clamp_min(-9).double())
    return (torch.round(x / step) * step).clamp(-E4M3_MAX, E4M3_MAX)


def _exact_append(s):
    """Page by page on the host's plan: which rows go where, and what the page held."""
    P, slots = s["page"], s["slots"].long().cpu().numpy()
    cache, scale = s["cache"].double(), s["scale"].double()
    new = torch.stack([s["k"].double(), s["v"].double()], 2)
    order = np.argsort(slots // P, kind="stable")
    pages, begin = np.unique(slots[order] // P, return_index=True)
    if len(pages) > 20000:
        return None
    for i, page in enumerate(pages):
        rows = order[begin[i]:begin[i + 1] if i + 1 < len(pages) else len(order)]
        place = torch.from_numpy(slots[rows] % P).cuda()
        x = new[torch.from_numpy(rows).cuda()]              # [n][H][2][D]
        top = x.abs().amax((0, 3))
        now = torch.full_like(top, 2.0 ** MIN_EXP)
        for k in range(MIN_EXP + 1, 16):                    # the inputs end far below 448 * 2^15
            now[top > E4M3_MAX * 2.0 ** (k - 1)] = 2.0 ** k
        if 0 not in slots[rows] % P:
            now = torch.maximum(now, scale[page])
            cache[page] = _to_e4m3(cache[page] * (scale[page] / now)[..., None, None])
        cache[page][:, :, place] = _to_e4m3(x / now[None, :, :, None]).permute(1, 2, 0, 3)
        scale[page] = now
    return dict(cache=cache, scale=scale)


def _exact_logits(s):
    """Request by request, with the counts of the tokens that each one holds."""
    B, G, V = s["x"].shape
    out = torch.empty(B, G, V, dtype=torch.float64, device="cuda")
    for b in range(B):
        held = s["history"][b, :s["history_len"][b]].long()
        prompt, spoken = held[:s["prompt_len"][b]], held[s["prompt_len"][b]:]
        was = torch.zeros(V, dtype=torch.bool, device="cuda")
        was[prompt] = True
        times = torch.bincount(spoken, minlength=V).double()
        bias = torch.zeros(V, dtype=torch.float64, device="cuda")
        if s["bias_tokens"] is not None:
            bias[s["bias_tokens"][b].long()] = s["bias_values"][b].double()
        r, f, p = (s[k][b].double() for k in ("repetition", "frequency", "presence"))
        for j in range(G):
            times[s["block"][b, j].long()] += 1
            x = s["x"][b, j].double()
            x = torch.where(was | (times > 0), torch.where(x > 0, x / r, x * r), x)
            x = x - f * times - p * (times > 0).double() + bias
            if s["mask"] is not None:
                word = s["mask"][b, j].long() & 0xFFFFFFFF
                t = torch.arange(V, device="cuda")
                x = x.masked_fill((word[t // 32] >> (t % 32)) & 1 == 0, -math.inf)
            out[b, j] = x
    return dict(out=out)
