"""Cases by which the operators of a speculative step over the paged cache are measured.

A serving instance that drafts tokens ahead verifies a whole tree of them in one iteration: the drafted tokens' queries and
keys are normed for each head and rotated by their positions while their K and V are appended to the paged cache
(``write_rope``), every drafted token attends the request's context and its own ancestors (``run_tree``), and the K and V of
the accepted path move to the front of the tree's slots (``accept``).  ``read`` gives stretches of many sequences back as
bf16, whatever the cache holds, as an instance does that hands requests on or goes over an FP8 cache's context in bf16.

Where ``own`` is false ``run`` computes the same with elementary torch operations over a plain cache of
[pages * 16 slots, kv heads, head dim], in 32 bits.  Outputs of a cache's update are the tokens that it touched, read back.

The head shapes are those of the repository's configurations (32/8/128, 64/8/128, 8/8/64, 4/2/64), with 16-token pages,
N(0,1) data and contexts uniform on a range.
"""
import math

import numpy as np
import torch

own = False

PAGE = 16
EPS = 1e-6
THETA = 500000.0
FILL_TOKENS = 1 << 17  # tokens drawn and cached at a time when a cache is filled


def _case(name, kind, heads, kv_heads, dim, **kw):
    """``rows`` requests of ctx_lo .. ctx_hi cached tokens and new_lo .. new_hi new ones.  ``tree``: the new tokens are a
    drafted tree (positions by depth).  ``rot``: rotated dimensions of a head.  ``q_scale``: standard deviation of q."""
    c = {"kind": kind, "heads": heads, "kv_heads": kv_heads, "dim": dim, "fp8": False, "rows": 1, "ctx_lo": 0, "ctx_hi": 0,
         "new_lo": 1, "new_hi": 1, "tree": False, "norm": False, "rot": dim, "interleaved": False, "q_scale": 1.0, "len_seed": 1}
    c.update(kw)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # eight requests of one new token each: what every decode iteration does before attention; launches and latency
        _case("append_decode", "append", 32, 8, 128, rows=8, ctx_lo=256, ctx_hi=768, norm=True, len_seed=2),
        # fresh prompts out of one fused projection, positions counted from the start of each
        _case("append_prompts", "append", 32, 8, 128, rows=4, new_lo=1500, new_hi=2050, norm=True, len_seed=3),
        # drafted trees of 64 requests into an FP8 cache: normed, rotated by depth and quantised
        _case("append_trees_fp8", "append", 64, 8, 128, fp8=True, rows=64, ctx_lo=512, ctx_hi=4096, new_lo=16, new_hi=64, tree=True,
              norm=True, len_seed=4),
        # one request, a tree of eight drafted tokens on a short context: latency
        _case("tree_one", "tree", 32, 8, 128, rows=1, ctx_lo=700, ctx_hi=700, new_lo=8, new_hi=8, tree=True, len_seed=5),
        # an ordinary verification step: 32 requests of an 8B-class model, ragged trees, peaked scores
        _case("tree_32", "tree", 32, 8, 128, rows=32, ctx_lo=512, ctx_hi=4096, new_lo=11, new_hi=32, tree=True, q_scale=2.0, len_seed=6),
        # the same on the FP8 cache with more requests
        _case("tree_fp8", "tree", 32, 8, 128, fp8=True, rows=64, ctx_lo=512, ctx_hi=4096, new_lo=7, new_hi=32, tree=True, len_seed=7),
        # head dimension 64 without head grouping
        _case("tree_d64", "tree", 8, 8, 64, rows=24, ctx_lo=300, ctx_hi=5000, new_lo=20, new_hi=61, tree=True, len_seed=8),
        # the largest: 64 trees of up to 64 tokens on long contexts, 2 GB of K and V
        _case("tree_large", "tree", 32, 8, 128, rows=64, ctx_lo=4096, ctx_hi=12288, new_lo=48, new_hi=64, tree=True, len_seed=9),
        # accepted paths of 32 trees; latency
        _case("accept_32", "accept", 32, 8, 128, rows=32, ctx_lo=512, ctx_hi=4096, new_lo=11, new_hi=32, tree=True, len_seed=10),
        # accepted paths of a large batch in an FP8 cache
        _case("accept_fp8", "accept", 32, 8, 128, fp8=True, rows=256, ctx_lo=100, ctx_hi=1000, new_lo=16, new_hi=64, tree=True, len_seed=11),
        # the newest tokens of 16 sequences, read from the middle of their pages
        _case("read_recent", "read", 32, 8, 128, rows=16, ctx_lo=100, ctx_hi=2000, new_lo=33, new_hi=200, len_seed=12),
        # six requests on the FP8 cache handed on whole
        _case("read_fp8", "read", 32, 8, 128, fp8=True, rows=6, new_lo=1000, new_hi=9000, len_seed=13),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "append", "tree", "tree", "tree", "accept", "read"])
    heads, kv_heads, dim = rng.choice([(32, 8, 128), (32, 8, 128), (64, 8, 128), (8, 8, 64), (4, 2, 64)])
    kw = {"len_seed": rng.randrange(1 << 30)}
    if dim == 128:
        kw["fp8"] = rng.random() < 0.35
    kw["rows"] = rows = _log_int(rng, 1, 128)
    ctx = _log_int(rng, 16, min(32768, 400_000 // rows))
    kw["ctx_lo"], kw["ctx_hi"] = ctx // 2, ctx
    if kind == "append":
        kw["norm"] = rng.random() < 0.7
        kw["interleaved"] = rng.random() < 0.3
        kw["rot"] = rng.choice([dim, dim, dim // 2])
        kw["tree"] = rng.random() < 0.5
        new = _log_int(rng, 1, 64) if kw["tree"] else _log_int(rng, 1, max(1, 8192 // rows))
    elif kind == "read":
        new = _log_int(rng, 1, 32768 // rows)
    else:
        kw["tree"] = True
        kw["q_scale"] = rng.choice([1.0, 1.0, 2.0, 3.0])
        new = _log_int(rng, 1, 64)
    kw["new_lo"], kw["new_hi"] = max(1, new // 2), new
    return _case(None, kind, heads, kv_heads, dim, **kw)


def lengths(case):
    """(tokens in the cache before, new tokens) of the case's requests."""
    rng = np.random.Generator(np.random.PCG64(case["len_seed"]))
    prior = rng.integers(case["ctx_lo"], case["ctx_hi"] + 1, case["rows"])
    new = rng.integers(case["new_lo"], case["new_hi"] + 1, case["rows"])
    return prior.astype(np.int32), new.astype(np.int32)


def _quantised(x):
    """bf16 or fp32 vectors -> (E4M3 codes as bytes, fp32 scale): scale = amax / 448 rounded up to 8 significant bits."""
    x = x.float()
    amax = x.abs().amax(dim=-1, keepdim=True)
    # (by a tensor: torch multiplies by the rounded reciprocal of a number)
    bits = torch.where(amax > 0, amax / torch.full_like(amax, 448.0), torch.ones_like(amax)).view(torch.int32)
    scale = torch.where((bits & 0xFFFF) != 0, (bits | 0xFFFF) + 1, bits).view(torch.float32)
    return (x / scale).to(torch.float8_e4m3fn).view(torch.uint8), scale


def _put(pool, slots, k, v):
    if pool["fp8"]:
        for name, x in (("k", k), ("v", v)):
            codes, scale = _quantised(x)
            pool[name][slots] = codes
            pool[name + "_scale"][slots] = scale
    else:
        pool["k"][slots] = k.to(torch.bfloat16)
        pool["v"][slots] = v.to(torch.bfloat16)


def _values(pool, name, slots):
    """Cached vectors in fp32."""
    x = pool[name][slots]
    return x.view(torch.float8_e4m3fn).float() * pool[name + "_scale"][slots] if pool["fp8"] else x.float()


def prepare(case, seed):
    prior, new = lengths(case)
    heads, kv_heads, dim, rows = case["heads"], case["kv_heads"], case["dim"], case["rows"]
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device=dev, dtype=torch.bfloat16)

    # pages: a seeded permutation of a pool with a quarter to spare
    kv_len = prior.astype(np.int64) + new
    need = (kv_len + PAGE - 1) // PAGE
    num_pages = int(need.sum() + need.sum() // 4 + 8)
    max_pages = int(need.max())
    perm = torch.randperm(num_pages, generator=gen, device=dev, dtype=torch.int32)
    first = torch.from_numpy(np.cumsum(need) - need).to(dev)
    column = torch.arange(max_pages, device=dev)[None, :]
    table = torch.where(column < torch.from_numpy(need).to(dev)[:, None], perm[(first[:, None] + column).clamp_(max=num_pages - 1)], 0)
    table = table.to(torch.int32).contiguous()

    fp8 = case["fp8"]
    if own:
        from paper_2507_17769_b200 import PagedAttention

        pool = PagedAttention(heads, kv_heads, dim, num_pages, kv_dtype=1 if fp8 else 0)
    else:
        slots = num_pages * PAGE
        pool = {"fp8": fp8}
        for name in ("k", "v"):
            pool[name] = torch.empty((slots, kv_heads, dim), device=dev, dtype=torch.uint8 if fp8 else torch.bfloat16)
            if fp8:
                pool[name + "_scale"] = torch.empty((slots, kv_heads, 1), device=dev)

    # the cached context: a stretch of each of some requests at a time (an append fills its own new tokens)
    filled = prior if case["kind"] == "append" else kv_len
    r = done = 0
    while r < rows:
        part, begin, count, tokens = [], [], [], 0
        while r < rows and tokens < FILL_TOKENS:
            take = min(int(filled[r]) - done, FILL_TOKENS - tokens)
            if take > 0:
                part.append(r)
                begin.append(done)
                count.append(take)
                tokens += take
                done += take
            if done == int(filled[r]):
                r, done = r + 1, 0
        if part:
            k, v = normal(tokens, kv_heads, dim), normal(tokens, kv_heads, dim)
            if own:
                pool.write(k, v, table[torch.tensor(part, device=dev)].contiguous(), begin, count, max_pages=max_pages)
            else:
                pos = torch.from_numpy(np.concatenate([np.arange(b, b + c) for b, c in zip(begin, count)])).to(dev)
                row = torch.from_numpy(np.repeat(part, count)).to(dev)
                _put(pool, table[row, pos // PAGE].long() * PAGE + pos % PAGE, k, v)

    total = int(new.sum())
    start = np.cumsum(new) - new
    row = torch.from_numpy(np.repeat(np.arange(rows), new)).to(dev)         # request of each new token
    node = torch.from_numpy(np.arange(total) - np.repeat(start, new)).to(dev)  # its index in the request
    state = {"case": case, "pool": pool, "table": table, "max_pages": max_pages, "prior": prior, "new": new, "row": row, "node": node,
             "start": torch.from_numpy(start).to(dev), "prior_dev": torch.from_numpy(prior).to(dev).long(), "new_dev": torch.from_numpy(new).to(dev).long()}

    depth = node
    if case["tree"]:
        # a node's parent is one of the eight before it; its mask holds its ancestors and itself
        n = int(new.max())
        i = torch.arange(n, device=dev)
        low = (i - 8).clamp(min=0)
        parent = (low + (torch.rand((rows, n), generator=gen, device=dev) * (i - low)).long()).clamp(max=n - 1)
        sees = torch.eye(n, device=dev)[None].repeat(rows, 1, 1)
        sees[:, i[1:], :] += torch.nn.functional.one_hot(parent[:, 1:], n).float()
        for _ in range(max(1, n.bit_length())):
            sees = (torch.bmm(sees, sees) > 0).float()
        depth = (sees.sum(dim=2).long() - 1)[row, node]
        words = (n + 63) // 64
        bits = torch.nn.functional.pad(sees, (0, 64 * words - n)).long().view(rows, n, words, 64)
        packed = (bits << torch.arange(64, device=dev)).sum(dim=3)
        state["mask"] = packed[row, node].contiguous()  # int64 [tokens, words]
        # the accepted path: the ancestors of a drawn node, in order
        last = (torch.rand(rows, generator=gen, device=dev) * state["new_dev"]).long()
        on_path = sees[torch.arange(rows, device=dev), last] > 0
        state["index"] = torch.argsort((~on_path).long(), dim=1, stable=True).to(torch.int32).contiguous()
        state["count"] = on_path.sum(dim=1).to(torch.int32)

    if case["kind"] == "append":
        state["qkv"] = normal(total, (heads + 2 * kv_heads) * dim)  # a fused projection's output
        pos = state["prior_dev"][row] + depth
        state["pos"] = pos
        state["positions"] = pos.to(torch.int32) if case["tree"] else None
        rot = case["rot"]
        freq = THETA ** (-torch.arange(0, rot, 2, device=dev, dtype=torch.float64) / rot)
        angle = torch.arange(int(kv_len.max()), device=dev, dtype=torch.float64)[:, None] * freq
        state["cos_sin"] = torch.cat([angle.cos(), angle.sin()], dim=1).float()
        for name in ("q_weight", "k_weight"):
            state[name] = (1 + 0.2 * torch.randn(dim, generator=gen, device=dev)).to(torch.bfloat16) if case["norm"] else None
    if case["kind"] == "tree":
        state["q"] = (torch.randn((total, heads, dim), generator=gen, device=dev) * case["q_scale"]).to(torch.bfloat16)
    return state


def _qkv(state):
    c = state["case"]
    hq, hkv, d = c["heads"], c["kv_heads"], c["dim"]
    x = state["qkv"].view(-1, hq + 2 * hkv, d)
    return x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]


def _new_slots(state):
    pos = state["prior_dev"][state["row"]] + state["node"]
    return state["table"][state["row"], pos // PAGE].long() * PAGE + pos % PAGE


def _normed_rotated(x, weight, state):
    c = state["case"]
    x = x.float()
    if weight is not None:
        x = x * torch.rsqrt(x.square().mean(dim=-1, keepdim=True) + EPS) * weight.float()
    h = c["rot"] // 2
    cos, sin = (t[:, None, :] for t in state["cos_sin"][state["pos"]].split(h, dim=1))
    y = x.clone()
    if c["interleaved"]:
        a, b = x[..., 0:2 * h:2], x[..., 1:2 * h:2]
        y[..., 0:2 * h:2], y[..., 1:2 * h:2] = a * cos - b * sin, b * cos + a * sin
    else:
        a, b = x[..., :h], x[..., h:2 * h]
        y[..., :h], y[..., h:2 * h] = a * cos - b * sin, b * cos + a * sin
    return y


def _plain_append(state):
    q, k, v = _qkv(state)
    q = _normed_rotated(q, state["q_weight"], state).to(torch.bfloat16)
    slots = _new_slots(state)
    _put(state["pool"], slots, _normed_rotated(k, state["k_weight"], state), v)
    return {"q": q, "k": _values(state["pool"], "k", slots).to(torch.bfloat16), "v": _values(state["pool"], "v", slots).to(torch.bfloat16)}


def _plain_tree(state):
    c = state["case"]
    hkv, d, rows = c["kv_heads"], c["dim"], c["rows"]
    g, n = c["heads"] // hkv, int(state["new"].max())
    dev = state["q"].device
    keys = int((state["prior"] + state["new"]).max())
    pos = torch.arange(keys, device=dev)
    slots = state["table"][:, pos // PAGE].long() * PAGE + pos % PAGE  # [rows, keys]; entries past a sequence are not visible
    inside = pos[None] < (state["prior_dev"] + state["new_dev"])[:, None]
    k = _values(state["pool"], "k", slots).masked_fill_(~inside[:, :, None, None], 0).permute(0, 2, 3, 1)  # [rows, hkv, d, keys]
    node = torch.arange(n, device=dev)
    token = (state["start"][:, None] + node).clamp(max=state["q"].size(0) - 1)
    j = pos[None] - state["prior_dev"][:, None]  # index in the tree
    at = j.clamp(min=0, max=64 * state["mask"].size(1) - 1)
    words = torch.gather(state["mask"][token], 2, (at // 64)[:, None, :].expand(rows, n, keys))
    visible = ((((words >> (at % 64)[:, None, :]) & 1) != 0) | (j < 0)[:, None, :]) & inside[:, None, :]
    visible = visible.repeat_interleave(g, dim=1)[:, None]  # [rows, 1, n * g, keys]
    del words
    q = state["q"][token].float().view(rows, n, hkv, g, d).permute(0, 2, 1, 3, 4).reshape(rows, hkv, n * g, d)
    s = torch.matmul(q, k).mul_(d ** -0.5).masked_fill_(~visible, -math.inf)
    del k
    top = s.amax(dim=3, keepdim=True)
    p = s.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = p.sum(dim=3, keepdim=True)
    v = _values(state["pool"], "v", slots).masked_fill_(~inside[:, :, None, None], 0).permute(0, 2, 1, 3)
    out = torch.matmul(p, v) / torch.where(total > 0, total, 1.0)
    lse = (top + total.log()).squeeze(3)

    def packed(x):  # [rows, hkv, n * g, ...] -> [tokens, heads, ...]
        x = x.view(rows, hkv, n, g, *x.shape[3:])
        return x[state["row"], :, state["node"]].flatten(1, 2)

    return {"out": packed(out).to(torch.bfloat16), "lse": packed(lse)}


def _plain_accept(state):
    pool, prior = state["pool"], state["prior_dev"][:, None]
    i = torch.arange(state["index"].size(1), device=prior.device)[None]
    here = torch.minimum(i, state["new_dev"][:, None] - 1)
    there = torch.where(i < state["count"][:, None], state["index"].long(), here)  # (behind the path: onto itself)
    row = torch.arange(len(state["prior"]), device=prior.device)[:, None]
    src, dst = (state["table"][row, (prior + x) // PAGE].long() * PAGE + (prior + x) % PAGE for x in (there, here))
    names = ("k", "v", "k_scale", "v_scale") if pool["fp8"] else ("k", "v")
    moved = [pool[name][src] for name in names]
    for name, x in zip(names, moved):
        pool[name][dst] = x
    return _plain_read(state)


def _plain_read(state):
    slots = _new_slots(state)
    return {"k": _values(state["pool"], "k", slots).to(torch.bfloat16), "v": _values(state["pool"], "v", slots).to(torch.bfloat16)}


def run(state):
    kind = state["case"]["kind"]
    if not own:
        return {"append": _plain_append, "tree": _plain_tree, "accept": _plain_accept, "read": _plain_read}[kind](state)
    pa, table, prior, new = state["pool"], state["table"], state["prior"], state["new"]
    if kind == "tree":
        out, lse = pa.run_tree(state["q"], table, state["mask"], prior, new)
        return {"out": out, "lse": lse}
    got = {}
    if kind == "append":
        q, k, v = _qkv(state)
        got["q"] = pa.write_rope(q, k, v, table, prior, new, state["cos_sin"], positions=state["positions"], q_weight=state["q_weight"],
                                 k_weight=state["k_weight"], eps=EPS, interleaved=state["case"]["interleaved"])
    elif kind == "accept":
        pa.accept(table, prior, new, state["index"], state["count"])
    got["k"], got["v"] = pa.read(table, prior, new)
    return got


def work(case):
    prior, new = (x.astype(np.float64) for x in lengths(case))
    heads, kv_heads, dim = case["heads"], case["kv_heads"], case["dim"]
    tokens = float(new.sum())
    token_kv = 2 * kv_heads * (dim + 4) if case["fp8"] else 2 * kv_heads * dim * 2  # K and V of a cached token
    token_bf16 = 2 * kv_heads * dim * 2
    pages = 4 * float(np.ceil((prior + new) / PAGE).sum())
    if case["kind"] == "append":
        # q, k and v read, q and the cache written, the new tokens given back; one row of the table of angles a token
        byts = tokens * (2 * heads * dim * 2 + token_bf16 + token_kv + token_bf16 + 4 * case["rot"])
        return {"bytes": byts, "flops": tokens * (heads + kv_heads) * dim * 6}
    if case["kind"] == "tree":
        byts = float((prior + new).sum()) * token_kv + tokens * heads * (dim * 4 + 4) + tokens * 8 * math.ceil(new.max() / 64) + pages
        return {"bytes": byts, "flops": 4.0 * dim * heads * float((new * (prior + new)).sum())}
    if case["kind"] == "accept":
        # the path's tokens (some five a tree: the depth of a drawn node) moved, the tree's slots given back
        return {"bytes": 2 * 5 * case["rows"] * token_kv + tokens * (token_kv + token_bf16), "flops": 0.0}
    return {"bytes": tokens * (token_kv + token_bf16), "flops": 0.0}


def exact(case, seed):
    """The definitions in 64 bits, request by request (E4M3: nearest value, ties to even, with the scale as defined)."""
    s = prepare(case, seed)
    pool, table = s["pool"], s["table"]
    f64 = torch.float64

    def cached(name, slot):
        x = pool[name][slot]
        return x.view(torch.float8_e4m3fn).to(f64) * pool[name + "_scale"][slot].to(f64) if case["fp8"] else x.to(f64)

    def slots_of(r, lo, hi):
        p = torch.arange(lo, hi, device=table.device)
        return table[r].long()[p // PAGE] * PAGE + p % PAGE

    def e4m3(x):
        amax = x.abs().amax(-1, keepdim=True)
        m, e = torch.frexp(torch.where(amax > 0, amax / torch.full_like(amax, 448), torch.ones_like(amax)))
        scale = torch.ldexp(torch.ceil(m * 256) / 256, e)
        y = x / scale
        step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
        return torch.round(y / step) * step * scale

    spans = [(int(a), int(a + b)) for a, b in zip(s["prior"], s["new"])]
    if case["kind"] == "read":
        return {n: torch.cat([cached(n, slots_of(r, a, b)) for r, (a, b) in enumerate(spans)]) for n in ("k", "v")}
    if case["kind"] == "accept":
        got = {}
        for n in ("k", "v"):
            parts = []
            for r, (a, b) in enumerate(spans):
                x = cached(n, slots_of(r, a, b))
                path = s["index"][r, : int(s["count"][r])].long()
                parts.append(torch.cat([x[path], x[len(path):]]))
            got[n] = torch.cat(parts)
        return got
    if case["kind"] == "append":
        hq, hkv, d, h = case["heads"], case["kv_heads"], case["dim"], case["rot"] // 2
        x = s["qkv"].to(f64).view(-1, hq + 2 * hkv, d)
        angles = s["cos_sin"].to(f64)[s["pos"]]
        turn = torch.complex(angles[:, :h], angles[:, h:])[:, None]
        w = torch.ones((hq + hkv, d), device=x.device, dtype=f64)
        qk = x[:, : hq + hkv]
        if case["norm"]:
            w[:hq], w[hq:] = s["q_weight"].to(f64), s["k_weight"].to(f64)
            qk = qk / (qk.pow(2).mean(-1, keepdim=True) + EPS).sqrt()
        qk = qk * w
        front = qk[..., : 2 * h]
        pairs = front.unflatten(-1, (h, 2)) if case["interleaved"] else front.unflatten(-1, (2, h)).transpose(-1, -2)
        turned = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
        front = turned.flatten(-2) if case["interleaved"] else turned.transpose(-1, -2).flatten(-2)
        qk = torch.cat([front, qk[..., 2 * h:]], dim=-1)
        k, v = qk[:, hq:], x[:, hq + hkv:]
        return {"q": qk[:, :hq], "k": e4m3(k) if case["fp8"] else k, "v": e4m3(v) if case["fp8"] else v}
    group = case["heads"] // case["kv_heads"]
    outs, lses, t = [], [], 0
    for r, (a, b) in enumerate(spans):
        n = b - a
        k, v = (cached(name, slots_of(r, 0, b)).repeat_interleave(group, dim=1).transpose(0, 1) for name in ("k", "v"))  # [heads, keys, d]
        scores = s["q"][t:t + n].to(f64).transpose(0, 1) @ k.transpose(1, 2) / math.sqrt(case["dim"])
        j = torch.arange(n, device=table.device)
        sees = (s["mask"][t:t + n][:, j // 64] >> (j % 64)) & 1
        scores[:, :, a:] = scores[:, :, a:].masked_fill(sees[None] == 0, -math.inf)
        lse = torch.logsumexp(scores, dim=2)
        outs.append(((scores - lse[..., None]).exp() @ v).transpose(0, 1))
        lses.append(lse.transpose(0, 1))
        t += n
    return {"out": torch.cat(outs), "lse": torch.cat(lses)}
