"""Speculative decoding and a bounded KV cache, as cases that can be timed.

Four operators over the persistent KV cache of a rank (`paper_2411_01783_amd.binding.KVCache`):

  tree     attention of a tree of drafted tokens over the cache: a node sees the cached tokens at
           or before its position and, of its own tree, the nodes that its mask bits name
           (`cp_tree_attn`); O and the log-sum-exp come out, as of any partial attention
  accept   the K/V rows of the accepted path of every tree go into the cache (`cp_tree_accept`)
  weight   every cached key's attention weight, exp(score - LSE) summed over queries and heads, is
           added to what it had before (`cp_kv_attn_weight`)
  evict    every sequence's cache shrinks to a budget: the slots of the largest weight stay, the
           ones that lie behind the budget move into the holes in front of it (`cp_kv_evict`)

q, k and v are drawn from N(0, 1) in fp32 and rounded once, 16 query heads on 1 KV head of
dimension 128 per GPU unless a case says otherwise. Sequences' lengths belong to the case, not to
the seed: one case is one amount of work.
"""
import math
import random

import numpy as np
import torch

own = False

PAD_KV = 2**31 - 1


def listed():
    return [
        # Drafts of a single chat: one short conversation, the smallest call there is.
        dict(name="tree_chat", kind="tree", batch=1, len_lo=430, len_hi=430, nodes_lo=8, nodes_hi=8,
             words=1, nh=16, nkv=1, d=128, dtype="bf16", out="bf16"),
        # A batch of trees on one rank of a ring, whose results are merged with the other ranks'.
        dict(name="tree_rank_b16", kind="tree", batch=16, len_lo=2048, len_hi=8192, nodes_lo=12,
             nodes_hi=64, words=1, nh=16, nkv=1, d=128, dtype="bf16", out="fp32"),
        # One long document of 128K tokens and a wide tree: the most work for one sequence.
        dict(name="tree_long", kind="tree", batch=1, len_lo=131072, len_hi=131072, nodes_lo=61,
             nodes_hi=61, words=1, nh=16, nkv=1, d=128, dtype="bf16", out="bf16"),
        # Grouped KV heads of dimension 64 and trees wider than one word of mask.
        dict(name="tree_d64", kind="tree", batch=8, len_lo=900, len_hi=6000, nodes_lo=30,
             nodes_hi=100, words=2, nh=8, nkv=2, d=64, dtype="bf16", out="bf16"),
        # The small fp32 configuration.
        dict(name="tree_fp32", kind="tree", batch=3, len_lo=200, len_hi=900, nodes_lo=5,
             nodes_hi=33, words=1, nh=4, nkv=1, d=64, dtype="fp32", out="fp32"),
        # After the verification of a few chats' drafts, and of a large batch's.
        dict(name="accept_b4", kind="accept", batch=4, len_lo=300, len_hi=1800, nodes_lo=8,
             nodes_hi=25, words=1, nkv=1, d=128, dtype="bf16"),
        dict(name="accept_b64", kind="accept", batch=64, len_lo=500, len_hi=2500, nodes_lo=40,
             nodes_hi=128, words=2, nkv=8, d=128, dtype="bf16"),
        # A decode step of 32 long sequences as one of 16 ranks sees it.
        dict(name="weight_step", kind="weight", batch=32, len_lo=2048, len_hi=8192, q_lo=1, q_hi=1,
             nh=16, nkv=1, d=128, dtype="bf16", decay=0.98, ranks=16),
        # The last tokens of a few prompts say which of the prompts' keys matter.
        dict(name="weight_window", kind="weight", batch=4, len_lo=10000, len_hi=33000, q_lo=64,
             q_hi=64, nh=16, nkv=1, d=128, dtype="bf16", decay=0.0, ranks=1),
        # All of a prompt's queries weigh all of its keys.
        dict(name="weight_prompt", kind="weight", batch=1, len_lo=8192, len_hi=8192, q_lo=8192,
             q_hi=8192, nh=16, nkv=1, d=128, dtype="bf16", decay=0.0, ranks=1),
        # Full caches after a decode step: what came in beyond the budget has to go again.
        dict(name="evict_step", kind="evict", batch=32, len_lo=2048, len_hi=8192, over_lo=1,
             over_hi=4, budget=0, nkv=1, d=128, dtype="bf16", inplace=True),
        # Long prompts are cut down to a small cache that the decode steps then read.
        dict(name="evict_prompt", kind="evict", batch=4, len_lo=16000, len_hi=64000, over_lo=0,
             over_hi=0, budget=4096, nkv=1, d=128, dtype="bf16", inplace=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    kind = rng.choice(["tree", "tree", "accept", "weight", "weight", "evict"])
    nh, nkv, d, dtype = rng.choice([(16, 1, 128, "bf16")] * 3 + [
        (8, 1, 128, "bf16"), (8, 8, 128, "bf16"), (16, 4, 128, "bf16"), (8, 2, 64, "bf16"),
        (24, 3, 64, "bf16"), (4, 1, 64, "fp32"), (4, 2, 128, "fp32")])
    small = dtype == "fp32"
    if kind == "tree":
        batch = _log_int(rng, 1, 8 if small else 32)
        lo = _log_int(rng, 1, 600 if small else 60000 // batch)
        hi = lo + _log_int(rng, 1, 400 if small else 60000 // batch)
        nodes = _log_int(rng, 1, 40 if small else max(1, min(120, (1 << 27) // (nh * batch * hi))))
        return dict(kind="tree", batch=batch, len_lo=lo, len_hi=hi,
                    nodes_lo=max(1, nodes // 2), nodes_hi=nodes, words=(nodes + 63) // 64, nh=nh,
                    nkv=nkv, d=d, dtype=dtype, out="fp32" if small else rng.choice(["bf16", "fp32"]))
    if kind == "accept":
        lo, nodes = _log_int(rng, 4, 1500), _log_int(rng, 1, 128)
        return dict(kind="accept", batch=_log_int(rng, 1, 64), len_lo=lo,
                    len_hi=lo + _log_int(rng, 1, 1000), nodes_lo=max(1, nodes // 2), nodes_hi=nodes,
                    words=(nodes + 63) // 64, nkv=nkv, d=d, dtype=dtype)
    if kind == "weight":
        batch = _log_int(rng, 1, 4 if small else 32)
        lo = _log_int(rng, 3, 900 if small else 40000 // batch)
        hi = lo + _log_int(rng, 1, 500 if small else 40000 // batch)
        most = max(1, min(lo, (1 << 29) // (nh * batch * hi)))
        q = rng.choice([1, _log_int(rng, 1, min(most, 200)), _log_int(rng, 1, most)])
        return dict(kind="weight", batch=batch, len_lo=lo, len_hi=hi, q_lo=max(1, q // 2), q_hi=q,
                    nh=nh, nkv=nkv, d=d, dtype=dtype, decay=rng.choice([0.0, 0.9, 1.0]),
                    ranks=rng.choice([1, 4, 16]))
    batch = _log_int(rng, 1, 48)
    lo = _log_int(rng, 1, 100000 // batch)
    hi = lo + _log_int(rng, 1, 100000 // batch)
    inplace = rng.random() < 0.6
    if inplace and rng.random() < 0.5:
        over = _log_int(rng, 1, 64)
        return dict(kind="evict", batch=batch, len_lo=lo, len_hi=hi, over_lo=1, over_hi=over,
                    budget=0, nkv=nkv, d=d, dtype=dtype, inplace=True)
    return dict(kind="evict", batch=batch, len_lo=lo, len_hi=hi, over_lo=0, over_hi=0,
                budget=_log_int(rng, 1, hi), nkv=nkv, d=d, dtype=dtype, inplace=inplace)


# ---------------------------------------------------------------------------
# sizes of a case

def _spread(case, what, salt):
    lo, hi = case[what + "_lo"], case[what + "_hi"]
    rng = np.random.default_rng(lo * 131 + hi * 7 + case["batch"] + salt)
    return [int(x) for x in rng.integers(lo, hi + 1, size=case["batch"])]


def _lengths(case):
    return _spread(case, "len", 0)


def _nodes(case):
    return _spread(case, "nodes", 1)


def _queries(case):      # the newest tokens of every sequence
    return [min(q, n) for q, n in zip(_spread(case, "q", 2), _lengths(case))]


def _budgets(case):
    lens = _lengths(case)
    if case["budget"]:
        return [min(case["budget"], n) for n in lens]
    return [max(n - o, 0) for n, o in zip(lens, _spread(case, "over", 3))]


SINKS = 4                # positions that an eviction never drops, and how many of the newest
RECENT = 64


def _kept(case):
    """Slots that every sequence keeps: its budget, or what is protected if that is more."""
    lens = _lengths(case)
    return [min(n, max(b, min(n, SINKS) + max(0, min(n - SINKS, RECENT))))
            for n, b in zip(lens, _budgets(case))]


def _paths(case):
    """Parents of every tree's nodes and the node that the verification accepts; -1: none."""
    rng = random.Random(case["batch"] * 977 + case["nodes_hi"])
    trees, accepted = [], []
    for n in _nodes(case):
        parents = [-1]
        for i in range(1, n):    # chains with side branches, as a draft model's best guesses give
            parents.append(i - 1 if rng.random() < 0.5 else rng.randrange(-1, i))
        trees.append(parents)
        accepted.append(rng.randrange(-1, n))
    return trees, accepted


def _ancestors(parents):
    """For every node of a tree the nodes on its path from the root, itself the last."""
    out = []
    for i, p in enumerate(parents):
        out.append((out[p] if p >= 0 else []) + [i])
    return out


def _pairs(case):
    """(query, key) pairs that see each other, over all sequences."""
    if case["kind"] == "tree":
        trees, _ = _paths(case)
        return sum(n * len(t) + sum(len(a) for a in _ancestors(t))
                   for n, t in zip(_lengths(case), trees))
    return sum(q * n - q * (q - 1) // 2 for q, n in zip(_queries(case), _lengths(case)))


def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    row = case["nkv"] * case["d"] * e            # a token's K, or V
    keys = sum(_lengths(case))
    if case["kind"] == "tree":
        n, eo = sum(_nodes(case)), 2 if case["out"] == "bf16" else 4
        q = case["nh"] * case["d"]
        return {"bytes": 2 * keys * row + 4 * keys + n * (q * e + 2 * row + 4 + 8 * case["words"])
                + n * (q * eo + 4 * case["nh"]),
                "flops": 4 * q * _pairs(case)}
    if case["kind"] == "accept":
        trees, accepted = _paths(case)
        rows = sum(len(_ancestors(t)[a]) for t, a in zip(trees, accepted) if a >= 0)
        return {"bytes": 4 * rows * row + 8 * rows + case["batch"] * (16 + 8 * case["words"]),
                "flops": 0}
    if case["kind"] == "weight":
        n = sum(_queries(case))
        return {"bytes": keys * row + 4 * keys + n * (case["nh"] * (case["d"] * e + 4) + 4)
                + 4 * keys * (2 if case["decay"] else 1),
                "flops": 2 * case["nh"] * case["d"] * _pairs(case)}
    lens, kept = _lengths(case), _kept(case)
    # in place at most the slots behind the kept ones move (each hole takes one of them)
    moved = sum(min(k, n - k) for n, k in zip(lens, kept)) if case["inplace"] else sum(kept)
    written = sum(n - k for n, k in zip(lens, kept)) if case["inplace"] else 0
    return {"bytes": 8 * keys + moved * (4 * row + 8) + 8 * written, "flops": 0}


# ---------------------------------------------------------------------------
# inputs

def _dt(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _gen(seed, i):
    return torch.Generator("cuda").manual_seed((int(seed) * 1000 + i) % (1 << 62))


def _normal(seed, i, shape, dtype):
    return torch.randn(shape, generator=_gen(seed, i), device="cuda").to(_dt(dtype))


def _i32(x):
    return torch.as_tensor(np.asarray(x, dtype=np.int32)).to("cuda")


def _ends(counts):
    return [0] + [int(x) for x in np.cumsum(np.asarray(counts, dtype=np.int64))]


def _cache(case, seed, capacity, lens, grow=0):
    """A cache whose sequences hold `lens` tokens at positions 0, 1, ..., the slots behind them
    unused. Rows of `grow` tokens behind them are there too (for caches that take them back)."""
    ends = _ends(capacity)
    slots = ends[-1]
    pos = np.full(slots, PAD_KV, dtype=np.int32)
    for b, n in enumerate(lens):
        pos[ends[b]:ends[b] + n] = np.arange(n)
    shape = (slots, case["nkv"], case["d"])
    used_slot = torch.as_tensor(pos != PAD_KV).to("cuda")[:, None, None]
    st = dict(k=_normal(seed, 1, shape, case["dtype"]) * used_slot,
              v=_normal(seed, 2, shape, case["dtype"]) * used_slot,
              kv_pos=_i32(pos), cu=_i32(ends), used=_i32(list(lens) + [0]), ends=ends,
              lens=list(lens), capacity=list(capacity))
    return st


def _handle(cache):
    """The cache as the binding's handle."""
    from paper_2411_01783_amd import binding as B
    h = B.KVCache(cache["capacity"], cache["k"].shape[1], cache["k"].shape[2],
                  dtype=cache["k"].dtype)
    h.k, h.v, h.kv_pos, h.used = cache["k"], cache["v"], cache["kv_pos"], cache["used"]
    return h


def _masks(case, trees):
    """Mask bits of all trees' nodes, 64 a word, and the nodes' depths."""
    rows, depth = [], []
    for parents in trees:
        for path in _ancestors(parents):
            words = [0] * case["words"]
            for t in path:
                words[t // 64] |= 1 << (t % 64)
            rows.append([w - (1 << 64) if w >> 63 else w for w in words])
            depth.append(len(path) - 1)
    return torch.as_tensor(np.asarray(rows, dtype=np.int64)).to("cuda"), depth


def prepare(case, seed):
    st = dict(case=case)
    lens = _lengths(case)
    # caches are allocated with room to grow
    if case["kind"] in ("tree", "accept"):
        nodes = _nodes(case)
        trees, accepted = _paths(case)
        c = _cache(case, seed, [n + 128 + 64 for n in lens], lens)
        total = sum(nodes)
        st["mask"], depth = _masks(case, trees)
        start = np.repeat(np.asarray(lens), nodes)
        st.update(k_new=_normal(seed, 3, (total, case["nkv"], case["d"]), case["dtype"]),
                  v_new=_normal(seed, 4, (total, case["nkv"], case["d"]), case["dtype"]),
                  q_pos=_i32(start + np.asarray(depth)), cu_q=_i32(_ends(nodes)), ends_q=_ends(nodes),
                  most_q=max(nodes))
        if case["kind"] == "tree":
            st["q"] = _normal(seed, 0, (total, case["nh"], case["d"]), case["dtype"])
        else:
            st["accepted"] = _i32(accepted)
            st["used0"] = c["used"].clone()
    elif case["kind"] == "weight":
        nq = _queries(case)
        c = _cache(case, seed, [n + 128 for n in lens], lens)
        q_pos = np.concatenate([np.arange(n - q, n) for q, n in zip(nq, lens)])
        st.update(q=_normal(seed, 0, (sum(nq), case["nh"], case["d"]), case["dtype"]),
                  q_pos=_i32(q_pos), cu_q=_i32(_ends(nq)), ends_q=_ends(nq), most_q=max(nq))
        # the log-sum-exp over all ranks' keys, of which this rank holds its share
        seen = torch.as_tensor((q_pos + 1) * case["ranks"], dtype=torch.float32).to("cuda")
        st["lse"] = (seen.log()[:, None] + 0.5 + 0.1 * torch.randn(
            (sum(nq), case["nh"]), generator=_gen(seed, 5), device="cuda")).contiguous()
        st["weight"] = (c["kv_pos"] != PAD_KV) * torch.rand(
            (c["k"].shape[0],), generator=_gen(seed, 6), device="cuda")
        st["weight0"] = st["weight"].clone()
    else:
        budgets = _budgets(case)
        c = _cache(case, seed, [n + 128 for n in lens], lens)
        slots = c["k"].shape[0]
        # a heavy tail, and keys that nothing has looked at since they came
        w = torch.rand((slots,), generator=_gen(seed, 6), device="cuda")
        w = torch.where(w < 0.1, 0.0, (w - 0.1) ** 8) * (c["kv_pos"] != PAD_KV)
        # what a pass changes besides K and V in one buffer, set back by one copy
        buf = torch.cat([c["kv_pos"], w.view(torch.int32), c["used"]])
        st["book"], st["book0"] = buf, buf.clone()
        c["kv_pos"], c["used"] = buf[:slots], buf[2 * slots:]
        st["weight"] = buf[slots:2 * slots].view(torch.float32)
        st["budget"], st["keep_from"] = _i32(budgets), _i32([max(n - RECENT, 0) for n in lens])
        if not case["inplace"]:
            st["into"] = _cache(case, seed + 1, [k + 256 for k in _kept(case)], [0] * case["batch"])
            st["into_weight"] = torch.zeros(st["into"]["k"].shape[0], device="cuda")
    st["cache"] = c
    if own:
        st["handle"] = _handle(c)
        if "into" in st:
            st["into_handle"] = _handle(st["into"])
    return st


# ---------------------------------------------------------------------------
# one pass

def run(st):
    case, c = st["case"], st["cache"]
    kind = case["kind"]
    if kind == "accept":
        c["used"].copy_(st["used0"])         # the same step again
    elif kind == "weight" and case["decay"]:
        st["weight"].copy_(st["weight0"])
    elif kind == "evict" and case["inplace"]:
        st["book"].copy_(st["book0"])
    return (_run_own if own else _run_plain)(st, case, c, kind)


def _run_own(st, case, c, kind):
    from paper_2411_01783_amd import binding as B
    h = st["handle"]
    if kind == "tree":
        return B.cp_tree_attn(h, st["q"], st["q_pos"], st["k_new"], st["v_new"], st["cu_q"],
                              st["mask"], out_dtype=_dt(case["out"]))
    if kind == "accept":
        B.cp_tree_accept(h, st["k_new"], st["v_new"], st["q_pos"], st["cu_q"], st["mask"],
                         st["accepted"])
        return h.k, h.v, h.kv_pos, h.used
    if kind == "weight":
        return B.cp_kv_attn_weight(h, st["q"], st["q_pos"], st["lse"], st["weight"], st["cu_q"],
                                   decay=case["decay"])
    into = st.get("into_handle")
    B.cp_kv_evict(h, st["weight"], st["budget"], protect_from=st["keep_from"], sinks=SINKS,
                  into=into, into_weight=st.get("into_weight"))
    if into is None:
        return h.k, h.v, h.kv_pos, st["weight"], h.used
    return into.k, into.v, into.kv_pos, st["into_weight"], into.used


def _run_plain(st, case, c, kind):
    return {"tree": _plain_tree, "accept": _plain_accept, "weight": _plain_weight,
            "evict": _plain_evict}[kind](st, case, c)


def _padded(first, count, longest):
    """Rows of the sequences as [batch, longest], those behind a sequence's end read from its last
    one, and which of them there are."""
    i = torch.arange(longest, device="cuda")
    n = count.long()[:, None]
    return first.long()[:, None] + torch.minimum(i, n - 1), i < n


def _cached(c):
    return _padded(c["cu"][:-1], c["used"][:-1], max(c["lens"]))


def _asked(st):
    return _padded(st["cu_q"][:-1], st["cu_q"][1:] - st["cu_q"][:-1], st["most_q"])


def _heads(x, rows, nkv):
    """[tokens, heads, d] as fp32 [batch, nkv, rows * heads of a KV head, d]."""
    batch, n = rows.shape
    x = x[rows].float().unflatten(2, (nkv, -1)).transpose(1, 2)
    return x.reshape(batch, nkv, -1, x.shape[-1])


def _plain_tree(st, case, c):
    nh, nkv, d = case["nh"], case["nkv"], case["d"]
    key, there = _cached(c)
    row, real = _asked(st)
    batch, m = row.shape
    bit = torch.arange(64, device="cuda")
    tree = ((st["mask"][row][..., None] >> bit) & 1).bool().reshape(batch, m, -1)[:, :, :m]
    cached = (c["kv_pos"][key][:, None] <= st["q_pos"][row][..., None]) & there[:, None]
    seen = torch.cat([cached, tree & real[:, None]], 2)[:, None, :, None]     # of [b, 1, m, 1, keys]
    k = torch.cat([_heads(c["k"], key, nkv), _heads(st["k_new"], row, nkv)], 2)
    v = torch.cat([_heads(c["v"], key, nkv), _heads(st["v_new"], row, nkv)], 2)
    s = (_heads(st["q"], row, nkv) @ k.transpose(2, 3).contiguous()).mul_(1.0 / math.sqrt(d))
    s = s.view(batch, nkv, m, nh // nkv, -1).masked_fill_(~seen, -math.inf)
    top = s.amax(-1, keepdim=True).clamp_(min=-3e38)
    p = s.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = (p.view(batch, nkv, -1, p.shape[-1]) @ v).view(batch, nkv, m, nh // nkv, d) / total
    o = torch.where(total > 0, o, 0.0).transpose(1, 2).reshape(batch, m, nh, d)
    lse = (top + total.log())[..., 0].transpose(1, 2).reshape(batch, m, nh)
    return o[real].to(_dt(case["out"])), lse[real]


def _plain_accept(st, case, c):
    batch = case["batch"]
    bit = torch.arange(64, device="cuda")
    first, acc = st["cu_q"][:-1].long(), st["accepted"].long()
    row = st["mask"][(first + acc).clamp(min=0)]                       # [batch, words]
    take = ((row[:, :, None] >> bit) & 1).bool().reshape(batch, -1) & (acc >= 0)[:, None]
    size = (st["cu_q"][1:] - st["cu_q"][:-1])[:, None]
    take &= torch.arange(take.shape[1], device="cuda") < size
    slot = c["cu"][:-1, None] + c["used"][:batch, None] + take.cumsum(1) - 1
    count = take.sum(1)
    b, t = (take & (slot < c["cu"][1:, None])).nonzero(as_tuple=True)
    src, dst = first[b] + t, slot[b, t]
    c["k"][dst] = st["k_new"][src]
    c["v"][dst] = st["v_new"][src]
    c["kv_pos"][dst] = st["q_pos"][src]
    room = c["cu"][1:] - c["cu"][:-1] - c["used"][:batch]
    c["used"][:batch] += torch.minimum(count, room).to(torch.int32)
    return c["k"], c["v"], c["kv_pos"], c["used"]


def _plain_weight(st, case, c):
    nh, nkv, d = case["nh"], case["nkv"], case["d"]
    key, there = _cached(c)
    row, real = _asked(st)
    batch, m = row.shape
    k = _heads(c["k"], key, nkv).transpose(2, 3).contiguous()
    s = (_heads(st["q"], row, nkv) @ k).mul_(1.0 / math.sqrt(d)).view(batch, nkv, m, nh // nkv, -1)
    lse = st["lse"][row].view(batch, m, nkv, -1, 1).transpose(1, 2)
    p = s.sub_(lse).exp_()
    seen = (c["kv_pos"][key][:, None] <= st["q_pos"][row][..., None]) & real[..., None]
    add = p.masked_fill_(~seen[:, None, :, None], 0.0).sum((1, 2, 3))[there]
    w, at = st["weight"], key[there]
    w[at] = w[at] * case["decay"] + add if case["decay"] else add
    return w


def _plain_evict(st, case, c):
    d, wd = st.get("into", c), st.get("into_weight", st["weight"])
    key, there = _cached(c)
    batch, longest = key.shape
    i = torch.arange(longest, device="cuda").expand(batch, -1)
    pos, w = c["kv_pos"][key], st["weight"][key]
    safe = ((pos < SINKS) | (pos >= st["keep_from"][:, None])) & there
    cap = (d["cu"][1:] - d["cu"][:-1])
    keep = torch.minimum(torch.maximum(st["budget"], safe.sum(1)), torch.minimum(cap, there.sum(1)))
    w = torch.where(safe, math.inf, torch.where(there, w, -math.inf))
    rank = w.sort(dim=1, descending=True, stable=True).indices.argsort(1)
    kept, front = rank < keep[:, None], i < keep[:, None]
    hole, mover = front & ~kept, ~front & kept
    # the n-th slot that moves goes to the n-th hole
    order = torch.where(mover, mover.cumsum(1) - 1, longest)
    nth = torch.zeros((batch, longest + 1), dtype=torch.int64, device="cuda").scatter_(1, order, i)
    source = torch.where(hole, nth.gather(1, (hole.cumsum(1) - 1).clamp(min=0)), i)
    b, to = (hole if d is c else front).nonzero(as_tuple=True)
    src, dst = c["cu"].long()[b] + source[b, to], d["cu"].long()[b] + to
    d["k"][dst] = c["k"][src]
    d["v"][dst] = c["v"][src]
    d["kv_pos"][dst], wd[dst] = c["kv_pos"][src], st["weight"][src]
    # what lies behind the kept slots is unused
    owner = torch.repeat_interleave(torch.arange(batch, device="cuda"), cap.long(),
                                    output_size=wd.shape[0])
    free = torch.arange(wd.shape[0], device="cuda") - d["cu"][owner] >= keep[owner]
    d["kv_pos"].masked_fill_(free, PAD_KV)
    wd.masked_fill_(free, 0.0)
    d["used"][:batch] = keep.to(torch.int32)
    return d["k"], d["v"], d["kv_pos"], wd, d["used"]


# ---------------------------------------------------------------------------
# the same from the definitions, in 64 bits

def exact(case, seed):
    st = prepare(case, seed)
    return {"tree": _exact_tree, "accept": _exact_accept, "weight": _exact_weight,
            "evict": _exact_evict}[case["kind"]](st, case, st["cache"])


def _blocks(n, heads, keys):
    step = max(1, (1 << 26) // (heads * keys))
    return [(i, min(n, i + step)) for i in range(0, n, step)]


def _exact_tree(st, case, c):
    nh, nkv, d = case["nh"], case["nkv"], case["d"]
    trees, _ = _paths(case)
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(st["q"].shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    for b, n in enumerate(c["lens"]):
        q0, k0 = st["ends_q"][b], c["ends"][b]
        paths = _ancestors(trees[b])
        keys = torch.cat([c["k"][k0:k0 + n], st["k_new"][q0:q0 + len(paths)]]).double()
        vals = torch.cat([c["v"][k0:k0 + n], st["v_new"][q0:q0 + len(paths)]]).double()
        hide = torch.ones((len(paths), n + len(paths)), dtype=torch.bool, device="cuda")
        hide[:, :n] = st["q_pos"][q0:q0 + len(paths), None] < c["kv_pos"][k0:k0 + n]
        for i, path in enumerate(paths):
            hide[i, [n + t for t in path]] = False
        for h in range(nh):
            kh, vh = keys[:, h * nkv // nh], vals[:, h * nkv // nh]
            for i, j in _blocks(len(paths), 1, n + len(paths)):
                s = st["q"][q0 + i:q0 + j, h].double() @ kh.T / d ** 0.5
                s[hide[i:j]] = -math.inf
                lse[q0 + i:q0 + j, h] = torch.logsumexp(s, 1)
                out[q0 + i:q0 + j, h] = torch.softmax(s, 1) @ vh
    return out, lse


def _exact_accept(st, case, c):
    trees, accepted = _paths(case)
    for b, (parents, node) in enumerate(zip(trees, accepted)):
        path = []
        while node >= 0:
            path.insert(0, node)
            node = parents[node]
        for t in path[:c["capacity"][b] - c["lens"][b]]:
            dst, src = c["ends"][b] + int(c["used"][b]), st["ends_q"][b] + t
            c["k"][dst], c["v"][dst] = st["k_new"][src], st["v_new"][src]
            c["kv_pos"][dst] = st["q_pos"][src]
            c["used"][b] += 1
    return c["k"].double(), c["v"].double(), c["kv_pos"], c["used"]


def _exact_weight(st, case, c):
    nh, nkv, d = case["nh"], case["nkv"], case["d"]
    w = st["weight"].double()
    for b, n in enumerate(c["lens"]):
        q0, q1, k0 = st["ends_q"][b], st["ends_q"][b + 1], c["ends"][b]
        w[k0:k0 + n] *= case["decay"]
        pos = c["kv_pos"][k0:k0 + n]
        for h in range(nh):
            kh = c["k"][k0:k0 + n, h * nkv // nh].double()
            for i, j in _blocks(q1 - q0, 1, n):
                s = kh @ st["q"][q0 + i:q0 + j, h].double().T / d ** 0.5
                p = torch.exp(s - st["lse"][q0 + i:q0 + j, h].double())
                w[k0:k0 + n] += (p * (pos[:, None] <= st["q_pos"][q0 + i:q0 + j])).sum(1)
    return w


def _exact_evict(st, case, c):
    d, wd = (c, st["weight"]) if case["inplace"] else (st["into"], st["into_weight"])
    pos_of, w_of = c["kv_pos"].cpu().numpy().copy(), st["weight"].cpu().numpy().copy()
    keep_from, budget = st["keep_from"].tolist(), st["budget"].tolist()
    pos_to, w_to, used_to = d["kv_pos"].cpu().numpy(), wd.cpu().numpy(), d["used"].cpu().numpy()
    pos_to, w_to, used_to = pos_to.copy(), w_to.copy(), used_to.copy()
    where, whence = [], []
    for b, n in enumerate(c["lens"]):
        k0, d0, d1 = c["ends"][b], d["ends"][b], d["ends"][b + 1]
        p, w = pos_of[k0:k0 + n], w_of[k0:k0 + n].astype(np.float64)
        must = (p < SINKS) | (p >= keep_from[b])
        keep = int(min(n, d1 - d0, max(budget[b], must.sum())))
        # by protection, then by weight, then by slot
        rank = np.lexsort((np.arange(n), -w, ~must))
        stays = np.zeros(n, dtype=bool)
        stays[rank[:keep]] = True
        behind = iter(np.flatnonzero(stays[keep:]) + keep)
        for i in range(keep):
            s = i if stays[i] else int(next(behind))
            where.append(d0 + i)
            whence.append(k0 + s)
        pos_to[d0:d1], w_to[d0:d1] = PAD_KV, 0.0
        used_to[b] = keep
    where, whence = np.asarray(where, dtype=np.int64), np.asarray(whence, dtype=np.int64)
    pos_to[where], w_to[where] = pos_of[whence], w_of[whence]
    to = torch.as_tensor(where).to("cuda")
    fro = torch.as_tensor(whence).to("cuda")
    k, v = d["k"].double(), d["v"].double()
    k[to], v[to] = c["k"].double()[fro], c["v"].double()[fro]
    return (k, v, torch.as_tensor(pos_to).to("cuda"), torch.as_tensor(w_to).double().to("cuda"),
            torch.as_tensor(used_to).to("cuda"))
