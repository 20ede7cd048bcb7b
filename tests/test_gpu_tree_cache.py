"""Trees of drafted tokens over the KV cache, their commit, accumulated attention weight and eviction,
against plain 64-bit forms."""
import ctypes

import numpy as np
import pytest
import torch

from gpu_util import dev, i32, randn
from paper_2411_01783_amd import binding as B
from tree_cache_util import (PAD, bits, check_tree, ends, evict_reference, make_cache, random_parents,
                             tree_reference, weight_reference)

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def tree_inputs(seed, lens, nodes, nh, nkv, d, dtype, words=None):
    rng = np.random.default_rng(seed)
    cu = ends(nodes)
    t = int(cu[-1])
    parents = random_parents(rng, nodes)
    mask = B.cp_tree_mask(parents, cu, words)
    depth = np.array([bits(mask[i:i + 1], 64 * mask.shape[1]).sum() - 1 for i in range(t)], dtype=np.int64)
    q_pos = np.repeat(np.asarray(lens, dtype=np.int64), nodes) + depth
    q, q64 = randn(seed + 2, (t, nh, d), dtype)
    k, k64 = randn(seed + 3, (t, nkv, d), dtype)
    v, v64 = randn(seed + 4, (t, nkv, d), dtype)
    return dict(q=q, k=k, v=v, q64=q64, k64=k64, v64=v64, q_pos=q_pos.astype(np.int32), cu=cu, mask=mask,
                parents=parents)


def run_tree(cache, x, out_dtype, own=True, **kw):
    return B.cp_tree_attn(cache, dev(x["q"]), i32(x["q_pos"]), dev(x["k"]) if own else None,
                          dev(x["v"]) if own else None, i32(x["cu"]),
                          dev(x["mask"]) if own else None, out_dtype=out_dtype, **kw)


def reference(x, host, own=True, scale=None):
    return tree_reference(x["q64"], x["q_pos"], x["cu"], host, x["k64"] if own else None,
                          x["v64"] if own else None, x["mask"] if own else None, scale)


# lens, nodes, heads, KV heads, head_dim, dtype. What they are for: one node; a tile's edges; a cache
# that holds nothing, a tree without nodes; many short sequences; wide trees; many rows; odd groups
TREES = {
    "one": ([5], [1], 1, 1, 128, "bf16"),
    "edges": ([31, 32, 33, 127, 128, 129], [1, 2, 1, 2, 1, 2], 16, 1, 128, "bf16"),
    "nothing": ([0, 40, 0, 7], [3, 0, 0, 1], 16, 1, 128, "bf16"),
    "chat": ([430], [8], 16, 1, 128, "bf16"),
    "many_seqs": ([3 + 5 * (i % 17) for i in range(150)], [1 + i % 3 for i in range(150)], 8, 2, 128, "bf16"),
    "wide": ([700, 90], [130, 65], 8, 2, 128, "bf16"),
    "rows": ([1500, 300], [64, 40], 16, 1, 128, "bf16"),
    "odd_group": ([260, 77], [20, 31], 15, 3, 128, "bf16"),
    "long": ([9000], [3], 16, 1, 128, "bf16"),
    "d64": ([333, 64, 65], [12, 33, 64], 8, 2, 64, "bf16"),
    "d64_rows": ([600], [100], 32, 2, 64, "bf16"),
    "d64_few": ([600, 1200], [1, 2], 8, 1, 64, "bf16"),
    # enough products for the form that takes 256 rows at a time: its edges, more than 64 sequences with
    # several to a workgroup, odd groups and counts of sub-tiles, one row block and a row more
    "m_edges": ([9991, 33, 0, 64, 63], [61, 16, 17, 1, 40], 16, 1, 128, "bf16"),
    "m_seqs": ([700 + 97 * (i % 17) if i % 9 else 0 for i in range(100)], [5 + 5 * (i % 4) if i % 7 else 0 for i in range(100)],
               8, 2, 128, "bf16"),
    "m_odd_group": ([2500, 31], [131, 130], 15, 3, 128, "bf16"),
    "m_one_more": ([16417], [257], 2, 2, 128, "bf16"),
    "d64_mid": ([3303, 700], [100, 61], 32, 2, 64, "bf16"),
    "m_d64": ([7003, 700], [100, 61], 32, 2, 64, "bf16"),
    "d64_seqs": ([500 + 131 * (i % 7) for i in range(70)], [9 + i % 8 for i in range(70)], 8, 2, 64, "bf16"),
    "m_d64_seqs": ([1500 + 131 * (i % 7) for i in range(70)], [9 + i % 8 for i in range(70)], 8, 2, 64, "bf16"),
    "m_few_rows": ([26000, 9001], [3, 4], 16, 8, 128, "bf16"),
    "fp32": ([200, 0, 333], [5, 33, 66], 4, 1, 64, "fp32"),
    "fp32_128": ([200, 129], [9, 2], 6, 2, 128, "fp32"),
}


@pytest.mark.parametrize("out_dtype", [BF16, F32])
@pytest.mark.parametrize("name", list(TREES))
def test_tree_attention(name, out_dtype):
    lens, nodes, nh, nkv, d, dtype = TREES[name]
    cache, host = make_cache(11, lens, [n + 1 + 37 * (i % 3) for i, n in enumerate(lens)], nkv, d, dtype)
    x = tree_inputs(21, lens, nodes, nh, nkv, d, dtype)
    got = run_tree(cache, x, out_dtype)
    check_tree(got, reference(x, host), d, out_dtype, dtype == "bf16" and out_dtype == BF16, name)
    got = run_tree(cache, x, out_dtype, own=False)
    check_tree(got, reference(x, host, own=False), d, out_dtype, dtype == "bf16" and out_dtype == BF16, name)


def test_which_trees_have_many_rows():
    # (the workspace holds two row blocks of parts a workgroup)
    for name, (lens, nodes, nh, nkv, d, dtype) in TREES.items():
        s = B.make_shape(B.CP_BF16 if dtype == "bf16" else B.CP_FP32, d, nh, nkv, sum(nodes), sum(lens) + 40 * len(lens),
                         len(lens))
        few = 2 * 512 * 32 * (d + 2) * 4 + 512
        assert (B.cp_workspace_bytes(s, B.CP_WS_TREE) > few) == name.startswith("m_"), name


@pytest.mark.parametrize("out_dtype", [BF16, F32])
@pytest.mark.parametrize("name", ["chat", "long", "d64", "fp32", "m_edges", "m_odd_group", "m_d64", "m_seqs"])
def test_scores_that_keep_growing(name, out_dtype):
    """The running maximum rises all the way along the cache, in the tree, and by hundreds at single keys."""
    lens, nodes, nh, nkv, d, dtype = TREES[name]
    cache, host = make_cache(61, lens, [n + 5 for n in lens], nkv, d, dtype)
    x = tree_inputs(62, lens, nodes, nh, nkv, d, dtype)
    grow = np.ones(cache.slots)
    for b, n in enumerate(lens):
        lo = host["cu"][b]
        grow[lo:lo + n] = np.linspace(0.1, 9.0, n)
        grow[lo + n // 3:lo + n:997] = 60.0
    k = (cache.k.double().cpu() * torch.as_tensor(grow)[:, None, None]).to(cache.k.dtype)
    cache.k.copy_(k)
    host["k"] = k.double().numpy()
    x["k"] = (x["k"].double() * 10).to(x["k"].dtype)
    x["k64"] = x["k"].double().numpy()
    check_tree(run_tree(cache, x, out_dtype), reference(x, host), d, out_dtype, dtype == "bf16" and out_dtype == BF16, name)


def test_rows_too_wide_for_offsets_of_32_bits():
    # 65536 KV heads: the rows of a tile lie up to 500 MB apart
    nkv, group, d, n, t = 65536, 17, 128, 70, 2
    free, _ = torch.cuda.mem_get_info()
    if free < 20 << 30:
        pytest.skip("16 GB of tensors")
    cache = B.KVCache([n], nkv, d)
    g = torch.Generator(device="cuda").manual_seed(71)
    rand = lambda *s: torch.randn(s, device="cuda", dtype=BF16, generator=g)
    cache.k.copy_(rand(n, nkv, d))
    cache.v.copy_(rand(n, nkv, d))
    cache.kv_pos.copy_(torch.arange(n, dtype=torch.int32))
    cache.used.copy_(i32([n, 0]))
    q, k, v = rand(t, nkv * group, d), rand(t, nkv, d), rand(t, nkv, d)
    q_pos, cu, mask = np.array([40, n], dtype=np.int32), ends([t]), np.array([[1], [3]], dtype=np.int64)
    got = B.cp_tree_attn(cache, q, i32(q_pos), k, v, i32(cu), dev(torch.as_tensor(mask)), out_dtype=F32)
    some = [0, 1, 32767, 40000, 65535]
    at = torch.as_tensor(some).cuda()
    rows = (at[:, None] * group + torch.arange(group, device="cuda")).reshape(-1)
    h64 = lambda a, i: a[:, i].double().cpu().numpy()
    host = dict(k=h64(cache.k, at), v=h64(cache.v, at), kv_pos=np.arange(n), used=[n], cu=[0, n])
    ref = tree_reference(h64(q, rows), q_pos, cu, host, h64(k, at), h64(v, at), mask)
    check_tree((got[0][:, rows], got[1][:, rows]), ref, d, F32, False)


@pytest.mark.parametrize("name", ["edges", "rows", "chat", "d64", "fp32", "m_edges", "m_odd_group", "m_d64"])
def test_tree_masks_that_are_no_trees(name):
    """Any bits, bits of nodes that are not there, rows without any; positions in any order that hide
    part of the cache, all of it (padded queries) or padded tokens of it."""
    lens, nodes, nh, nkv, d, dtype = TREES[name]
    rng = np.random.default_rng(5)
    pos = [rng.permutation(n).astype(np.int32) for n in lens]
    for p in pos:
        p[rng.random(len(p)) < 0.1] = PAD
    cache, host = make_cache(12, lens, [n + 3 for n in lens], nkv, d, dtype, pos)
    x = tree_inputs(22, lens, nodes, nh, nkv, d, dtype, words=3)
    t = len(x["q_pos"])
    x["mask"] = rng.integers(-2**63, 2**63 - 1, size=x["mask"].shape, dtype=np.int64)
    x["mask"][rng.random(t) < 0.3] = 0
    x["q_pos"] = rng.integers(-1, max(lens) + 1, size=t).astype(np.int32)
    x["q_pos"][rng.random(t) < 0.3] = B.CP_POS_PAD_Q
    x["q_pos"][0], x["mask"][0] = B.CP_POS_PAD_Q, 0
    got = run_tree(cache, x, F32, softmax_scale=0.3)
    ref = reference(x, host, scale=0.3)
    assert np.isneginf(ref[1]).any()
    check_tree(got, ref, d, F32, False, name)


def test_tree_wider_than_its_words():
    # nodes that the words have no bit for are seen by none
    cache, host = make_cache(13, [50], [64], 1, 128)
    x = tree_inputs(23, [50], [90], 4, 1, 128, "bf16")
    x["mask"] = np.ascontiguousarray(x["mask"][:, :1])
    check_tree(run_tree(cache, x, F32), reference(x, host), 128, F32, False)


@pytest.mark.parametrize("name", ["chat", "rows", "d64", "d64_few", "fp32", "m_edges", "m_odd_group", "m_d64", "m_d64_seqs"])
def test_hidden_rows_that_are_not_finite(name):
    """What a node does not see does not reach it: bit by bit the same rows with NaN and infinity in
    hidden K and V rows, of the cache, of other nodes, and in the rows of other queries."""
    lens, nodes, nh, nkv, d, dtype = TREES[name]
    cache, host = make_cache(14, lens, [n + 3 for n in lens], nkv, d, dtype)
    x = tree_inputs(24, lens, nodes, nh, nkv, d, dtype)
    t = len(x["q_pos"])
    late = [max(n - 9, 0) for n in lens]         # the last tokens of the cache are hidden from some
    x["q_pos"] = np.where(np.arange(t) % 2 == 0, np.repeat(late, nodes), x["q_pos"]).astype(np.int32)
    odd = np.zeros(t, dtype=bool)
    for b in range(len(lens)):                   # the last node of every tree holds them as well
        if nodes[b] > 2:
            odd[x["cu"][b + 1] - 1] = True
    want = run_tree(cache, x, F32)
    for i, val in enumerate([float("nan"), float("inf"), -float("inf")]):
        for b, n in enumerate(lens):
            if n > 9:
                lo = int(cache.cu_host[b])
                cache.v[lo + n - 1 - i] = val
                cache.k[lo + n - 1 - i] = float("nan")
        x["v"][torch.as_tensor(odd)] = val
        x["k"][torch.as_tensor(odd)] = float("nan")
        x["q"][torch.as_tensor(odd)] = float("nan")
    got = run_tree(cache, x, F32)
    seen_odd = np.zeros(t, dtype=bool)           # rows that see one of them
    for b, n in enumerate(lens):
        q0, q1 = x["cu"][b], x["cu"][b + 1]
        seen_odd[q0:q1] |= (bits(x["mask"][q0:q1], q1 - q0) & odd[q0:q1][None]).any(1)
        if n > 9:
            seen_odd[q0:q1] |= x["q_pos"][q0:q1] >= n - 3
    keep = torch.as_tensor(~(seen_odd | odd)).cuda()
    assert keep.any() and not keep.all()
    for a, b in zip(got, want):
        assert torch.equal(a[keep].view(torch.int32), b[keep].view(torch.int32))


def test_visible_infinite_values():
    # a value that is seen: its sign comes through, both signs or a NaN give NaN; other channels do not care
    cache, host = make_cache(15, [40], [64], 1, 128)
    x = tree_inputs(25, [40], [6], 16, 1, 128, "bf16")
    x["mask"][:] = [[1 << i] for i in range(6)]
    inf = float("inf")
    x["v"][0, 0, 3], x["v"][1, 0, 3], x["v"][2, 0, 3] = inf, -inf, float("nan")
    x["mask"][3] = 3
    o, _ = run_tree(cache, x, F32)
    got = o[:, 0, 3].tolist()
    assert got[0] == inf and got[1] == -inf and np.isnan(got[2]) and np.isnan(got[3])
    assert np.isfinite(got[4]) and np.isfinite(got[5])
    assert torch.isfinite(o[:, :, [0, 1, 2] + list(range(4, 128))]).all()


def test_tree_over_a_ring():
    """Cached tokens sharded over ranks, the trees on one of them: the merge of the ranks' results is
    the attention over everything."""
    n_ranks, lens, nodes, nh, nkv, d = 4, [900, 123], [17, 40], 16, 2, 128
    cache, host = make_cache(16, lens, lens, nkv, d)
    x = tree_inputs(26, lens, nodes, nh, nkv, d, "bf16")
    outs, lses = [], []
    for r in range(n_ranks):
        pos = [B.cp_shard_positions(n, n_ranks, r) for n in lens]
        part = B.KVCache([len(p) + 5 for p in pos], nkv, d)
        idx = np.concatenate([host["cu"][b] + p for b, p in enumerate(pos)])
        B.cp_kv_append(part, cache.k[torch.as_tensor(idx).cuda()].contiguous(),
                       cache.v[torch.as_tensor(idx).cuda()].contiguous(), i32(np.concatenate(pos)),
                       i32(ends([len(p) for p in pos])))
        o, l = run_tree(part, x, F32, own=r == 2)
        outs.append(o)
        lses.append(l)
    got = B.cp_attn_merge(outs, lses, out_dtype=F32)
    check_tree(got, reference(x, host), d, F32, False)


def test_rows_behind_the_last_tree_are_left():
    cache, host = make_cache(17, [20, 30], [32, 32], 1, 128)
    x = tree_inputs(27, [20, 30], [4, 5], 16, 1, 128, "bf16")
    pad = lambda t, n=3: torch.cat([t, torch.zeros((n,) + t.shape[1:], dtype=t.dtype)])
    out = torch.full((12, 16, 128), 7.0, device="cuda")
    lse = torch.full((12, 16), 7.0, device="cuda")
    B.cp_tree_attn(cache, dev(pad(x["q"])), i32(np.append(x["q_pos"], [0, 0, 0])), dev(pad(x["k"])),
                   dev(pad(x["v"])), i32(x["cu"]), dev(pad(torch.as_tensor(x["mask"]))), out=out, lse=lse)
    check_tree((out[:9], lse[:9]), reference(x, host), 128, F32, False)
    assert (out[9:] == 7).all() and (lse[9:] == 7).all()


def test_seq_used_may_be_missing():
    # every slot of the ranges is read then; the unused ones hide behind their positions
    lib = B.load()
    cache, host = make_cache(18, [20, 130], [64, 140], 1, 128)
    x = tree_inputs(28, [20, 130], [4, 9], 16, 1, 128, "bf16")
    q, k, v, m = dev(x["q"]), dev(x["k"]), dev(x["v"]), dev(x["mask"])
    qp, cu = i32(x["q_pos"]), i32(x["cu"])
    out, lse = torch.empty(q.shape, device="cuda"), torch.empty(q.shape[:2], device="cuda")
    s = B.make_shape(B.CP_BF16, 128, 16, 1, 13, cache.slots, 2)
    ws = torch.empty(B.cp_workspace_bytes(s, B.CP_WS_TREE), dtype=torch.uint8, device="cuda")
    rc = lib.cp_tree_attn(ctypes.byref(s), q.data_ptr(), qp.data_ptr(), cu.data_ptr(), k.data_ptr(),
                          v.data_ptr(), m.data_ptr(), 1, cache.k.data_ptr(), cache.v.data_ptr(),
                          cache.kv_pos.data_ptr(), cache.cu.data_ptr(), None, out.data_ptr(),
                          lse.data_ptr(), B.CP_FP32, ws.data_ptr(), ws.numel(),
                          torch.cuda.current_stream().cuda_stream)
    assert rc == 0
    check_tree((out, lse), reference(x, host), 128, F32, False)


# ---------------------------------------------------------------------------

@pytest.mark.parametrize("lens,nodes,room,nkv,d,dtype", [
    ([10, 0, 7], [8, 3, 5], [40, 4, 9], 1, 128, "bf16"),     # one that starts empty, two that overflow
    ([300] * 70, [20] * 70, [340] * 70, 2, 64, "bf16"),
    ([5], [200], [220], 8, 128, "bf16"),
    ([5, 6], [1, 2], [9, 9], 3, 128, "fp32"),
    ([4], [6], [64], 1, 24, "fp32"),
])
def test_accept(lens, nodes, room, nkv, d, dtype):
    cache, host = make_cache(31, lens, room, nkv, d, dtype)
    x = tree_inputs(41, lens, nodes, nkv, nkv, d, dtype)
    rng = np.random.default_rng(3)
    acc = np.array([n - 1 if i % 2 == 0 else rng.integers(-1, n) for i, n in enumerate(nodes)])
    want = {n: host[n].copy() for n in ("k", "v", "kv_pos")}
    used, dropped = list(lens), 0
    for b, a in enumerate(acc):
        if a < 0:
            continue
        q0 = x["cu"][b]
        for t in np.flatnonzero(bits(x["mask"][q0 + a:q0 + a + 1], nodes[b])[0]):
            if used[b] >= room[b]:
                dropped += 1
                continue
            at = host["cu"][b] + used[b]
            want["k"][at], want["v"][at] = x["k64"][q0 + t], x["v64"][q0 + t]
            want["kv_pos"][at] = x["q_pos"][q0 + t]
            used[b] += 1
    B.cp_tree_accept(cache, dev(x["k"]), dev(x["v"]), i32(x["q_pos"]), i32(x["cu"]), dev(x["mask"]), i32(acc))
    assert cache.used.tolist() == used + [0] and cache.dropped.item() == dropped
    assert np.array_equal(cache.k.double().cpu().numpy(), want["k"])
    assert np.array_equal(cache.v.double().cpu().numpy(), want["v"])
    assert np.array_equal(cache.kv_pos.cpu().numpy(), want["kv_pos"])


def test_accept_nothing_and_nodes_that_are_not_there():
    cache, host = make_cache(32, [3, 4, 5], [9, 9, 9], 1, 128)
    x = tree_inputs(42, [3, 4, 5], [2, 3, 4], 1, 1, 128, "bf16")
    before = [t.clone() for t in (cache.k, cache.v, cache.kv_pos, cache.used)]
    B.cp_tree_accept(cache, dev(x["k"]), dev(x["v"]), i32(x["q_pos"]), i32(x["cu"]), dev(x["mask"]),
                     i32([-1, 3, 2**31 - 1]))
    for a, b in zip((cache.k, cache.v, cache.kv_pos, cache.used), before):
        assert torch.equal(a, b)


# ---------------------------------------------------------------------------

WEIGHTS = {
    "step": ([300, 0, 257, 1], [1, 1, 1, 1], 16, 1, 128, "bf16"),
    "many_seqs": ([3 + 7 * (i % 40) for i in range(130)], [1 + i % 2 for i in range(130)], 8, 2, 128, "bf16"),
    "window": ([1000, 700], [40, 3], 16, 1, 128, "bf16"),
    "prompt": ([600], [600], 16, 1, 128, "bf16"),
    "no_queries": ([100, 50], [0, 4], 8, 2, 128, "bf16"),
    "odd_group": ([100, 350], [30, 9], 15, 5, 128, "bf16"),
    "d64": ([800, 33], [64, 33], 8, 8, 64, "bf16"),
    "fp32": ([300, 70], [17, 70], 4, 1, 64, "fp32"),
    "fp32_128": ([300, 70], [17, 70], 6, 2, 128, "fp32"),
}


def weight_inputs(seed, lens, nq, nh, d, dtype):
    rng = np.random.default_rng(seed)
    cu = ends(nq)
    q, q64 = randn(seed, (int(cu[-1]), nh, d), dtype)
    q_pos = np.concatenate([np.arange(n - m, n) for n, m in zip(lens, nq)]).astype(np.int32)
    lse = (np.log(np.maximum(q_pos, 0) + 1.0)[:, None] + rng.normal(size=(len(q_pos), nh))).astype(np.float32)
    return q, q64, q_pos, cu, lse


@pytest.mark.parametrize("decay", [0.0, 0.75, 1.0])
@pytest.mark.parametrize("name", list(WEIGHTS))
def test_attention_weight(name, decay):
    lens, nq, nh, nkv, d, dtype = WEIGHTS[name]
    cache, host = make_cache(51, lens, [n + 2 + i % 5 for i, n in enumerate(lens)], nkv, d, dtype)
    q, q64, q_pos, cu, lse = weight_inputs(61, lens, nq, nh, d, dtype)
    if len(q_pos) > 5:      # queries that see nothing: padded, and of LSE -inf
        q_pos[1], lse[1], lse[3] = B.CP_POS_PAD_Q, -np.inf, -np.inf
    w0 = np.random.default_rng(1).random(cache.slots).astype(np.float32)
    if decay == 0:          # overwritten without being read
        w0[:] = np.nan
    w = dev(w0)
    got = B.cp_kv_attn_weight(cache, dev(q), i32(q_pos), dev(lse), w, i32(cu), decay=decay)
    assert got is w
    want, tol = weight_reference(q64, q_pos, cu, lse, host, w0, decay)
    held = np.zeros(cache.slots, dtype=bool)
    for b, n in enumerate(lens):
        held[host["cu"][b]:host["cu"][b] + n] = True
    got = got.double().cpu().numpy()
    assert np.array_equal(got[~held].view(np.int64), w0.astype(np.float64)[~held].view(np.int64))
    err = np.abs(got - want)[held]
    assert np.all(err <= tol[held] + 1e-30), (err / (tol[held] + 1e-30)).max()


def test_calls_without_any_rows():
    """No queries at all: the weights decay; no nodes: nothing happens; a cache without slots: the tree alone."""
    cache, host = make_cache(53, [40, 7], [64, 9], 1, 128)
    w0 = np.random.default_rng(3).random(cache.slots).astype(np.float32)
    none = torch.empty((0, 16, 128), dtype=BF16, device="cuda")
    for decay in (0.0, 0.5):
        w = dev(w0.copy())
        B.cp_kv_attn_weight(cache, none, i32([]), torch.empty((0, 16), device="cuda"), w, i32([0, 0, 0]), decay=decay)
        want = w0.copy()
        want[:40] *= decay
        want[64:71] *= decay
        assert np.array_equal(w.cpu().numpy(), want)
    kv = torch.empty((0, 1, 128), dtype=BF16, device="cuda")
    m = torch.empty((0, 1), dtype=torch.int64, device="cuda")
    o, l = B.cp_tree_attn(cache, none, i32([]), kv, kv, i32([0, 0, 0]), m, out_dtype=F32)
    assert o.shape == (0, 16, 128) and l.shape == (0, 16)
    used = cache.used.tolist()
    B.cp_tree_accept(cache, kv, kv, i32([]), i32([0, 0, 0]), m, i32([0, 0]))
    assert cache.used.tolist() == used

    x = tree_inputs(55, [40, 7], [3, 2], 16, 1, 128, "bf16")   # rows, but of no tree
    x["cu"] = ends([0, 0])
    out, lse = torch.full((5, 16, 128), 7.0, device="cuda"), torch.full((5, 16), 7.0, device="cuda")
    run_tree(cache, x, F32, out=out, lse=lse)
    assert (out == 7).all() and (lse == 7).all()

    empty = B.KVCache([0, 0], 1, 128)
    x = tree_inputs(54, [0, 0], [40, 3], 16, 1, 128, "bf16")
    host = dict(k=np.zeros((0, 1, 128)), v=np.zeros((0, 1, 128)), kv_pos=np.zeros(0, dtype=np.int32), used=[0, 0], cu=[0, 0, 0])
    check_tree(run_tree(empty, x, F32), reference(x, host), 128, F32, False)
    B.cp_tree_accept(empty, dev(x["k"]), dev(x["v"]), i32(x["q_pos"]), i32(x["cu"]), dev(x["mask"]), i32([5, 2]))
    assert empty.used.tolist() == [0, 0, 0]
    assert empty.dropped.item() == bits(x["mask"][[5]], 40).sum() + bits(x["mask"][[42]], 3).sum()


def test_weights_of_finished_attention_sum_to_one():
    # with the LSE that the attention over the same keys returned, every row weighs 1 in all
    lens, nq, nh = [700, 130], [33, 130], 16
    cache, host = make_cache(52, lens, [n + 4 for n in lens], 1, 128)
    q, _, q_pos, cu, _ = weight_inputs(62, lens, nq, nh, 128, "bf16")
    _, lse = B.cp_tree_attn(cache, dev(q), i32(q_pos), None, None, i32(cu), None, out_dtype=F32)
    w = torch.zeros(cache.slots, device="cuda")
    B.cp_kv_attn_weight(cache, dev(q), i32(q_pos), lse, w, i32(cu))
    for b, n in enumerate(lens):
        total = w[host["cu"][b]:host["cu"][b] + n].double().sum().item()
        assert abs(total - nq[b] * nh) <= nq[b] * nh * 1e-5


def test_weight_keys_that_are_not_finite():
    # a hidden key's NaN reaches no weight, a query's NaN only its own sequence
    lens, nq = [90, 40], [5, 2]
    cache, host = make_cache(53, lens, [96, 48], 2, 128)
    q, _, q_pos, cu, lse = weight_inputs(63, lens, nq, 8, 128, "bf16")
    q_pos[:5] = 60
    w = lambda: torch.zeros(cache.slots, device="cuda")
    want = B.cp_kv_attn_weight(cache, dev(q), i32(q_pos), dev(lse), w(), i32(cu))
    cache.k[70] = float("nan")
    got = B.cp_kv_attn_weight(cache, dev(q), i32(q_pos), dev(lse), w(), i32(cu))
    assert torch.equal(got, want) and got[70] == 0
    q[6] = float("nan")
    got = B.cp_kv_attn_weight(cache, dev(q), i32(q_pos), dev(lse), w(), i32(cu))
    assert torch.equal(got[:96], want[:96]) and torch.isnan(got[96:96 + 39]).all()


# ---------------------------------------------------------------------------

def check_evict(cache, host, w, budget, protect=None, sinks=0, into=None):
    """One eviction against the reference, in place or into another cache."""
    w0 = w.cpu().numpy().copy()
    if into is None:
        want = evict_reference(host, w0, budget, protect, sinks)
        dst, dw = cache, w
    else:
        dst, dst_host = into
        dw = torch.full((dst.slots,), 5.0, device="cuda")
        want = evict_reference(host, w0, budget, protect, sinks, dst_host, dw.cpu().numpy())
    B.cp_kv_evict(cache, w, i32(budget), None if protect is None else i32(protect), sinks,
                  into=None if into is None else dst, into_weight=None if into is None else dw)
    k, v, kp, wt, used = want
    assert dst.used.tolist() == used + [0]
    assert np.array_equal(dst.kv_pos.cpu().numpy(), kp)
    assert np.array_equal(dw.cpu().numpy().view(np.int32), wt.view(np.int32))
    assert np.array_equal(dst.k.double().cpu().numpy(), k)
    assert np.array_equal(dst.v.double().cpu().numpy(), v)
    if into is not None:
        assert cache.used.tolist() == host["used"] + [0]
        assert np.array_equal(cache.kv_pos.cpu().numpy(), host["kv_pos"])
    return want


EVICTS = {     # lens, budgets, KV heads, head_dim, dtype
    "small": ([10, 0, 1, 33, 64], [4, 3, 1, 0, -5], 1, 128, "bf16"),
    "nothing_to_do": ([10, 20], [10, 999], 2, 64, "bf16"),
    "scan_edges": ([1023, 1024, 1025, 2049], [1000, 1, 1024, 2048], 1, 64, "bf16"),
    "one_each": ([700, 1500, 40], [699, 1499, 39], 1, 128, "bf16"),
    "long": ([70000], [5000], 1, 64, "bf16"),
    "long_and_short": ([40000, 3], [39990, 2], 1, 64, "bf16"),
    "chunks": ([90000, 0, 70000, 5, 8192], [50000, 0, 69999, 4, 8000], 1, 8, "bf16"),
    "chunks_one_each": ([66000, 65537], [65999, 65536], 1, 8, "bf16"),
    "fp32": ([100, 50], [30, 49], 3, 24, "fp32"),
}


def weights_like(rng, n, kind):
    if kind == "plain":
        return (rng.random(n) ** 8).astype(np.float32)
    if kind == "ties":       # mostly zeros, and a few values many times
        return rng.choice(np.array([0.0, 0.0, 0.0, 0.5, 1.0, -0.0], dtype=np.float32), n)
    w = rng.normal(size=n).astype(np.float32) * rng.choice([1e-30, 1e-3, 1.0, 1e30], n).astype(np.float32)
    w[rng.random(n) < 0.2] = rng.choice(np.array([np.nan, np.inf, -np.inf, 1e-45], dtype=np.float32))
    return w


@pytest.mark.parametrize("kind", ["plain", "ties", "odd"])
@pytest.mark.parametrize("protect", [False, True])
@pytest.mark.parametrize("name", list(EVICTS))
def test_evict(name, kind, protect):
    lens, budget, nkv, d, dtype = EVICTS[name]
    rng = np.random.default_rng(len(name))
    pos = [rng.permutation(2 * n)[:n].astype(np.int32) for n in lens]
    for p in pos[1:]:
        p[rng.random(len(p)) < 0.05] = PAD
    for into in (False, True):
        cache, host = make_cache(71, lens, [n + 2 + i for i, n in enumerate(lens)], nkv, d, dtype, pos)
        w = weights_like(rng, cache.slots, kind)
        w[host["kv_pos"] == PAD] = 0.25
        w = dev(w)
        keep_from = [2 * n - max(1, n // 10) for n in lens] if protect else None
        dst = None
        if into:
            room = [max(1, b // 2) if i % 3 == 2 else max(b, 0) + 9 for i, b in enumerate(budget)]
            dst = make_cache(81, [min(2, r) for r in room], room, nkv, d, dtype)
        check_evict(cache, host, w, budget, keep_from, 4 if protect else 0, dst)


@pytest.mark.parametrize("lens", [
    [9500 if i % 100 == 7 else 3 + i % 60 for i in range(300)],    # more sequences than CUs, some beyond what LDS holds then
    [25000 + 37 * i for i in range(67)],                           # in chunks, more than 64 sequences
], ids=["many", "many_in_chunks"])
def test_evict_many_sequences(lens):
    budget = [n - n // 3 if i % 2 else n // 5 for i, n in enumerate(lens)]
    rng = np.random.default_rng(4)
    cache, host = make_cache(73, lens, [n + i % 3 for i, n in enumerate(lens)], 1, 8)
    check_evict(cache, host, dev(weights_like(rng, cache.slots, "ties")), budget, [n - 2 for n in lens], 1)


def test_evicting_again_changes_nothing():
    cache, host = make_cache(72, [500, 90], [512, 96], 1, 128)
    w = dev(np.random.default_rng(2).random(cache.slots).astype(np.float32))
    w[500:512] = 0
    w[602:] = 0
    check_evict(cache, host, w, [100, 50])
    before = [t.clone() for t in (cache.k, cache.v, cache.kv_pos, cache.used, w)]
    B.cp_kv_evict(cache, w, i32([100, 50]))
    for a, b in zip((cache.k, cache.v, cache.kv_pos, cache.used, w), before):
        assert torch.equal(a, b)


# ---------------------------------------------------------------------------

def test_offsets_past_31_bits():
    """A cache whose rows lie more than 2^31 elements from its start."""
    nkv, d, first = 16, 128, (1 << 20) + 5000
    cap = [first, 600, 300]
    cache = B.KVCache.__new__(B.KVCache)
    slots = sum(cap)
    cache.batch, cache.slots = 3, slots
    cache.cu_host = ends(cap)
    cache.cu = i32(cache.cu_host)
    cache.k = torch.empty((slots, nkv, d), dtype=BF16, device="cuda")
    cache.v = torch.empty_like(cache.k)
    assert first * nkv * d > 2**31
    cache.kv_pos = torch.full((slots,), PAD, dtype=torch.int32, device="cuda")
    cache.used = i32([0, 500, 200, 0])
    cache.dropped = i32([0])
    lens, nodes = [0, 500, 200], [0, 6, 9]
    small, host = make_cache(91, lens[1:], cap[1:], nkv, d)
    cache.k[first:], cache.v[first:], cache.kv_pos[first:] = small.k, small.v, small.kv_pos
    x = tree_inputs(92, lens, nodes, 32, nkv, d, "bf16")
    for got in (run_tree(cache, x, F32),):
        near = dict(x, cu=x["cu"][1:])
        check_tree(got, tree_reference(x["q64"], x["q_pos"], x["cu"][1:], host, x["k64"], x["v64"], x["mask"]),
                   d, F32, False)
    w, w_small = torch.zeros(slots, device="cuda"), torch.zeros(900, device="cuda")
    lse = got[1]
    B.cp_kv_attn_weight(cache, dev(x["q"]), i32(x["q_pos"]), lse, w, i32(x["cu"]))
    B.cp_kv_attn_weight(small, dev(x["q"]), i32(x["q_pos"]), lse, w_small, i32(x["cu"][1:]))
    assert torch.equal(w[first:], w_small) and not w[:first].any()
    a = (dev(x["k"]), dev(x["v"]), i32(x["q_pos"]))
    B.cp_tree_accept(cache, *a, i32(x["cu"]), dev(x["mask"]), i32([-1, 5, 8]))
    B.cp_tree_accept(small, *a, i32(x["cu"][1:]), dev(x["mask"]), i32([5, 8]))
    B.cp_kv_evict(cache, w, i32([0, 300, 50]))
    B.cp_kv_evict(small, w_small, i32([300, 50]))
    assert torch.equal(cache.k[first:], small.k) and torch.equal(cache.v[first:], small.v)
    assert torch.equal(cache.kv_pos[first:], small.kv_pos) and torch.equal(w[first:], w_small)
    assert cache.used.tolist() == [0] + small.used.tolist()


def steps(cache, w, x, accepted, budget, keep_from, ws=None):
    """A verification step of a serving loop: trees answered, accepted paths kept and weighed, the
    caches cut back to their budget. Everything stays on the device."""
    ws = ws or [None] * 3
    q, q_pos, cu = dev(x["q"]), i32(x["q_pos"]), i32(x["cu"])
    k, v, m, acc = dev(x["k"]), dev(x["v"]), dev(x["mask"]), i32(accepted)
    bud, frm = i32(budget), i32(keep_from)

    def step():
        o, lse = B.cp_tree_attn(cache, q, q_pos, k, v, cu, m, out_dtype=F32, workspace=ws[0])
        B.cp_tree_accept(cache, k, v, q_pos, cu, m, acc)
        B.cp_kv_attn_weight(cache, q, q_pos, lse, w, cu, decay=0.5, workspace=ws[1])
        B.cp_kv_evict(cache, w, bud, protect_from=frm, sinks=2, workspace=ws[2])
        return o, lse
    return step


def test_steps_together():
    """Draft, verify, commit, weigh, evict, several times, each against the reference."""
    lens, nodes, nh, nkv, d = [200, 60, 131], [9, 20, 1], 16, 1, 128
    cap = [n + 40 for n in lens]
    cache, host = make_cache(101, lens, cap, nkv, d)
    w = torch.zeros(cache.slots, device="cuda")
    length = list(lens)
    for it in range(4):
        x = tree_inputs(110 + 10 * it, length, nodes, nh, nkv, d, "bf16")
        acc = [4, 13, 0]
        step = steps(cache, w, x, acc, lens, [n - 5 for n in length])
        w0 = w.cpu().numpy().copy()
        got = step()
        check_tree(got, reference(x, host), d, F32, False, "step %d" % it)
        for b, a in enumerate(acc):             # accepted rows
            q0 = x["cu"][b]
            for t in np.flatnonzero(bits(x["mask"][q0 + a:q0 + a + 1], nodes[b])[0]):
                at = host["cu"][b] + host["used"][b]
                host["k"][at], host["v"][at] = x["k64"][q0 + t], x["v64"][q0 + t]
                host["kv_pos"][at] = x["q_pos"][q0 + t]
                host["used"][b] += 1
        want, tol = weight_reference(x["q64"], x["q_pos"], x["cu"], got[1].cpu().numpy(), host, w0, 0.5)
        # (the weights that the eviction went by: those of the kept slots tell them)
        k2, v2, kp2, w2, used = evict_reference(host, want.astype(np.float32), lens, [n - 5 for n in length], 2)
        assert cache.used.tolist() == used + [0]
        assert np.array_equal(cache.kv_pos.cpu().numpy(), kp2)
        assert np.array_equal(cache.k.double().cpu().numpy()[kp2 != PAD], k2[kp2 != PAD])
        assert np.array_equal(cache.v.double().cpu().numpy()[kp2 != PAD], v2[kp2 != PAD])
        assert np.all(np.abs(w.cpu().numpy() - w2) <= tol.max() + 1e-6 * w2)
        host.update(k=cache.k.double().cpu().numpy(), v=cache.v.double().cpu().numpy(), kv_pos=kp2, used=used)
        length = [n + int(bits(x["mask"][x["cu"][b] + acc[b]][None], nodes[b]).sum())
                  for b, n in enumerate(length)]


def test_steps_in_graphs():
    """Two captured steps, on their own workspaces, replayed in turn with eager work in between: every
    replay gives what the eager step gives from the same state."""
    made = []
    for seed in (121, 131):
        lens, nodes = [300, 90], [12, 5]
        cache, _ = make_cache(seed, lens, [n + 64 for n in lens], 2, 128)
        w = torch.zeros(cache.slots, device="cuda")
        x = tree_inputs(seed + 1, lens, nodes, 16, 2, 128, "bf16")
        s = B.make_shape(B.CP_BF16, 128, 16, 2, 17, cache.slots, 2)
        ws = [torch.empty(B.cp_workspace_bytes(s, kind) + 256, dtype=torch.uint8, device="cuda")
              for kind in (B.CP_WS_TREE, B.CP_WS_WEIGHT, B.CP_WS_EVICT)]
        step = steps(cache, w, x, [7, 3], lens, [n - 8 for n in lens], ws)
        state = [cache.k, cache.v, cache.kv_pos, cache.used, w]
        first = [t.clone() for t in state]

        def restore(state=state, first=first):
            for a, b in zip(state, first):
                a.copy_(b)
        step()                                   # (loads the kernels)
        restore()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = step()
        restore()
        want = []
        for _ in range(3):
            o, l = step()
            want.append([t.clone() for t in (o, l, *state)])
        restore()
        made.append((g, out, state, want, step))   # (the step holds the inputs that the graph reads)
    for i in range(3):
        for g, out, state, want, _ in made:
            g.replay()
            torch.ones(1 << 20, device="cuda").sum()
        torch.cuda.synchronize()
        for g, out, state, want, _ in made:
            for a, b in zip((*out, *state), want[i]):
                assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_another_stream():
    lens, nodes = [900, 400], [30, 11]
    cache, host = make_cache(141, lens, [n + 64 for n in lens], 1, 128)
    x = tree_inputs(142, lens, nodes, 16, 1, 128, "bf16")
    q, k, v, m = dev(x["q"]), dev(x["k"]), dev(x["v"]), dev(x["mask"])   # (they outlive the kernels)
    qp, cu = i32(x["q_pos"]), i32(x["cu"])
    tree = lambda stream=None: B.cp_tree_attn(cache, q, qp, k, v, cu, m, out_dtype=F32, stream=stream)
    want = tree()
    w0 = torch.zeros(cache.slots, device="cuda")
    B.cp_kv_attn_weight(cache, q, qp, want[1], w0, cu)
    side = torch.cuda.Stream()
    for stream in (side, side.cuda_stream):
        w = torch.zeros(cache.slots, device="cuda")
        torch.cuda.synchronize()
        got = tree(stream)
        B.cp_kv_attn_weight(cache, q, qp, want[1], w, cu, stream=stream)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)) and torch.equal(w, w0)
    bud = i32([100, 50])
    torch.cuda.synchronize()
    B.cp_kv_evict(cache, w, bud, stream=side)
    torch.cuda.synchronize()
    assert cache.used.tolist() == [100, 50, 0]


def test_same_inputs_same_bits():
    lens, nodes = [3000, 1700, 40], [40, 64, 3]
    cache, _ = make_cache(151, lens, [n + 64 for n in lens], 1, 128)
    x = tree_inputs(152, lens, nodes, 16, 1, 128, "bf16")
    first = run_tree(cache, x, BF16)
    w = lambda: B.cp_kv_attn_weight(cache, dev(x["q"]), i32(x["q_pos"]), first[1],
                                    torch.zeros(cache.slots, device="cuda"), i32(x["cu"]))
    w0 = w()
    for _ in range(5):
        assert all(torch.equal(a, b) for a, b in zip(run_tree(cache, x, BF16), first))
        assert torch.equal(w(), w0)


def test_trees_of_many_rows_in_a_graph():
    """Replayed with eager calls on the same workspace in between: bit by bit the eager result each time."""
    lens, nodes, nh, nkv, d, dtype = TREES["m_edges"]
    cache, _ = make_cache(161, lens, [n + 64 for n in lens], nkv, d)
    x = tree_inputs(162, lens, nodes, nh, nkv, d, dtype)
    other = tree_inputs(163, lens, nodes, nh, nkv, d, dtype)
    s = B.make_shape(B.CP_BF16, d, nh, nkv, len(x["q_pos"]), cache.slots, len(lens))
    ws = torch.empty(B.cp_workspace_bytes(s, B.CP_WS_TREE), dtype=torch.uint8, device="cuda")
    args = [dev(x["q"]), i32(x["q_pos"]), dev(x["k"]), dev(x["v"]), i32(x["cu"]), dev(x["mask"])]
    want = B.cp_tree_attn(cache, *args, out_dtype=BF16, workspace=ws)
    want = [t.clone() for t in want]
    out, lse = torch.empty_like(want[0]), torch.empty_like(want[1])
    step = lambda: B.cp_tree_attn(cache, *args, out=out, lse=lse, workspace=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(4):
        out.fill_(7), lse.fill_(7)
        run_tree(cache, other, BF16, workspace=ws)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


@pytest.mark.parametrize("seed", range(6))
def test_boundaries_that_contradict_the_shape_stay_inside(seed):
    """Boundaries that fall, overlap or lie outside and counts beyond the room are cut to the tensors: what lies
    around them stays as it was, and sequences that are described rightly get their results."""
    rng = np.random.default_rng(seed)
    nh, nkv, d, slots, t, guard = 16, 1, 128, 900, 40, 64
    cu_kv = [0, 300, 600, 900] + list(rng.integers(-50, 1200, 3))
    cu_q = [0, 10, 25, 40] + list(rng.integers(-20, 80, 3))
    used = [250, 300, 17] + list(rng.integers(-5, 2000, 3)) + [0]
    batch = len(cu_kv) - 1

    def inside(shape, dtype, fill):
        n = shape[0]
        big = torch.full((n + 2 * guard,) + tuple(shape[1:]), fill, dtype=dtype, device="cuda")
        return big, big[guard:guard + n]
    cache = B.KVCache.__new__(B.KVCache)
    cache.batch, cache.slots, cache.cu_host = batch, slots, np.asarray(cu_kv, dtype=np.int32)
    cache.cu, cache.used, cache.dropped = i32(cu_kv), i32(used), i32([0])
    (k_all, cache.k), (v_all, cache.v) = inside((slots, nkv, d), BF16, 3.0), inside((slots, nkv, d), BF16, 5.0)
    pos_all, cache.kv_pos = inside((slots,), torch.int32, 11)
    w_all, w = inside((slots,), F32, 2.0)
    o_all, out = inside((t, nh, d), F32, 7.0)
    l_all, lse = inside((t, nh), F32, 7.0)
    k64, v64 = (np.round(rng.standard_normal((slots, nkv, d)) * 8) / 8 for _ in range(2))
    cache.k.copy_(torch.as_tensor(k64))
    cache.v.copy_(torch.as_tensor(v64))
    kv_pos = np.concatenate([np.arange(300)] * 3).astype(np.int32)
    cache.kv_pos.copy_(torch.as_tensor(kv_pos))
    x = tree_inputs(171, [250, 300, 17], [10, 15, 15], nh, nkv, d, "bf16")
    x["cu"] = np.asarray(cu_q, dtype=np.int32)
    run_tree(cache, x, F32, out=out, lse=lse)
    B.cp_kv_attn_weight(cache, dev(x["q"]), i32(x["q_pos"]), lse, w, i32(x["cu"]))
    B.cp_tree_accept(cache, dev(x["k"]), dev(x["v"]), i32(x["q_pos"]), i32(x["cu"]), dev(x["mask"]),
                     i32([9, 14, 14] + list(rng.integers(-3, 60, 3))))
    into = B.KVCache([100] * batch, nkv, d)
    into_w = torch.zeros(into.slots, device="cuda")
    B.cp_kv_evict(cache, w, i32(rng.integers(-5, 500, batch)), into=into, into_weight=into_w)
    B.cp_kv_evict(cache, w, i32(rng.integers(-5, 500, batch)))
    torch.cuda.synchronize()
    for big, fill in ((k_all, 3), (v_all, 5), (pos_all, 11), (w_all, 2), (o_all, 7), (l_all, 7)):
        assert (big[:guard] == fill).all() and (big[-guard:] == fill).all()


def test_boundaries_that_rise_beside_ones_that_do_not():
    # the first sequences are right: what a later one claims does not change them
    nh, nkv, d = 16, 1, 128
    cache, host = make_cache(172, [250, 280], [300, 300], nkv, d)
    x = tree_inputs(173, [250, 280], [10, 15], nh, nkv, d, "bf16")
    want = run_tree(cache, x, F32)
    cache.batch, cache.cu, cache.used = 3, i32([0, 300, 600, 900]), i32([250, 280, 40, 0])
    x["cu"] = np.append(x["cu"], 70).astype(np.int32)
    got = run_tree(cache, x, F32)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
