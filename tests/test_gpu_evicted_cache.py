"""The attention calls on a cache after an eviction: slots are no longer in the order of positions, and those behind
the kept tokens hold what was there. Each against 64-bit attention over what the cache says that it holds."""
import numpy as np
import pytest
import torch

from gpu_util import LSE_RTOL_FP32, O_ATOL_FP32, check, dev, i32, randn
from paper_2411_01783_amd import binding as B
from tree_cache_util import ends, make_cache, tree_reference

pytestmark = pytest.mark.gpu
F32 = torch.float32
LENS, BUDGET = [900, 300, 77, 2100], [501, 300, 10, 640]


def evicted(seed, nkv, d, dtype="bf16", into=False, pos=None):
    """A cache cut down to BUDGET by weights that put the kept tokens anywhere, and its host copy."""
    cache, _ = make_cache(seed, LENS, [n + 20 for n in LENS], nkv, d, dtype, pos)
    w = dev(np.random.default_rng(seed).random(cache.slots).astype(np.float32))
    last = [int(p.max()) if pos is not None else n - 1 for n, p in zip(LENS, pos or LENS)]
    to = B.KVCache([b + 7 for b in BUDGET], nkv, d, dtype=cache.k.dtype) if into else None
    w_to = torch.zeros(to.slots, device="cuda") if into else None
    B.cp_kv_evict(cache, w, i32(BUDGET), protect_from=i32([x - 3 for x in last]), sinks=2, into=to, into_weight=w_to)
    return to if into else cache


def host_of(cache):
    return dict(k=cache.k.double().cpu().numpy(), v=cache.v.double().cpu().numpy(), kv_pos=cache.kv_pos.cpu().numpy(),
                used=cache.used.tolist()[:-1], cu=cache.cu_host.copy())


def test_the_order_is_not_that_of_positions():
    host = host_of(evicted(601, 1, 128))
    kept = host["kv_pos"][:BUDGET[0]]
    assert host["used"] == BUDGET and (np.diff(kept) < 0).any() and len(set(kept.tolist())) == BUDGET[0]


@pytest.mark.parametrize("into", [False, True], ids=["in_place", "into"])
@pytest.mark.parametrize("call", ["decode", "unique", "static"])
def test_decode(call, into):
    nh, nkv, d = 16, 1, 128
    cache = evicted(611, nkv, d, into=into)
    for step in range(2):                         # the second step behind an append
        host = host_of(cache)
        q, q64 = randn(612 + step, (4, nh, d), "bf16")
        q_pos = [n + step for n in LENS]
        q_pos[3] = 1000                           # (one that does not see all that was kept)
        a = (dev(q), cache.k, cache.v, i32(q_pos), cache.kv_pos, cache.cu, i32([0, 1, 2, 3]))
        if call == "static":
            out, lse = torch.empty(q.shape, dtype=F32, device="cuda"), torch.empty((4, nh), device="cuda")
            B.cp_attn_decode_static(*a, out, lse)
        else:
            out, lse = B.cp_attn_decode(*a, out_dtype=F32, unique_bid=call == "unique")
        o, l = tree_reference(q64, q_pos, np.arange(5), host)[:2]
        check(out, lse, o, l, what="%s, step %d" % (call, step))
        k, _ = randn(622 + step, (4, nkv, d), "bf16")
        v, _ = randn(632 + step, (4, nkv, d), "bf16")
        B.cp_kv_append(cache, dev(k), dev(v), i32(LENS), i32([0, 1, 2, 3, 4]))


@pytest.mark.parametrize("nq", [[3, 40, 1, 9], [64, 300, 77, 512]], ids=["few", "many"])
@pytest.mark.parametrize("nh,nkv,d,dtype", [(16, 1, 128, "bf16"), (8, 2, 64, "bf16"), (4, 1, 64, "fp32")],
                         ids=["bf16", "d64", "fp32"])
def test_partial(nh, nkv, d, dtype, nq):
    cache = evicted(641, nkv, d, dtype)
    host = host_of(cache)
    cu = ends(nq)
    q, q64 = randn(642, (int(cu[-1]), nh, d), dtype)
    rng = np.random.default_rng(643)
    q_pos = np.concatenate([np.sort(rng.integers(0, n, m)) for n, m in zip(LENS, nq)]).astype(np.int32)
    o, l = tree_reference(q64, q_pos, cu, host)[:2]
    tol = {} if dtype == "bf16" else dict(o_atol=O_ATOL_FP32, lse_rtol=LSE_RTOL_FP32)
    out, lse = B.cp_attn_partial(dev(q), cache.k, cache.v, i32(q_pos), cache.kv_pos, i32(cu), cache.cu, out_dtype=F32)
    check(out, lse, o, l, what="packed", **tol)
    for b in range(4):                            # a sequence's range by itself
        at = slice(cu[b], cu[b + 1])
        out, lse = B.cp_attn_partial(dev(q[at]), *cache.segment(b)[:2], i32(q_pos[at]), cache.segment(b)[2],
                                     out_dtype=F32)
        check(out, lse, o[at], l[at], what="sequence %d" % b, **tol)


def ranks_of(seed, n, nkv, d):
    """Evicted caches of n ranks, rank r with the positions r, r + n, ... of every sequence."""
    return [evicted(seed + r, nkv, d, pos=[np.arange(m, dtype=np.int32) * n + r for m in LENS]) for r in range(n)]


def all_ranks(caches):
    """What all ranks hold, as one host cache."""
    hosts = [host_of(c) for c in caches]
    seqs = [[(h["cu"][b], h["cu"][b] + h["used"][b]) for h in hosts] for b in range(len(LENS))]
    join = lambda name: np.concatenate([h[name][lo:hi] for s in seqs for h, (lo, hi) in zip(hosts, s)])
    used = [sum(hi - lo for lo, hi in s) for s in seqs]
    return dict(k=join("k"), v=join("v"), kv_pos=join("kv_pos"), used=used, cu=ends(used))


def test_ring_decode():
    n, nh, nkv, d = 3, 16, 1, 128
    caches = ranks_of(651, n, nkv, d)
    host = all_ranks(caches)
    bids = [[0, 3], [1], [2]]
    pos = [n * m for m in LENS]
    q, q64 = randn(661, (4, nh, d), "bf16")
    ring = B.Ring([dev(q[b]) for b in bids], [c.k for c in caches], [c.v for c in caches],
                  [i32([pos[b] for b in bs]) for bs in bids], [c.kv_pos for c in caches], out_dtype=F32,
                  cu_seqlens_kv=[c.cu for c in caches], bid=[i32(bs) for bs in bids])
    out, lse = B.cp_ring_passq_decode(ring)
    o, l = tree_reference(q64, pos, np.arange(5), host)[:2]
    for r, bs in enumerate(bids):
        check(out[r], lse[r], o[bs], l[bs], what="rank %d" % r)


@pytest.mark.parametrize("order", [B.cp_ring_passkv, B.cp_ring_passq], ids=["passkv", "passq"])
@pytest.mark.parametrize("b", range(4))
def test_ring_prefill(order, b):
    """A turn's new queries on every rank's range of one sequence."""
    n, nh, nkv, d, t_new = 3, 16, 1, 128, 210
    caches = ranks_of(671, n, nkv, d)
    host = all_ranks(caches)
    q, q64 = randn(681, (t_new, nh, d), "bf16")
    pos = [B.cp_shard_positions(t_new, n, r, offset=n * LENS[b]) for r in range(n)]
    idx = [p - n * LENS[b] for p in pos]
    seg = [c.segment(b) for c in caches]
    ring = B.Ring([dev(q[torch.as_tensor(i)]) for i in idx], [s[0] for s in seg], [s[1] for s in seg], [i32(p) for p in pos],
                  [s[2] for s in seg], out_dtype=F32)
    out, lse = order(ring)
    one = {k: host[k] for k in ("k", "v", "kv_pos")}
    lo, hi = host["cu"][b], host["cu"][b + 1]
    one = dict({k: x[lo:hi] for k, x in one.items()}, used=[hi - lo], cu=[0, hi - lo])
    for r in range(n):
        o, l = tree_reference(q64[idx[r]], pos[r], [0, len(pos[r])], one)[:2]
        check(out[r], lse[r], o, l, what="rank %d" % r)
