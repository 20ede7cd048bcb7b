"""Plain 64-bit forms of the calls on the KV cache (trees of drafted tokens, attention weight,
eviction), and how far fp32 and bf16 arithmetic may be from them."""
import numpy as np
import torch

from gpu_util import dev, i32, randn
from paper_2411_01783_amd import binding as B

PAD = B.CP_POS_PAD_KV
U32 = 2.0 ** -24                                      # half a step of fp32, of bf16
U16 = torch.finfo(torch.bfloat16).eps / 2


def ends(counts):
    return np.concatenate([[0], np.cumsum(np.asarray(counts, dtype=np.int64))]).astype(np.int32)


def make_cache(seed, lens, capacity, nkv, d, dtype="bf16", pos=None):
    """A KVCache whose sequences hold lens[b] tokens at positions 0 .. (or pos[b]), and its host copies."""
    cache = B.KVCache(capacity, nkv, d, dtype=torch.bfloat16 if dtype == "bf16" else torch.float32)
    slots = cache.slots
    k, k64 = randn(seed, (slots, nkv, d), dtype)
    v, v64 = randn(seed + 1, (slots, nkv, d), dtype)
    kp = np.full(slots, PAD, dtype=np.int32)
    for b, n in enumerate(lens):
        lo = cache.cu_host[b]
        kp[lo:lo + n] = np.arange(n) if pos is None else pos[b]
    free = torch.as_tensor(kp == PAD)
    k[free], v[free] = 0, 0
    k64[free.numpy()], v64[free.numpy()] = 0, 0
    cache.k.copy_(k)
    cache.v.copy_(v)
    cache.kv_pos.copy_(torch.as_tensor(kp))
    cache.used.copy_(torch.as_tensor(np.asarray(list(lens) + [0], dtype=np.int32)))
    return cache, dict(k=k64, v=v64, kv_pos=kp, used=list(lens), cu=cache.cu_host.copy())


def random_parents(rng, nodes):
    return np.concatenate([[rng.integers(-1, i) if i and rng.random() < 0.5 else i - 1
                            for i in range(n)] for n in nodes] + [[]]).astype(np.int32)


def bits(mask, n):
    """[rows, words] of int64 as [rows, n] of bool."""
    m = np.ascontiguousarray(mask).view(np.uint64)
    cols = [(m[:, t // 64] >> np.uint64(t % 64)) & np.uint64(1) if t // 64 < m.shape[1]
            else np.zeros(m.shape[0], dtype=np.uint64) for t in range(n)]
    return np.stack(cols, 1).astype(bool) if n else np.zeros((m.shape[0], 0), dtype=bool)


def tree_reference(q, q_pos, cu_q, host, k_new=None, v_new=None, mask=None, scale=None):
    """O and LSE in 64 bits, and per row the bounds that the tolerances are made of: a = softmax-weighted
    |v| per channel, s = the largest sum of |q c||k c| over its keys, n = the number of its keys."""
    t, nh, d = q.shape
    nkv = host["k"].shape[1]
    scale = 1 / np.sqrt(d) if scale is None else scale
    o, lse = np.zeros((t, nh, d)), np.full((t, nh), -np.inf)
    a, big, cnt = np.zeros((t, nh, d)), np.zeros((t, nh)), np.zeros((t, nh))
    for b in range(len(cu_q) - 1):
        q0, q1, k0 = cu_q[b], cu_q[b + 1], host["cu"][b]
        n = host["used"][b]
        if q1 == q0:
            continue
        see = host["kv_pos"][None, k0:k0 + n] <= np.asarray(q_pos)[q0:q1, None]
        kk, vv = host["k"][k0:k0 + n], host["v"][k0:k0 + n]
        if k_new is not None:
            see = np.concatenate([see, bits(mask[q0:q1], q1 - q0)], 1)
            kk, vv = np.concatenate([kk, k_new[q0:q1]]), np.concatenate([vv, v_new[q0:q1]])
        for h in range(nh):
            kh, vh = kk[:, h * nkv // nh], vv[:, h * nkv // nh]
            with np.errstate(invalid="ignore"):
                s = np.where(see, scale * (q[q0:q1, h] @ kh.T), -np.inf)
            if not s.shape[1]:
                continue
            top = s.max(1, keepdims=True)
            e = np.exp(s - np.where(np.isfinite(top), top, 0))
            total = e.sum(1, keepdims=True)
            with np.errstate(divide="ignore", invalid="ignore"):
                p = np.where(total > 0, e / total, 0)
                lse[q0:q1, h] = np.where(total[:, 0] > 0, top[:, 0] + np.log(total[:, 0]), -np.inf)
            o[q0:q1, h], a[q0:q1, h] = p @ vh, p @ np.abs(vh)
            big[q0:q1, h] = (np.where(see, np.abs(q[q0:q1, h]) @ np.abs(kh).T, 0)).max(1) * scale
            cnt[q0:q1, h] = see.sum(1)
    return o, lse, a, big, cnt


def check_tree(got, ref, d, out_dtype, p_bits16, what=""):
    """Worst case of fp32 arithmetic: a score is a sum of d products, scaled (d + 3 roundings of at
    most its absolute sum), a probability the exponential of the difference of two (with two roundings
    and 2^-22 of the hardware's exp2, log2), sums of n terms lose n roundings. P rounded to bf16 (one
    term) adds half a bf16 step of every term, the output half a step of its own type."""
    o, lse, a, big, cnt = ref
    go, gl = got[0].double().cpu().numpy(), got[1].double().cpu().numpy()
    assert go.shape == o.shape and gl.shape == lse.shape, what
    empty = np.isneginf(lse)
    assert np.array_equal(np.isneginf(gl), empty), what + ": which rows are empty"
    assert np.all(go[empty] == 0), what + ": empty rows are zero"
    ds = (d + 3) * U32 * big + 2.0 ** -22
    rel = 2 * ds + (2 * cnt + 40) * U32 + (U16 if p_bits16 else U32)
    tol = a * rel[..., None] + np.abs(o) * (U16 if out_dtype == torch.bfloat16 else U32) * (1 + 2e-2)
    err = np.abs(go - o)
    assert np.all(err <= tol + 1e-30), "%s: O off by %.3g of its bound" % (what, (err / (tol + 1e-30)).max())
    fin = ~empty
    tol_l = ds + (cnt + 40) * U32 + 4 * U32 * np.abs(np.where(fin, lse, 0)) + 2.0 ** -22
    err_l = np.abs(np.where(fin, gl, 0) - np.where(fin, lse, 0))
    assert np.all(err_l <= tol_l), "%s: LSE off by %.3g of its bound" % (what, (err_l / tol_l).max())


def weight_reference(q, q_pos, cu_q, lse, host, weight, decay, scale=None):
    """The weights in 64 bits, and how far fp32 arithmetic may be off: every term by its exponent's
    error (as above, and the LSE scaled: two roundings of it), the sum of n terms by n roundings."""
    t, nh, d = q.shape
    nkv = host["k"].shape[1]
    scale = 1 / np.sqrt(d) if scale is None else scale
    w, tol = weight.astype(np.float64).copy(), np.zeros(len(weight))
    for b in range(len(cu_q) - 1):
        q0, q1, k0, n = cu_q[b], cu_q[b + 1], host["cu"][b], host["used"][b]
        seg = slice(k0, k0 + n)
        w[seg] = w[seg] * decay if decay else 0.0
        tol[seg] += 2 * U32 * np.abs(w[seg])
        see = host["kv_pos"][seg][None] <= np.asarray(q_pos)[q0:q1, None]
        for h in range(nh):
            kh, l = host["k"][seg, h * nkv // nh], lse[q0:q1, h].astype(np.float64)
            ok = see & np.isfinite(l)[:, None]
            with np.errstate(invalid="ignore", over="ignore"):
                p = np.where(ok, np.exp(scale * (q[q0:q1, h] @ kh.T) - l[:, None]), 0.0)
            big = scale * (np.abs(q[q0:q1, h]) @ np.abs(kh).T)
            rel = (d + 3) * U32 * big + 3 * U32 * np.abs(np.where(np.isfinite(l), l, 0))[:, None] + 2.0 ** -22
            w[seg] += p.sum(0)
            tol[seg] += (p * (rel + ((q1 - q0) * nh + 8) * U32)).sum(0)
    return w, tol


def evict_reference(host, weight, budget, protect_from, sinks, to=None, to_weight=None):
    """(k, v, kv_pos, weight, used) after the eviction; exact (rows are copied)."""
    d = host if to is None else to
    k, v, kp, w = d["k"].copy(), d["v"].copy(), d["kv_pos"].copy(), \
        (weight if to is None else to_weight).copy()
    used = []
    for b, n in enumerate(host["used"]):
        k0, d0, cap = host["cu"][b], d["cu"][b], d["cu"][b + 1] - d["cu"][b]
        pos, wt = host["kv_pos"][k0:k0 + n], weight[k0:k0 + n].astype(np.float64)
        safe = (pos < sinks) & (pos != PAD)
        if protect_from is not None:
            safe |= (pos >= protect_from[b]) & (pos != PAD)
        rank = np.where(np.isnan(wt), -np.inf, wt)
        nan = np.isnan(wt) & ~safe
        keep = int(min(n, cap, max(budget[b], safe.sum(), 0)))
        order = sorted(range(n), key=lambda i: (not safe[i], nan[i], 0.0 if safe[i] else -rank[i], i))
        stays = np.zeros(n, dtype=bool)
        stays[order[:keep]] = True
        movers = iter(np.flatnonzero(stays[keep:]) + keep)
        src = [i if stays[i] else int(next(movers)) for i in range(keep)]
        for name, arr in (("k", k), ("v", v), ("kv_pos", kp)):
            arr[d0:d0 + keep] = host[name][k0 + np.asarray(src, dtype=np.int64)]
        w[d0:d0 + keep] = weight[k0 + np.asarray(src, dtype=np.int64)]
        behind = slice(d0 + keep, d0 + (cap if to is not None else n))
        kp[behind], w[behind] = PAD, 0.0
        used.append(keep)
    return k, v, kp, w, used
