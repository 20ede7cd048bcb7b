"""Attention weight of cached keys that are not finite, and of queries that weigh nothing."""
import numpy as np
import pytest
import torch

from gpu_util import dev, i32, randn
from paper_2411_01783_amd import binding as B
from tree_cache_util import ends, make_cache, weight_reference

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")

# lens, queries, heads, KV heads, head_dim, dtype: rows (queries times a KV head's heads) that fill no tile of 64, that
# fill one, that are more than several
SIZES = {
    "one": ([300], [1], 16, 1, 128, "bf16"),
    "tile": ([300], [4], 16, 1, 128, "bf16"),
    "more": ([300, 90], [21, 5], 16, 1, 128, "bf16"),
    "heads": ([260, 400], [3, 37], 8, 2, 128, "bf16"),
    "d64": ([333], [13], 15, 5, 64, "bf16"),
    "fp32": ([150, 70], [9, 2], 4, 1, 64, "fp32"),
}


def case(name):
    lens, nq, nh, nkv, d, dtype = SIZES[name]
    cache, host = make_cache(301, lens, [n + 3 for n in lens], nkv, d, dtype)
    cu = ends(nq)
    q, q64 = randn(302, (int(cu[-1]), nh, d), dtype)
    q_pos = np.repeat(np.asarray(lens), nq).astype(np.int32)      # every query sees every key
    lse = (np.log(q_pos + 1.0)[:, None] + np.random.default_rng(303).normal(size=(len(q_pos), nh))).astype(np.float32)
    w0 = np.random.default_rng(304).random(cache.slots).astype(np.float32)
    return cache, host, q, q64, q_pos, cu, lse, w0


def check(got, want, tol, host, skip=()):
    held = np.zeros(len(want), dtype=bool)
    for b, n in enumerate(host["used"]):
        held[host["cu"][b]:host["cu"][b] + n] = True
    held[list(skip)] = False
    err = np.abs(got.double().cpu().numpy() - want)[held]
    assert np.all(err <= tol[held] + 1e-30), (err / (tol[held] + 1e-30)).max()


@pytest.mark.parametrize("name", list(SIZES))
def test_visible_keys_that_are_not_finite(name):
    """A key with an infinite channel has scores of minus infinity, of which nothing comes, or of plus infinity,
    whatever number of rows the tiles are filled up with; the keys beside it keep their weight."""
    cache, host, q, q64, q_pos, cu, lse, w0 = case(name)
    q[:, :, 2] = -(q[:, :, 2].abs() + 1)
    q64[:, :, 2] = q[:, :, 2].double().numpy()
    last = host["cu"][-2]
    low, high, both = 40, 41, int(last) + 50
    host["k"][[low, high, both]] = 0
    cache.k[low, :, 2], cache.k[high, :, 2] = INF, -INF
    cache.k[both] = INF                            # (scores of both signs' infinities: a NaN)
    w = dev(w0)
    got = B.cp_kv_attn_weight(cache, dev(q), i32(q_pos), dev(lse), w, i32(cu), decay=0.5)
    want, tol = weight_reference(q64, q_pos, cu, lse, host, w0, 0.5)
    assert got[low].item() == 0.5 * w0[low]
    assert got[high].item() == INF and torch.isnan(got[both])
    check(got, want, tol, host, (low, high, both))


@pytest.mark.parametrize("name", [n for n in SIZES if n != "one"])
def test_queries_that_weigh_nothing_may_hold_anything(name):
    """A query of LSE = -inf weighs nothing, its Q not finite and its position behind every key's."""
    cache, host, q, q64, q_pos, cu, lse, w0 = case(name)
    for i, val in ((1, NAN), (len(q_pos) - 1, INF)):
        lse[i] = -np.inf
        q[i], q64[i] = val, 0
    got = B.cp_kv_attn_weight(cache, dev(q), i32(q_pos), dev(lse), dev(w0), i32(cu))
    want, tol = weight_reference(q64, q_pos, cu, lse, host, w0, 1.0)
    check(got, want, tol, host)
