"""Values that are not finite in rows that the queries see: of trees of drafted tokens over the KV cache."""
import numpy as np
import pytest
import torch

from gpu_util import dev, i32, randn
from paper_2411_01783_amd import binding as B
from tree_cache_util import bits, check_tree, ends, make_cache, random_parents, tree_reference

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
INF, NAN = float("inf"), float("nan")

# lens, nodes, heads, KV heads, head_dim, dtype: few rows (in one part, in many), many rows (whole, in parts), fp32
SIZES = {
    "few": ([430], [8], 16, 1, 128, "bf16"),
    "few_long": ([9000, 200], [3, 2], 16, 1, 128, "bf16"),
    "few_seqs": ([96 + 5 * (i % 17) for i in range(150)], [1 + i % 3 for i in range(150)], 8, 2, 128, "bf16"),
    "few_d64": ([333, 160, 165], [12, 33, 64], 8, 2, 64, "bf16"),
    "many": ([9991, 133], [61, 16], 16, 1, 128, "bf16"),
    "many_seqs": ([700 + 97 * (i % 17) for i in range(100)], [5 + 5 * (i % 4) for i in range(100)], 8, 2, 128, "bf16"),
    "many_d64": ([7003, 700], [100, 61], 32, 2, 64, "bf16"),
    "fp32": ([200, 333], [5, 33], 4, 1, 64, "fp32"),
    "fp32_128": ([900, 129], [9, 2], 6, 2, 128, "fp32"),
}


def case(name, spread):
    """A cache that every node sees the whole of, the trees and both in 64 bits. spread: one key of every sequence
    has scores hundreds above and below the others', so that their weights do not show in 32 bits."""
    lens, nodes, nh, nkv, d, dtype = SIZES[name]
    cache, host = make_cache(201, lens, [n + 5 for n in lens], nkv, d, dtype)
    if spread:
        for b, n in enumerate(lens):
            at = host["cu"][b] + n - 2
            cache.k[at] *= 128                      # (exact)
            host["k"][at] *= 128
    cu = ends(nodes)
    t = int(cu[-1])
    parents = random_parents(np.random.default_rng(202), nodes)
    q, q64 = randn(203, (t, nh, d), dtype)
    k, k64 = randn(204, (t, nkv, d), dtype)
    v, v64 = randn(205, (t, nkv, d), dtype)
    x = dict(q=q, k=k, v=v, q64=q64, k64=k64, v64=v64, cu=cu, mask=B.cp_tree_mask(parents, cu),
             q_pos=np.repeat(np.asarray(lens), nodes).astype(np.int32))
    return cache, host, x


# channel -> (offset of the cached slot that holds it from the sequence's start, value); all of them in sub-tiles
# that the rows see the whole of
CACHED = {3: [(40, INF)], 5: [(41, -INF)], 7: [(70, INF), (45, -INF)], 9: [(64, NAN)], 20: [(33, INF), (90, INF)]}
WANT = {3: INF, 5: -INF, 7: NAN, 9: NAN, 20: INF}
OWN = 30                                          # a channel that the trees' first nodes have an infinity in


@pytest.mark.parametrize("spread", [False, True], ids=["near", "spread"])
@pytest.mark.parametrize("out_dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("name", list(SIZES))
def test_visible_values_that_are_not_finite(name, out_dtype, spread):
    """Infinity comes through with its sign, both signs and a NaN as NaN, whatever else the sub-tile holds and
    however small the weight; the other channels and the LSE are those of finite values."""
    lens, nodes, nh, nkv, d, dtype = SIZES[name]
    cache, host, x = case(name, spread)
    odd = list(CACHED) + [OWN]
    host["v"][:, 0, odd], x["v64"][:, 0, odd] = 0, 0
    ref = tree_reference(x["q64"], x["q_pos"], x["cu"], host, x["k64"], x["v64"], x["mask"])
    for b in range(len(lens)):
        for c, places in CACHED.items():
            for off, val in places:
                cache.v[int(host["cu"][b]) + off, 0, c] = val
        x["v"][x["cu"][b], 0, OWN] = -INF
    o, lse = B.cp_tree_attn(cache, dev(x["q"]), i32(x["q_pos"]), dev(x["k"]), dev(x["v"]), i32(x["cu"]),
                            dev(x["mask"]), out_dtype=out_dtype)
    group = nh // nkv
    for c, val in WANT.items():
        got = o[:, :group, c].float()
        assert (torch.isnan(got) if val != val else got == val).all(), "channel %d" % c
    first = np.concatenate([bits(x["mask"][x["cu"][b]:x["cu"][b + 1]], 1)[:, 0] for b in range(len(lens))])
    first = torch.as_tensor(first).cuda()
    assert (o[first, :group, OWN] == -INF).all() and torch.isfinite(o[~first, :group, OWN]).all()
    o = o.clone()
    o[:, :group, odd] = 0
    for part in (ref[0], ref[2]):
        part[:, :group, odd] = 0
    check_tree((o, lse), ref, d, out_dtype, dtype == "bf16" and out_dtype == BF16, name)


@pytest.mark.parametrize("name", ["few", "few_long", "many", "many_d64", "fp32"])
def test_visible_infinities_without_the_trees(name):
    """The same on a rank that does not hold the trees."""
    lens, nodes, nh, nkv, d, dtype = SIZES[name]
    cache, host, x = case(name, True)
    for b in range(len(lens)):
        cache.v[int(host["cu"][b]) + 40, 0, 3] = INF
    o, lse = B.cp_tree_attn(cache, dev(x["q"]), i32(x["q_pos"]), None, None, i32(x["cu"]), None, out_dtype=F32)
    group = nh // nkv
    assert (o[:, :group, 3] == INF).all() and torch.isfinite(lse).all()
    o[:, :group, 3] = 0
    assert torch.isfinite(o).all()
