"""Trees of drafted tokens whose probabilities keep 24 bits: the bound on O has no rounding of P to bf16 in it."""
import numpy as np
import pytest
import torch

from gpu_util import dev, i32, randn
from paper_2411_01783_amd import binding as B
from tree_cache_util import check_tree, ends, make_cache, random_parents, tree_reference

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("own", [True, False], ids=["own", "cached"])
@pytest.mark.parametrize("lens,nodes,nh,nkv,d,out_dtype", [
    ([333, 64, 1265], [12, 33, 64], 8, 2, 64, BF16),       # few rows
    ([7003, 700], [100, 61], 32, 2, 64, BF16),             # many
    ([7003, 700], [100, 61], 32, 2, 64, F32),
    ([700, 90], [130, 65], 8, 2, 128, F32),
    ([9991, 33], [61, 16], 16, 1, 128, F32),
], ids=["d64_few", "d64_many", "d64_many_fp32", "d128_few_fp32", "d128_many_fp32"])
def test_probabilities_keep_24_bits(lens, nodes, nh, nkv, d, out_dtype, own):
    cache, host = make_cache(401, lens, [n + 9 for n in lens], nkv, d)
    cu = ends(nodes)
    t = int(cu[-1])
    q, q64 = randn(402, (t, nh, d), "bf16")
    k, k64 = randn(403, (t, nkv, d), "bf16")
    v, v64 = randn(404, (t, nkv, d), "bf16")
    mask = B.cp_tree_mask(random_parents(np.random.default_rng(405), nodes), cu)
    q_pos = np.repeat(np.asarray(lens), nodes).astype(np.int32)
    new = (dev(k), dev(v), dev(mask)) if own else (None,) * 3
    got = B.cp_tree_attn(cache, dev(q), i32(q_pos), new[0], new[1], i32(cu), new[2], out_dtype=out_dtype)
    ref = tree_reference(q64, q_pos, cu, host, *((k64, v64, mask) if own else (None,) * 3))
    check_tree(got, ref, d, out_dtype, False)
