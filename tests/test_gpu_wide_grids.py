"""Attention on the vector pipe at sizes whose workgroups pass one grid dimension."""
import numpy as np
import pytest
import torch

from gpu_util import check, i32, randn
from paper_2411_01783_amd import binding as B
from tree_cache_util import make_cache, tree_reference

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def test_partial_of_more_rows_than_a_grid_dimension_has_wavefronts():
    """2^20 packed queries of 64 heads of 64, nearly all of a sequence without keys: the last sequence's rows are
    computed like the first ones."""
    nh, d, t = 64, 64, (1 << 20) + 5
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("18 GB of tensors")
    lens = [300, 0, 500]
    cache, host = make_cache(511, lens, lens, 1, d)
    some = np.array([0, 1, 2, t - 2, t - 1])
    at = torch.as_tensor(some).cuda()
    q_some, q64 = randn(512, (5, nh, d), "bf16")
    q = torch.zeros((t, nh, d), dtype=BF16, device="cuda")
    q[at] = q_some.cuda()
    q_pos = torch.full((t,), 1000, dtype=torch.int32, device="cuda")
    out = torch.full((t, nh, d), 7.0, dtype=BF16, device="cuda")
    lse = torch.full((t, nh), 7.0, device="cuda")
    B.cp_attn_partial(q, cache.k, cache.v, q_pos, cache.kv_pos, i32([0, 3, t - 2, t]), cache.cu, out=out, lse=lse)
    o, l = tree_reference(q64, np.full(5, 1000), np.array([0, 3, 3, 5]), host)[:2]
    check(out[at], lse[at], o, l)
    assert torch.isneginf(lse[3:-2]).all()
    for part in out[3:-2].split(1 << 17):
        assert not part.any()
