"""Trees of drafted tokens at sizes near the limits of the card."""
import numpy as np
import pytest
import torch

from gpu_util import i32, randn
from paper_2411_01783_amd import binding as B
from tree_cache_util import check_tree, make_cache, tree_reference

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def test_more_rows_than_a_grid_dimension_has_wavefronts():
    """2^20 nodes of 64 heads, nearly all of a sequence that has nothing cached: the last sequence's rows, which lie
    in several parts, are merged like the first ones."""
    nh, d, t = 64, 64, (1 << 20) + 5
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("18 GB of tensors")
    lens = [3000, 0, 75000]
    cache, host = make_cache(501, lens, [3010, 4, 75008], 1, d)
    cu = np.array([0, 3, t - 2, t], dtype=np.int32)
    some = np.array([0, 1, 2, t - 2, t - 1])
    q_some, q64 = randn(502, (5, nh, d), "bf16")
    q = torch.zeros((t, nh, d), dtype=BF16, device="cuda")
    q[torch.as_tensor(some).cuda()] = q_some.cuda()
    q_pos = torch.full((t,), 80000, dtype=torch.int32, device="cuda")
    out = torch.full((t, nh, d), 7.0, dtype=BF16, device="cuda")
    lse = torch.full((t, nh), 7.0, device="cuda")
    B.cp_tree_attn(cache, q, q_pos, None, None, i32(cu), None, out=out, lse=lse)
    at = torch.as_tensor(some).cuda()
    ref = tree_reference(q64, np.full(5, 80000), np.array([0, 3, 3, 5]), host)
    check_tree((out[at], lse[at]), ref, d, BF16, False)
    assert torch.isneginf(lse[3:-2]).all()
    for part in out[3:-2].split(1 << 17):
        assert not part.any()
