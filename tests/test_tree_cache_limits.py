"""Sizes at which the calls on the KV cache are refused, without a GPU."""
import ctypes

import numpy as np
import pytest

from paper_2411_01783_amd import binding as B

ONE = ctypes.c_void_p(256)    # never dereferenced: the calls below fail validation first
SHAPE, WORKSPACE = -2, -4


def shape(**kw):
    a = dict(dtype=B.CP_BF16, head_dim=128, n_q_heads=16, n_kv_heads=2, total_q=8, total_kv=64, batch=2)
    a.update(kw)
    return B.make_shape(**a)


def accept(s):
    return B.load().cp_tree_accept(ctypes.byref(s), ONE, ONE, ONE, ONE, ONE, 1, ONE, ONE, ONE, ONE, ONE, ONE, None,
                                   None)


def test_paths_of_more_sequences_than_a_grid_holds():
    assert accept(shape(batch=2**23)) == SHAPE
    assert accept(shape(batch=2**31 - 1)) == SHAPE
    assert accept(shape(batch=2**23 - 1, total_q=0)) == 0


def tree(s):
    return B.load().cp_tree_attn(ctypes.byref(s), ONE, ONE, ONE, ONE, ONE, ONE, 1, ONE, ONE, ONE, ONE, ONE, ONE, ONE, 0,
                                 ONE, ctypes.c_size_t(1 << 62), None)


def weight(s):
    return B.load().cp_kv_attn_weight(ctypes.byref(s), ONE, ONE, ONE, ONE, ONE, ONE, ONE, ONE, 1.0, ONE, ONE,
                                      ctypes.c_size_t(1 << 62), None)


def test_batches_that_a_walk_would_not_end_in():
    for batch in (65536, 2**24, 2**31 - 1):
        assert tree(shape(batch=batch)) == SHAPE
        assert weight(shape(batch=batch)) == SHAPE
    assert tree(shape(batch=65535, total_q=0)) == 0
    assert weight(shape(batch=65535, total_kv=0)) == 0


def evict(s, slots_to=None):
    to = [None] * 6 + [0] if slots_to is None else [ctypes.c_void_p(4096)] * 6 + [slots_to]
    return B.load().cp_kv_evict(ctypes.byref(s), ONE, ONE, ONE, ONE, ONE, ONE, ONE, None, 0, *to, None, ctypes.c_size_t(0),
                                None)


def test_evictions_whose_slots_pass_31_bits():
    """Steps over the slots end up to 2^18 behind the last: those of larger caches would have wrapped, and the cache
    of a sequence of nearly 2^31 tokens been given up."""
    most = 2**31 - 1 - 2**18
    for slots in (most + 1, 2**31 - 1):
        assert evict(shape(head_dim=8, n_q_heads=1, n_kv_heads=1, batch=1, total_kv=slots)) == SHAPE
        assert evict(shape(), slots) == SHAPE
    assert evict(shape(total_kv=most)) == WORKSPACE and evict(shape(), most) == WORKSPACE   # (there is none)


def test_tokens_and_channels_that_pass_31_bits():
    # a tree's own keys are counted on behind the cached ones
    assert tree(shape(total_q=1000, total_kv=2**31 - 1 - 1024 - 999)) == SHAPE
    # heads times head_dim of one token
    for heads in (dict(n_q_heads=2**24, n_kv_heads=1), dict(n_q_heads=2**25, n_kv_heads=2**10)):
        assert tree(shape(total_q=1, **heads)) == SHAPE
        assert weight(shape(total_q=1, **heads)) == SHAPE


def test_trees_of_more_nodes_than_words_have_bits_for():
    # refused before there is a mask of that many words (125 GB of them here)
    nodes = 1000000
    with pytest.raises(B.CpError) as e:
        B.cp_tree_mask(np.full(nodes, -1, dtype=np.int32), [0, nodes])
    assert e.value.status == SHAPE
