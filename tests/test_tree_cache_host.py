"""The calls on the KV cache (trees of drafted tokens, attention weight, eviction) without a GPU: masks
from parents, and what is refused before anything is launched."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2411_01783_amd import binding as B

ONE = ctypes.c_void_p(256)    # never dereferenced: the calls below fail validation first
ODD = ctypes.c_void_p(264)    # not 16-byte aligned
NULL, SHAPE, UNSUPPORTED, WORKSPACE, ALIGN = -1, -2, -3, -4, -6


def shape(**kw):
    a = dict(dtype=B.CP_BF16, head_dim=128, n_q_heads=16, n_kv_heads=2, total_q=8, total_kv=64, batch=2)
    a.update(kw)
    return B.make_shape(**a)


def refused(fn, s, args, workspace=True):
    tail = [ONE, ctypes.c_size_t(1 << 40)] if workspace else []
    return fn(ctypes.byref(s) if s is not None else None, *args, *tail, None)


@pytest.mark.parametrize("words", [1, 2, 16])
def test_tree_mask(words):
    rng = np.random.default_rng(words)
    nodes = [5, 0, 64 * words, 1]
    parents = np.concatenate([[rng.integers(-1, i) if i else -1 for i in range(n)] for n in nodes]).astype(np.int32)
    cu = np.concatenate([[0], np.cumsum(nodes)])
    mask = B.cp_tree_mask(parents, cu, words).view(np.uint64)
    for b, n in enumerate(nodes):
        for i in range(n):
            want, at = [0] * words, i
            while at >= 0:
                want[at // 64] |= 1 << (at % 64)
                at = int(parents[cu[b] + at])
            assert [int(x) for x in mask[cu[b] + i]] == want
    assert B.cp_tree_mask(parents[:5], [0, 5]).shape == (5, 1)
    assert B.cp_tree_mask(np.arange(-1, 64), [0, 65]).shape == (65, 2)


@pytest.mark.parametrize("parents,cu,words", [
    ([-1, 1], [0, 2], 1),                 # a node that is its own parent
    ([-1, -2], [0, 2], 1),
    ([-1, 0, 2], [0, 2, 3], 1),           # a parent in another tree
    ([-1] * 65, [0, 65], 1),              # more nodes than bits
    ([-1], [0, 1], 0),
    ([-1], [0, 1], 17),
    ([-1, 0], [0, 3, 2], 1),              # boundaries that fall
])
def test_tree_mask_refuses(parents, cu, words):
    with pytest.raises(B.CpError):
        B.cp_tree_mask(parents, cu, words)


def test_tree_attn_validates_before_launching():
    fn = B.load().cp_tree_attn
    # q, q_pos, cu_q, k_new, v_new, mask, words, k, v, kv_pos, cu_kv, used, out, lse, out_dtype
    good = [ONE, ONE, ONE, ONE, ONE, ONE, 1, ONE, ONE, ONE, ONE, ONE, ONE, ONE, 0]

    def call(s=None, **kw):
        a = list(good)
        for i, x in kw.items():
            a[int(i[1:])] = x
        return refused(fn, s or shape(), a)
    assert refused(fn, None, good) == NULL
    assert call(shape(dtype=7)) == UNSUPPORTED
    assert call(shape(head_dim=96)) == UNSUPPORTED
    assert call(shape(n_q_heads=5)) == SHAPE
    assert call(shape(batch=0)) == SHAPE
    assert call(shape(total_q=-1)) == SHAPE
    assert call(shape(total_kv=2**31)) == SHAPE
    assert call(shape(total_q=2**31 - 1)) == SHAPE           # rows past 31 bits
    assert call(shape(softmax_scale=float("nan"))) == SHAPE
    assert call(_14=2) == UNSUPPORTED
    for i in (0, 1, 2, 5, 7, 8, 9, 10, 12, 13):
        assert call(**{"_%d" % i: None}) == NULL, i
    assert call(_3=None) == NULL and call(_4=None) == NULL   # one of K and V
    assert call(_6=0) == SHAPE and call(_6=17) == SHAPE
    for i in (0, 3, 4, 7, 8, 12):
        assert call(**{"_%d" % i: ODD}) == ALIGN, i
    lib = B.load()
    s = shape()
    need = B.cp_workspace_bytes(s, B.CP_WS_TREE)
    assert need > 0
    for ws, size in ((None, need), (ODD, need), (ONE, need - 1)):
        assert fn(ctypes.byref(s), *good, ws, ctypes.c_size_t(size), None) == WORKSPACE
    # no nodes: accepted without touching any buffer
    assert call(shape(total_q=0), _0=None, _12=None) == 0
    assert lib.cp_workspace_bytes(ctypes.byref(shape(head_dim=96)), B.CP_WS_TREE) == 0


def test_tree_accept_validates_before_launching():
    fn = B.load().cp_tree_accept
    # k_new, v_new, pos_new, cu_new, mask, words, accepted, k, v, kv_pos, cu, used, dropped
    good = [ONE, ONE, ONE, ONE, ONE, 1, ONE, ONE, ONE, ONE, ONE, ONE, None]

    def call(s=None, **kw):
        a = list(good)
        for i, x in kw.items():
            a[int(i[1:])] = x
        return refused(fn, s or shape(), a, workspace=False)
    assert refused(fn, None, good, workspace=False) == NULL
    assert call(shape(dtype=3)) == UNSUPPORTED and call(shape(head_dim=12)) == UNSUPPORTED
    assert call(shape(batch=0)) == SHAPE and call(shape(total_kv=-1)) == SHAPE
    assert call(_5=0) == SHAPE and call(_5=17) == SHAPE
    for i in (0, 1, 2, 3, 4, 6, 7, 8, 9, 10, 11):
        assert call(**{"_%d" % i: None}) == NULL, i
    for i in (0, 1, 7, 8):
        assert call(**{"_%d" % i: ODD}) == ALIGN, i
    assert call(shape(n_kv_heads=2**20)) == SHAPE            # a path's chunks past 31 bits
    assert call(shape(total_q=0), _0=None) == 0


def test_attn_weight_validates_before_launching():
    fn = B.load().cp_kv_attn_weight
    # q, q_pos, cu_q, lse, k, kv_pos, cu_kv, used, decay, weight
    good = [ONE, ONE, ONE, ONE, ONE, ONE, ONE, ONE, 1.0, ONE]

    def call(s=None, **kw):
        a = list(good)
        for i, x in kw.items():
            a[int(i[1:])] = x
        return refused(fn, s or shape(), a)
    assert refused(fn, None, good) == NULL
    assert call(shape(dtype=3)) == UNSUPPORTED and call(shape(head_dim=80)) == UNSUPPORTED
    assert call(shape(n_q_heads=3)) == SHAPE and call(shape(batch=0)) == SHAPE
    for decay in (-0.5, float("nan"), float("inf")):
        assert call(_8=decay) == SHAPE
    for i in (0, 1, 2, 3, 4, 5, 6, 9):
        assert call(**{"_%d" % i: None}) == NULL, i
    for i in (0, 4):
        assert call(**{"_%d" % i: ODD}) == ALIGN, i
    s = shape()
    need = B.cp_workspace_bytes(s, B.CP_WS_WEIGHT)           # two KV heads: two parts
    assert need > 0
    for ws, size in ((None, need), (ODD, need), (ONE, need - 1)):
        assert fn(ctypes.byref(s), *good, ws, ctypes.c_size_t(size), None) == WORKSPACE
    assert call(shape(total_kv=0), _4=None, _9=None) == 0


def test_evict_validates_before_launching():
    fn = B.load().cp_kv_evict
    two = ctypes.c_void_p(4096)
    # k, v, kv_pos, weight, cu, used, budget, protect, sinks, k, v, kv_pos, weight, cu, used (to), slots_to
    inplace = [ONE, ONE, ONE, ONE, ONE, ONE, ONE, None, 0] + [None] * 6 + [0]
    into = inplace[:9] + [two] * 6 + [32]

    def call(s=None, base=inplace, **kw):
        a = list(base)
        for i, x in kw.items():
            a[int(i[1:])] = x
        return refused(fn, s or shape(), a)
    assert refused(fn, None, inplace) == NULL
    assert call(shape(dtype=3)) == UNSUPPORTED and call(shape(head_dim=300)) == UNSUPPORTED
    assert call(shape(batch=0)) == SHAPE and call(_8=-1) == SHAPE and call(shape(batch=70000)) == SHAPE
    for i in range(7):
        assert call(**{"_%d" % i: None}) == NULL, i
    for i in range(9, 15):
        assert call(base=into, **{"_%d" % i: None}) == NULL, i
    for i in range(10, 15):
        assert call(**{"_%d" % i: two}) == NULL, i           # part of a destination
    for i in (9, 10, 11, 12, 14):
        assert call(base=into, **{"_%d" % i: ONE}) == SHAPE, i   # the source itself
    assert call(base=into, _15=-1) == SHAPE
    for i in (0, 1):
        assert call(**{"_%d" % i: ODD}) == ALIGN, i
    for i in (9, 10):
        assert call(base=into, **{"_%d" % i: ODD}) == ALIGN, i
    s = shape(head_dim=24)
    need = B.cp_workspace_bytes(s, B.CP_WS_EVICT)
    assert need > 0
    for ws, size in ((None, need), (ODD, need), (ONE, need - 1)):
        assert fn(ctypes.byref(s), *inplace, ws, ctypes.c_size_t(size), None) == WORKSPACE


class HostCache:
    """What the binding reads of a KVCache, in host memory."""

    def __init__(self, nkv=2, d=128, dtype=torch.bfloat16, slots=64, batch=2):
        self.k = torch.zeros((slots, nkv, d), dtype=dtype)
        self.v = torch.zeros_like(self.k)
        self.kv_pos = torch.zeros(slots, dtype=torch.int32)
        self.cu = torch.zeros(batch + 1, dtype=torch.int32)
        self.used = torch.zeros(batch + 1, dtype=torch.int32)
        self.dropped = torch.zeros(1, dtype=torch.int32)


def tree_args(**kw):
    a = dict(cache=HostCache(), q=torch.zeros((8, 16, 128), dtype=torch.bfloat16),
             q_pos=torch.zeros(8, dtype=torch.int32), k_new=torch.zeros((8, 2, 128), dtype=torch.bfloat16),
             v_new=torch.zeros((8, 2, 128), dtype=torch.bfloat16), cu_seqlens_q=torch.zeros(3, dtype=torch.int32),
             tree_mask=torch.zeros((8, 1), dtype=torch.int64), stream=0)
    a.update(kw)
    return a


I32 = torch.int32


@pytest.mark.parametrize("kw,error", [
    (dict(q=torch.zeros((8, 16, 64), dtype=torch.bfloat16)), ValueError),
    (dict(q=torch.zeros((8, 16, 128))), ValueError),
    (dict(q=torch.zeros((8, 128), dtype=torch.bfloat16)), ValueError),
    (dict(q_pos=torch.zeros(7, dtype=I32)), ValueError),
    (dict(q_pos=torch.zeros(8, dtype=torch.int64)), TypeError),
    (dict(cu_seqlens_q=torch.zeros(4, dtype=I32)), ValueError),
    (dict(k_new=torch.zeros((7, 2, 128), dtype=torch.bfloat16)), ValueError),
    (dict(v_new=torch.zeros((8, 1, 128), dtype=torch.bfloat16)), ValueError),
    (dict(k_new=None), ValueError),
    (dict(tree_mask=None), ValueError),
    (dict(tree_mask=torch.zeros((8, 1), dtype=I32)), TypeError),
    (dict(tree_mask=torch.zeros((7, 1), dtype=torch.int64)), ValueError),
    (dict(lse=torch.zeros((8, 15))), ValueError),
    (dict(out=torch.zeros((8, 15, 128))), ValueError),
])
def test_binding_refuses_trees(kw, error):
    with pytest.raises(error):
        B.cp_tree_attn(**tree_args(**kw))


@pytest.mark.parametrize("kw,error", [
    (dict(accepted=torch.zeros(3, dtype=I32)), ValueError),
    (dict(accepted=torch.zeros(2, dtype=torch.int64)), TypeError),
    (dict(k_new=torch.zeros((8, 2, 64), dtype=torch.bfloat16)), ValueError),
    (dict(v_new=torch.zeros((9, 2, 128), dtype=torch.bfloat16)), ValueError),
    (dict(pos_new=torch.zeros(9, dtype=I32)), ValueError),
])
def test_binding_refuses_paths(kw, error):
    a = tree_args()
    a = dict(cache=a["cache"], k_new=a["k_new"], v_new=a["v_new"], pos_new=a["q_pos"],
             cu_seqlens_new=a["cu_seqlens_q"], tree_mask=a["tree_mask"], accepted=torch.zeros(2, dtype=I32), stream=0)
    a.update(kw)
    with pytest.raises(error):
        B.cp_tree_accept(**a)


@pytest.mark.parametrize("kw,error", [
    (dict(lse=torch.zeros((8, 2))), ValueError),
    (dict(lse=torch.zeros((8, 16), dtype=torch.float64)), TypeError),
    (dict(weight=torch.zeros(63)), ValueError),
    (dict(weight=torch.zeros(64, dtype=torch.bfloat16)), TypeError),
    (dict(cu_seqlens_q=torch.zeros(2, dtype=I32)), ValueError),
])
def test_binding_refuses_weights(kw, error):
    a = tree_args()
    a = dict(cache=a["cache"], q=a["q"], q_pos=a["q_pos"], lse=torch.zeros((8, 16)), weight=torch.zeros(64),
             cu_seqlens_q=a["cu_seqlens_q"], stream=0)
    a.update(kw)
    with pytest.raises(error):
        B.cp_kv_attn_weight(**a)


@pytest.mark.parametrize("kw,error", [
    (dict(budget=torch.zeros(3, dtype=I32)), ValueError),
    (dict(budget=torch.zeros(2)), TypeError),
    (dict(protect_from=torch.zeros(1, dtype=I32)), ValueError),
    (dict(sinks=-1), ValueError),
    (dict(into=HostCache()), ValueError),
    (dict(into=HostCache(), into_weight=torch.zeros(9)), ValueError),
    (dict(into=HostCache(nkv=1), into_weight=torch.zeros(64)), ValueError),
    (dict(into=HostCache(batch=3), into_weight=torch.zeros(64)), ValueError),
    (dict(into=HostCache(dtype=torch.float32), into_weight=torch.zeros(64)), ValueError),
])
def test_binding_refuses_evictions(kw, error):
    a = dict(cache=HostCache(), weight=torch.zeros(64), budget=torch.zeros(2, dtype=I32), stream=0)
    a.update(kw)
    with pytest.raises(error):
        B.cp_kv_evict(**a)
