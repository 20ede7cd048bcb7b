"""Workspaces that end in front of their first aligned byte, without a GPU: they hold nothing, and are refused as
such before anything is launched."""
import pytest
import torch

from paper_2411_01783_amd import binding as B

I32 = torch.int32


def small_view():
    whole = torch.zeros(1024, dtype=torch.uint8)
    first = (-whole.data_ptr()) % 256 + 16          # 16 bytes behind an aligned one
    return whole[first:first + 8]


def refused(call):
    with pytest.raises(B.CpError) as e:
        call()
    assert e.value.status == -4, e.value            # CP_ERR_WORKSPACE


def test_a_view_without_an_aligned_byte_is_no_workspace():
    assert B._ws_ptr(small_view())[1] == 0
    rows = lambda *s: torch.zeros(s, dtype=torch.bfloat16)
    q, kv = rows(2, 16, 128), rows(4096, 1, 128)
    refused(lambda: B.cp_attn_decode(q, kv, kv, torch.zeros(2, dtype=I32), torch.zeros(4096, dtype=I32),
                                     torch.tensor([0, 2048, 4096], dtype=I32), torch.tensor([0, 1], dtype=I32),
                                     workspace=small_view(), stream=0))
