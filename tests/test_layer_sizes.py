"""Sizes beyond 32 bits are refused where the library counts in int (host side; tensors without memory)."""
import pytest
import torch

import paper_2502_04507_amd as sta

BF = torch.bfloat16
MANY = 2 ** 32 + 5                                          # 5, if the upper bits were dropped


def meta(*shape, dtype=BF):
    return torch.empty(shape, dtype=dtype, device="meta")


def beyond():
    return pytest.raises(ValueError, match="does not fit 32 bits")


@pytest.mark.parametrize("shape", [(1, MANY, 1, 2), (MANY, 1, 1, 2), (1, 1, MANY, 2), (1, 1, 1, MANY)])
def test_rows(shape):
    x, ok = meta(*shape), meta(1, 1, 1, 2)

    class Rotary:                                           # (one on the device is not to be had here)
        _at = (1 << 20, -1, -1)

        def _struct(self, B, N):
            raise AssertionError("sizes come first")

    with beyond():
        sta.sta_rope(x, x, Rotary())
    with beyond():
        sta.sta_qk_norm_rope(x, ok, None, x, ok, None, None, None, Rotary())
    with beyond():
        sta.sta_qk_norm_rope_backward(x, ok, x, ok, None, x, ok, None, None, None, None, None, Rotary(), None)


@pytest.mark.parametrize("max_q,max_k,S", [(MANY, 4, 1), (4, MANY, 1), (2 ** 31, 4, 1), (4, 4, MANY)])
def test_packed(max_q, max_k, S):
    x, lse, cu = meta(4, 2, 64), meta(2, 4, dtype=torch.float32), meta(S + 1, dtype=torch.int32)
    with beyond():
        sta.sta_packed_forward(x, x, x, x, cu, cu, max_q, max_k)
    with beyond():
        sta.sta_packed_backward(x, x, x, x, x, lse, x, x, x, cu, cu, max_q, max_k, lse)


def test_heads_and_workspaces():
    x = meta(4, MANY, 64)
    cu = meta(2, dtype=torch.int32)
    with beyond():
        sta.sta_packed_forward(x, x, x, x, cu, cu, 4, 4)
    for at in range(7):
        args = [8, 2, 128, 1, 1, 1, 100000]
        if at != 4:                                         # tokens are counted in 64 bits
            args[at] += 2 ** 32
            with beyond():
                sta.sta_packed_workspace_bytes(*args)
    with beyond():
        sta.sta_packed_backward_workspace_bytes(MANY, 100)
    with beyond():
        sta.sta_qk_norm_rope_workspace_bytes(2 ** 32 + 64)
    with beyond():
        sta.sta_rope_steps(2 ** 32 + 64)
