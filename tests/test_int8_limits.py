"""The stated limits of the dense half in 8-bit integers, on a host without a GPU.  No call here reaches a kernel."""
import os
import re

import pytest
import torch

import paper_2606_21712_amd as moe

INVALID, UNSUPPORTED = 1, 2
P = 0x10000          # a 16-byte aligned address that is never dereferenced
NAN, INF = float("nan"), float("inf")
HEADER = re.sub(r"\s*\n \*\s*", " ", open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "moe.h")).read())


def join(eps=1e-6, alpha=1.0, offset=0.0):
    """The checks of a call without rows, which come before its rows are looked at."""
    return moe.lib().moe_norm_join(P, 64, moe.DTYPE_BF16, P, 64, 1, P, P, 64, 3, 0, alpha, P, offset, eps, 0, 64, P, 64, 0, P, None,
                                   None)


@pytest.mark.parametrize("name", ["eps", "alpha", "offset"])
def test_norm_join_says_which_numbers_it_takes(name):
    """Up to 1e30 in size; the message and the header give the limit, not that a finite number is none."""
    signs = (1,) if name == "eps" else (1, -1)
    for sign in signs:
        for value in (0.0, 1e-30, 1.0, 1e30):
            assert join(**{name: sign * value}) == 0, value
    for value in [sign * v for sign in signs for v in (1.1e30, 3e38, INF)] + [NAN] + ([-1e-30] if name == "eps" else []):
        assert join(**{name: value}) == INVALID, value
        message = moe.lib().moe_last_error().decode()
        assert name in message and "1e30" in message and "finite" not in message
    contract = HEADER.split("moe_norm_join - ")[1].split("moe_status moe_norm_join(")[0]
    assert "eps, alpha or offset beyond 1e30 or NaN" in contract


WIDE = (1 << 32) + 64        # what a 32-bit argument would cut off to 64


def meta(shape, dtype):
    return torch.empty(shape, dtype=dtype, device="meta")


def test_sizes_past_32_bits_are_not_cut_off():
    """The library's columns and channels are 32 bits wide; more are refused, not taken as what is left of them."""
    bf, i8 = torch.bfloat16, torch.int8
    assert moe.moe_int8_code_bytes(16, 64) == 2048 and moe.moe_int8_code_bytes(16, WIDE) == 0
    for size in (moe.moe_matmul_int8_workspace_bytes, moe.moe_gated_int8_workspace_bytes):
        moe.set_cu_budget(256)
        try:
            need = size(128, 4096, 14336)
            assert need > 0 and size(128, (1 << 32) + 4096, 14336) == 0 and size(128, 4096, (1 << 32) + 14336) == 0
            assert size(128, -(1 << 32) + 4096, 14336) == 0
        finally:
            moe.set_cu_budget(0)
    for call in (lambda: moe.Int8(torch.zeros(2048, dtype=i8), torch.ones(16), (16, WIDE)),
                 lambda: moe.Int8(torch.zeros(2048, dtype=i8), meta(WIDE, torch.float32), (WIDE, 64)),
                 lambda: moe.moe_pack_int8(meta((1, WIDE), i8), torch.ones(1)),
                 lambda: moe.moe_quantize_int8(meta((1, WIDE), bf)),
                 lambda: moe.moe_norm_join(meta((1, WIDE), bf), pre=True),
                 lambda: moe.moe_norm_join(meta((1, WIDE), torch.float32), meta((1, WIDE), bf))):
        with pytest.raises(moe.MoEError) as e:
            call()
        assert e.value.status == UNSUPPORTED


def test_norm_join_says_which_rows_it_takes():
    """fp32 squares have an end on both sides."""
    contract = HEADER.split("moe_norm_join - ")[1].split("moe_status moe_norm_join(")[0]
    assert "sum to 2^128 or more" in contract and "eps below 2^-100" in contract and "below 2^-50" in contract


def test_products_say_in_which_order_scales_are_applied():
    """The sum times the token's scale comes first: the scales' own product may lie outside of fp32."""
    contract = HEADER.split("moe_matmul_int8 - ")[1].split("moe_gated_int8 - ")[0]
    assert "(sum_k x[t][k] w[n][k]) * x_scales[t] * w_scales[n] + bias[n]" in contract and "in this order" in contract


def test_norm_join_says_which_codes_a_product_takes():
    """Codes come for every H that is a multiple of 8, products take multiples of 16."""
    assert "H % 16 == 0" in HEADER.split("moe_norm_join - ")[1].split("moe_status moe_norm_join(")[0]
    assert moe.lib().moe_matmul_int8(P, P, P, P, None, 1, 16, 72, P, None, 0, None) == INVALID


def test_gated_products_say_where_their_gate_ends():
    """1 / (1 + exp(-g)) is under the smallest normal fp32 number there, and the reciprocal gives 0."""
    contract = HEADER.split("moe_gated_int8 - ")[1].split("size_t moe_matmul_int8_workspace_bytes")[0]
    assert "g below -87.3" in contract
