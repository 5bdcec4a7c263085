"""Sizes past 32 bits are refused by the binding of the calls on e4m3 blocks of 128 and of the selection, whose library takes them in 32 (no GPU)."""
import pytest
import torch

from paper_2303_06182_amd import binding

MANY = 2 ** 32 + 5  # its low 32 bits are a size that would be taken


def huge(*shape, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device="meta")


@pytest.mark.parametrize("call", [
    lambda: binding.moe_select_experts(huge(MANY, 1), 1),
    lambda: binding.moe_select_experts(huge(4, MANY), 1),
    lambda: binding.moe_select_experts(huge(4, 8), MANY),
    lambda: binding.moe_select_experts(huge(4, 8), 1 - 2 ** 32),
    lambda: binding.moe_select_experts(huge(4, 8), 1, n_groups=MANY, groups_kept=1),
    lambda: binding.moe_select_experts(huge(4, 8), 1, groups_kept=2 ** 32 + 1),
    lambda: binding.moe_select_experts(huge(4, 8), 1, group_top=2 ** 32 + 1),
    lambda: binding.moe_select_experts(huge(4, 8), 1, renormalize=2 ** 32),
    lambda: binding.moe_quantize_b128(huge(MANY, 16)),
    lambda: binding.moe_quantize_b128(huge(16, 2 ** 32 + 16)),
    lambda: binding.moe_quantize_b128(huge(2 ** 16, 2 ** 16 + 1, 8, 16)),
    lambda: binding.moe_gemm_b128(huge(MANY, 16, dtype=torch.uint8), None, huge(8, 16, dtype=torch.uint8), None),
    lambda: binding.moe_gemm_b128(huge(4, 16, dtype=torch.uint8), None, huge(8, 16, dtype=torch.uint8), None, a_rows=huge(MANY, dtype=torch.int32)),
    lambda: binding.moe_gemm_b128(huge(4, 16, dtype=torch.uint8), None, huge(2 ** 32 + 8, 16, dtype=torch.uint8), None),
])
def test_functions(call):
    with pytest.raises(ValueError, match="32 bits"):
        call()


def test_layer():
    layer = binding.MoeLayer.__new__(binding.MoeLayer)  # no handle: refused before one is needed
    layer.h = None
    with pytest.raises(ValueError, match="32 bits"):
        layer.moe_expert_ffn_b128(huge(MANY, 16), None, None, None, None, None)
    with pytest.raises(ValueError, match="32 bits"):
        layer.moe_expert_ffn_b128(huge(4, 16), None, None, None, None, None, src_tok=huge(MANY, dtype=torch.int32))
    with pytest.raises(ValueError, match="32 bits"):
        layer.moe_layer_forward_b128(huge(MANY, 16), None, None, None, None, None)
