"""What the calls on e4m3 operands in blocks of 128 and the selection of experts refuse, found on the host before anything is launched (no GPU)."""
import ctypes
import math

import pytest
import torch
import torch

from paper_2303_06182_amd import binding

INVALID, UNSUPPORTED, WORKSPACE = binding.MOE_ERR_INVALID_ARG, binding.MOE_ERR_UNSUPPORTED, binding.MOE_ERR_WORKSPACE
P = 1 << 20  # an address that nothing reads, because the call is refused or has no rows


@pytest.fixture(scope="module")
def lib():
    return binding.load_library()


def refused(lib, rc, code):
    assert rc == code and lib.moe_last_error() != b""


def select(lib, cfg=None, dtype=0, stride=64, T=2, logits=P, bias=None, idx=P, w=P, **kw):
    c = dict(E=64, k=4, score=1, n_groups=8, groups_kept=2, group_top=2, renormalize=1, scale=1.0)
    c.update(kw)
    cfg = binding.MoeSelectConfig(*c.values()) if cfg is None else cfg
    return lib.moe_select_experts(ctypes.byref(cfg), logits, dtype, stride, bias, T, idx, w, None)


@pytest.mark.parametrize("kw,code", [
    (dict(E=0), UNSUPPORTED), (dict(E=1025), UNSUPPORTED), (dict(k=0), UNSUPPORTED), (dict(k=9), UNSUPPORTED), (dict(score=2), UNSUPPORTED),
    (dict(score=-1), UNSUPPORTED), (dict(n_groups=0), UNSUPPORTED), (dict(n_groups=7), UNSUPPORTED), (dict(E=128, n_groups=128, groups_kept=128), UNSUPPORTED),
    (dict(groups_kept=0), UNSUPPORTED), (dict(groups_kept=9), UNSUPPORTED), (dict(n_groups=32, groups_kept=1), UNSUPPORTED), (dict(group_top=0), UNSUPPORTED),
    (dict(group_top=3), UNSUPPORTED), (dict(renormalize=2), INVALID), (dict(scale=math.inf), INVALID), (dict(scale=math.nan), INVALID),
    (dict(dtype=2), UNSUPPORTED), (dict(T=-1), INVALID), (dict(T=1 << 29), INVALID), (dict(stride=63), INVALID), (dict(logits=None), INVALID),
    (dict(logits=P + 2), INVALID), (dict(logits=P + 1, dtype=1), INVALID), (dict(bias=P + 2), INVALID), (dict(idx=None), INVALID), (dict(w=P + 1), INVALID),
])
def test_select_refuses(lib, kw, code):
    refused(lib, select(lib, **kw), code)


def test_select_without_tokens(lib):
    assert select(lib, T=0, logits=None, idx=None, w=None) == binding.MOE_OK
    refused(lib, lib.moe_select_experts(None, P, 0, 64, None, 1, P, P, None), INVALID)


def quantize(lib, x=P, dtype=1, stride=256, matrices=1, rows=4, cols=256, block_rows=1, q=P, scale=P):
    return lib.moe_quantize_b128(x, dtype, stride, matrices, rows, cols, block_rows, q, scale, None)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=4), UNSUPPORTED), (dict(block_rows=2), UNSUPPORTED), (dict(block_rows=0), UNSUPPORTED), (dict(cols=0), UNSUPPORTED), (dict(cols=24), UNSUPPORTED),
    (dict(rows=-1), INVALID), (dict(matrices=-1), INVALID), (dict(x=None), INVALID), (dict(x=P + 8), INVALID), (dict(q=None), INVALID), (dict(q=P + 4), INVALID),
    (dict(scale=None), INVALID), (dict(scale=P + 1), INVALID), (dict(stride=240), INVALID), (dict(stride=260), INVALID), (dict(stride=258, dtype=0), INVALID),
])
def test_quantize_refuses(lib, kw, code):
    refused(lib, quantize(lib, **kw), code)


def test_quantize_of_nothing(lib):
    assert quantize(lib, rows=0, x=None, q=None, scale=None) == binding.MOE_OK
    assert quantize(lib, matrices=0, x=None, q=None, scale=None) == binding.MOE_OK
    assert [binding.b128_scale_cols(c) for c in (1, 16, 128, 512, 513, 2048)] == [4, 4, 4, 4, 8, 16]
    with pytest.raises(binding.MoeError):
        binding.b128_scale_cols(0)


def gemm(lib, a=P, a_scale=P, count=8, a_rows=None, w=P, w_scale=P, offsets=P, E=4, rows=8, N=64, K=128, c=P, dtype=1):
    return lib.moe_gemm_b128(a, a_scale, count, a_rows, w, w_scale, offsets, E, rows, N, K, c, dtype, None)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=2), UNSUPPORTED), (dict(E=0), INVALID), (dict(E=1025), INVALID), (dict(offsets=None), INVALID), (dict(N=0), UNSUPPORTED), (dict(N=12), UNSUPPORTED),
    (dict(K=0), UNSUPPORTED), (dict(K=72), UNSUPPORTED), (dict(rows=-1), INVALID), (dict(rows=1 << 30, count=1 << 30), INVALID), (dict(count=7), INVALID),
    (dict(count=-1, a_rows=P), INVALID), (dict(count=0, a_rows=P), INVALID), (dict(a=None), INVALID), (dict(a=P + 8), INVALID), (dict(a_scale=P + 2), INVALID),
    (dict(a_rows=P + 2), INVALID), (dict(w=None), INVALID), (dict(w=P + 1), INVALID), (dict(w_scale=None), INVALID), (dict(offsets=P + 1), INVALID),
    (dict(c=None), INVALID), (dict(c=P + 8), INVALID),
])
def test_gemm_refuses(lib, kw, code):
    refused(lib, gemm(lib, **kw), code)


def test_gemm_of_nothing(lib):
    assert gemm(lib, rows=0, count=0, a=None, w=None, c=None) == binding.MOE_OK


def test_null_handles(lib):
    refused(lib, lib.moe_b128_workspace_bytes(None), INVALID)
    refused(lib, lib.moe_expert_ffn_b128(None, P, 1, None, P, P, P, P, P, 1, 1, P, P, 1 << 40, None), INVALID)
    refused(lib, lib.moe_layer_forward_b128(None, P, P, None, None, None, P, P, P, P, 1, 1, P, None, P, 1 << 40, None), INVALID)


def test_binding_refuses_before_the_library():
    x = torch.zeros((4, 256), dtype=torch.bfloat16)
    for call in (lambda: binding.moe_quantize_b128(x), lambda: binding.moe_select_experts(x, 2), lambda: binding.moe_quantize_b128(x[0]),
                 lambda: binding.moe_select_experts(x.half(), 2), lambda: binding.moe_quantize_b128(x.t()),
                 lambda: binding.moe_gemm_b128(x, x, x, x), lambda: binding.moe_gemm_b128(x[0], x, x, x)):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("dtype,fits", [(torch.float8_e4m3fn, True), (torch.uint8, True), (torch.int8, False), (torch.bool, False), (torch.float8_e5m2, False),
                                        (torch.float8_e4m3fnuz, False)])
def test_other_bytes_are_refused(dtype, fits):
    """One byte an element is not enough: only e4m3 as it is here, or its bytes."""
    q, scale = torch.empty((3, 128), dtype=dtype), torch.empty((3, 4), dtype=torch.uint8)
    if fits:
        binding._b128_operand(q, scale, (3, 128), (), 1, -1, "a")
    else:
        with pytest.raises(ValueError):
            binding._b128_operand(q, scale, (3, 128), (), 1, -1, "a")
