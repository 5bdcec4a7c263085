"""What moe_attn_create and moe_sample refuse, found on the host before anything is launched (no GPU)."""
import ctypes

import pytest

from paper_2303_06182_amd import binding

GEOMETRY = dict(B_max=4, T_max=64, n_heads=8, n_kv_heads=2, head_dim=64, page_size=16, num_pages=8, max_pages=4, dtype=binding.MOE_DTYPE_BF16,
                rot_dim=64, rot_interleaved=0)


@pytest.fixture(scope="module")
def lib():
    return binding.load_library()


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=7), binding.MOE_ERR_UNSUPPORTED), (dict(head_dim=96), binding.MOE_ERR_UNSUPPORTED), (dict(n_kv_heads=0), binding.MOE_ERR_UNSUPPORTED),
    (dict(n_heads=9), binding.MOE_ERR_UNSUPPORTED), (dict(n_heads=0), binding.MOE_ERR_UNSUPPORTED), (dict(n_heads=512), binding.MOE_ERR_UNSUPPORTED),
    (dict(page_size=8), binding.MOE_ERR_UNSUPPORTED), (dict(page_size=48), binding.MOE_ERR_UNSUPPORTED), (dict(page_size=256), binding.MOE_ERR_UNSUPPORTED),
    (dict(rot_dim=80), binding.MOE_ERR_UNSUPPORTED), (dict(rot_dim=8), binding.MOE_ERR_UNSUPPORTED), (dict(B_max=0), binding.MOE_ERR_UNSUPPORTED),
    (dict(B_max=5000), binding.MOE_ERR_UNSUPPORTED), (dict(T_max=-1), binding.MOE_ERR_INVALID_ARG), (dict(T_max=1 << 24), binding.MOE_ERR_INVALID_ARG),
    (dict(num_pages=0), binding.MOE_ERR_INVALID_ARG), (dict(max_pages=0), binding.MOE_ERR_INVALID_ARG),
    (dict(max_pages=1 << 27), binding.MOE_ERR_INVALID_ARG), (dict(rot_interleaved=2), binding.MOE_ERR_INVALID_ARG),
])
def test_attn_create_refuses(lib, kw, code):
    cfg = binding.MoeAttnConfig(**{**GEOMETRY, **kw})
    h = ctypes.c_void_p()
    assert lib.moe_attn_create(ctypes.byref(cfg), ctypes.byref(h)) == code
    assert not h.value and lib.moe_last_error() != b""


def test_null_handles(lib):
    cfg = binding.MoeAttnConfig(**GEOMETRY)
    h = ctypes.c_void_p()
    assert lib.moe_attn_create(None, ctypes.byref(h)) == binding.MOE_ERR_INVALID_ARG
    assert lib.moe_attn_create(ctypes.byref(cfg), None) == binding.MOE_ERR_INVALID_ARG
    assert lib.moe_attn_workspace_bytes(None) == binding.MOE_ERR_INVALID_ARG
    assert lib.moe_attn_destroy(None) == binding.MOE_OK
    z = [None, 0]
    assert lib.moe_kv_append(None, None, *z, *z, *z, None, None, None, None, 0, 0, 0, None, None) == binding.MOE_ERR_INVALID_ARG
    assert lib.moe_attn_forward(None, None, None, 0, None, None, None, 0, 0, 0, 0, 1.0, 1, 0, None, None, None, 0, None) == binding.MOE_ERR_INVALID_ARG


def call(lib, **kw):
    """moe_sample with addresses that nothing reads, because the call is refused (or has no rows)."""
    a = dict(logits=1 << 20, dtype=0, stride=1000, B=2, V=1000, u=1 << 20, temperature=None, top_k=None, top_p=None, min_p=None, token=1 << 20,
             logprob=None, ws=1 << 20, wsb=1 << 40)
    a.update(kw)
    return lib.moe_sample(a["logits"], a["dtype"], a["stride"], a["B"], a["V"], a["u"], a["temperature"], a["top_k"], a["top_p"], a["min_p"], a["token"],
                          a["logprob"], a["ws"], a["wsb"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(B=-1), binding.MOE_ERR_INVALID_ARG), (dict(V=0), binding.MOE_ERR_INVALID_ARG), (dict(V=(1 << 19) + 1), binding.MOE_ERR_INVALID_ARG),
    (dict(dtype=5), binding.MOE_ERR_UNSUPPORTED), (dict(logits=None), binding.MOE_ERR_INVALID_ARG), (dict(logits=(1 << 20) + 2), binding.MOE_ERR_INVALID_ARG),
    (dict(u=None), binding.MOE_ERR_INVALID_ARG), (dict(u=(1 << 20) + 2), binding.MOE_ERR_INVALID_ARG), (dict(token=None), binding.MOE_ERR_INVALID_ARG),
    (dict(top_k=(1 << 20) + 1), binding.MOE_ERR_INVALID_ARG), (dict(stride=999), binding.MOE_ERR_INVALID_ARG), (dict(dtype=1, logits=(1 << 20) + 1), binding.MOE_ERR_INVALID_ARG),
    (dict(ws=None), binding.MOE_ERR_WORKSPACE), (dict(ws=(1 << 20) + 16), binding.MOE_ERR_WORKSPACE),
    (dict(wsb=0), binding.MOE_ERR_WORKSPACE),
])
def test_sample_refuses(lib, kw, code):
    assert call(lib, **kw) == code
    assert lib.moe_last_error() != b""


def test_sample_without_rows(lib):
    assert call(lib, B=0) == binding.MOE_OK
    assert lib.moe_sample_workspace_bytes(0, 0) == binding.MOE_ERR_INVALID_ARG
    assert lib.moe_sample_workspace_bytes(256, 128000) > 0
