"""What the binding of append, attention and sampling refuses before the library is called (no GPU): tensors on another device than the handle's, and
outputs that are not what the call writes."""
import types

import pytest
import torch

from paper_2303_06182_amd import binding


class Reached(Exception):
    pass


def reached(*_):
    raise Reached


@pytest.fixture
def att(monkeypatch):
    """A handle of nothing, for a device of number -1, which is what tensors in host memory say; a call that gets as far as the library raises Reached."""
    a = object.__new__(binding.PagedAttention)
    a.h, a.device, a.index, a.torch_dtype = None, torch.device("cpu"), -1, torch.bfloat16
    a.cfg = binding.MoeAttnConfig(2, 8, 4, 2, 64, 16, 6, 3, binding.MOE_DTYPE_BF16, 64, 0)
    a.cache_shape = (6, 2, 16, 64)
    a.lib = types.SimpleNamespace(moe_kv_append=reached, moe_attn_forward=reached)
    a.workspace = torch.empty(256, dtype=torch.uint8)
    monkeypatch.setattr(binding, "_stream_on", lambda index: 0)
    return a


def cache():
    bytes_, scales = lambda: torch.zeros((6, 2, 16, 64), dtype=torch.uint8), lambda: torch.ones((6, 2))  # noqa: E731
    return binding.KvCache(bytes_(), bytes_(), scales(), scales())


def rows(heads, T=3, dtype=torch.bfloat16):
    return torch.zeros((T, heads, 64), dtype=dtype)


def batch():
    return torch.tensor([0, 1, 3], dtype=torch.int32), torch.tensor([5, 9], dtype=torch.int32), torch.zeros((2, 3), dtype=torch.int32)


def append(a, q_out=None):
    return a.moe_kv_append(cache(), rows(4), rows(2), rows(2), torch.ones(32, dtype=torch.float64), *batch(), 2, q_out=q_out)


def attend(a, **kw):
    return a.moe_attn_forward(cache(), rows(4), *batch(), 2, 9, **kw)


def test_what_fits_reaches_the_library(att):
    for call in (lambda: append(att), lambda: append(att, rows(4)), lambda: attend(att), lambda: attend(att, out=rows(4), lse=torch.zeros((3, 4)))):
        with pytest.raises(Reached):
            call()


WRONG = [lambda: rows(4, 2), lambda: rows(4, 4), lambda: rows(2), lambda: rows(4, dtype=torch.float32), lambda: rows(8)[:, ::2], lambda: rows(4).view(3, 256)]


@pytest.mark.parametrize("make", WRONG)
def test_outputs_of_another_shape_type_or_layout(att, make):
    with pytest.raises(ValueError, match="q_out"):
        append(att, make())
    with pytest.raises(ValueError, match="out"):
        attend(att, out=make())


@pytest.mark.parametrize("lse", [torch.zeros((3, 2)), torch.zeros((2, 4)), torch.zeros((3, 4), dtype=torch.bfloat16), torch.zeros((4, 3)).T, torch.zeros(12)])
def test_lse_of_another_shape_type_or_layout(att, lse):
    with pytest.raises(ValueError, match="lse"):
        attend(att, lse=lse)


def test_tensors_in_host_memory(att):
    att.index, att.device = 0, torch.device("cuda:0")
    for call in (lambda: append(att), lambda: attend(att)):
        with pytest.raises(ValueError, match="on cuda:0"):
            call()
    c = cache()
    c.index = 0
    q = rows(4)
    with pytest.raises(ValueError, match="on cuda:0"):
        att._rows(q, 4, "q")
    for name in ("out", "lse"):
        with pytest.raises(ValueError, match="cuda:0"):
            binding._output(torch.zeros(3), (3,), torch.float32, 0, name)
    logits, u = torch.zeros((2, 10)), torch.zeros(2)
    with pytest.raises(ValueError, match="GPU"):
        binding.moe_sample(logits, u)
