"""Quantisation to e4m3 in blocks of 128 at the largest number of rows that its arguments can name."""
import numpy as np
import pytest
import torch

from oracle import b128
from paper_2303_06182_amd import binding

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def memory_is_given_back():
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("block_rows", [128, 1])
def test_quantize_most_rows(block_rows):
    """2^31 - 1 rows: the last block of 128 ends with the last of them."""
    rows, cols = 2 ** 31 - 1, 16
    if torch.cuda.get_device_properties(0).total_memory < 150 * 2 ** 30:
        pytest.skip("needs 110 GB")
    x = torch.zeros((rows, cols), dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    x[-300:] = torch.randn((300, cols), device="cuda", generator=g).bfloat16()
    x[0, 3] = 448.0 * 4
    q, scale = torch.full((rows, cols), 0x55, dtype=torch.uint8, device="cuda"), torch.full((rows if block_rows == 1 else 1 << 24, 4), 9, dtype=torch.uint8, device="cuda")
    binding.moe_quantize_b128(x, block_rows, q=q.view(torch.float8_e4m3fn), scale=scale)
    tail = x[-383:].double().cpu().numpy()  # three blocks of 128 rows, the last of 127
    number, byte = b128.quantize(tail, block_rows)
    assert np.array_equal(q[-383:].view(torch.float8_e4m3fn).double().cpu().numpy(), number)
    assert np.array_equal(scale[-len(byte):].cpu().numpy(), byte)
    assert q[0].tolist() == [0, 0, 0, 0x7e] + [0] * 12 and scale[0].tolist() == [129, 127, 127, 127]
    assert not q[1:-383].any() and (scale[1:-len(byte)].view(torch.int32) == 0x7f7f7f7f).all()
