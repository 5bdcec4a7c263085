"""moe_b128_workspace_bytes: no size for a handle that the calls which need one refuse."""
import pytest

from paper_2303_06182_amd import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,F,fits", [(128, 144, True), (120, 144, False), (128, 136, False), (2 ** 23, 64, True), (2 ** 23 + 16, 64, False), (64, 2 ** 23 + 16, False),
                                      (64, 2 ** 31 - 16, False)])
def test_sizes(D, F, fits):
    layer = binding.MoeLayer(0, D, F, 2, 1, "bf16", alloc_workspace=False)
    n = layer.lib.moe_b128_workspace_bytes(layer.h)
    assert n > 0 if fits else n == binding.MOE_ERR_UNSUPPORTED
    if not fits:
        with pytest.raises(binding.MoeError):
            layer.b128_workspace()
