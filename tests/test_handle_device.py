"""A handle is for a GPU: other devices are refused, before a GPU is looked for."""
import pytest

from paper_2303_06182_amd import binding


@pytest.mark.parametrize("device", ["cpu", "cpu:0", "meta"])
@pytest.mark.parametrize("make", [lambda d: binding.MoeLayer(4, 64, 64, 4, 2, "bf16", device=d), lambda d: binding.PagedAttention(2, 4, 4, 2, 64, 16, 8, 4, "bf16", device=d)])
def test_other_devices_are_refused(make, device):
    with pytest.raises(ValueError):
        make(device)


def test_a_gpu_by_its_number():
    assert str(binding._gpu("cuda:3")) == "cuda:3" and binding._gpu("cuda:0").index == 0
