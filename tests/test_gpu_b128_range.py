"""e4m3 operands whose scaled elements reach 2^128, and those next to it, as include/moe.h states them: bf16 results take the scales as exponents, fp32 results and
the feed-forward's first product widen each element, to an infinite one.  No other row or column is touched by that."""
import numpy as np
import pytest
import torch

from oracle import b128
from paper_2303_06182_amd import binding
from test_gpu_b128 import BF16, DEV, F32, check_ffn, check_sums, ffn_case, host, ints, operands

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,N,K", [(9, 136, 400), (3000, 1032, 400)])  # few output tiles, and whole ones
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_gemm(rows, N, K, dtype):
    (a, sa, _), (w, sw, _) = operands(rows, 2, N, K, rows, spread=1)
    sa, sw = sa.cpu().numpy(), sw.cpu().numpy()
    sa[:], sw[:] = 127, 80
    sa[3, 1], sa[5, 2] = 254, 247      # 2^127 and 2^120, times 448 at most
    sa[6, 0] = 246                     # 448 * 2^119 is less than 2^128
    sw[1, 1, 2], sw[1, 0, 1] = 254, 246  # of the second expert, whose rows have no large scales: columns 128 to 255, and up to 127
    cut = rows // 2 + 2
    sa[cut:] = 90
    av, wv = b128.value(host(a), sa), np.stack([b128.value(host(w[e]), sw[e], 128) for e in range(2)])
    want, size = b128.gemm(av, wv, [0, cut, rows])
    got = binding.moe_gemm_b128(a, torch.tensor(sa, device=DEV), w, torch.tensor(sw, device=DEV), offsets=ints([0, cut, rows]), out_dtype=dtype)
    spoiled = np.zeros(want.shape, dtype=bool)
    if dtype == F32:  # elements of 256 and more are among the 128 of each such block
        spoiled[3], spoiled[5], spoiled[cut:, 128:256] = True, True, True
    assert np.array_equal(~np.isfinite(host(got)), spoiled)
    for r in range(0, rows) if rows < 10 else list(range(0, 10)) + list(range(cut - 3, rows, 97)):  # rows and halves apart: their numbers are
        for cols in (slice(0, 128), slice(128, min(N, 256)), slice(256, N)):
            if not spoiled[r, cols].any() and want[r, cols].size:
                check_sums(got[r:r + 1, cols], want[r:r + 1, cols], size[r:r + 1, cols], K, dtype)


@pytest.mark.parametrize("rows", [6, 400])  # the stream, and tiles
@pytest.mark.parametrize("activation", ["relu", "silu"])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_ffn(rows, activation, dtype):
    x, src, weights, values, offsets = ffn_case(rows, rows, 2, 256, 144, activation, dtype, rows)
    x[4], x[5, 3] = 0.0, 248 * 2.0 ** 120  # the tie: rounds to 2^128
    x[4, 200] = 240 * 2.0 ** 120           # exact, 1.875 * 2^127
    assert torch.isfinite(x).all()
    layer = binding.MoeLayer(rows, 256, 144, 2, 1, "bf16" if dtype == BF16 else "f32", alloc_workspace=False)
    src = np.arange(rows)
    y = layer.moe_expert_ffn_b128(x, ints(offsets), *weights, activation=activation)
    keep = [r for r in range(rows) if r not in (4, 5)]
    at = np.searchsorted(keep, offsets)
    check_ffn(y[keep], x, src[keep], values, at.tolist(), activation, dtype, 256)
    assert not torch.isfinite(y[5]).any()
