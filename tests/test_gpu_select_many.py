"""Batches of thousands of tokens (moe_select_experts) against the 64-bit oracle, at rows made for what decides there: keys, and sums of groups, that lie within the
error of 32-bit ones of each other, and rows that lie just outside it.  Tolerance of the weights as in test_gpu_b128.py: 2^-24 and 2^-40 of them."""
import math

import numpy as np
import pytest
import torch

from oracle import b128
from paper_2303_06182_amd import binding
from test_gpu_b128 import BF16, DEV, F32, host

pytestmark = pytest.mark.gpu


def rows_for(E, G, rng):
    """About 300 rows of E logits."""
    size, out = E // G, []
    spread = rng.standard_normal((60, E)) * 1.5
    out += list(spread)
    for step in (2.0 ** -26, 2.0 ** -24, 2.0 ** -23, 2.0 ** -22, 2.0 ** -21, 2.0 ** -20, 2.0 ** -18):
        for base in (-3.0, 0.25, 1.0, 6.0, 12.0):
            out.append(base + step * max(1.0, abs(base)) * rng.permutation(E))                      # all keys close
            r = rng.standard_normal(E) - 4.0
            r[rng.permutation(E)[:min(E, 14)]] = base + step * max(1.0, abs(base)) * rng.permutation(min(E, 14))  # those at the border of k close
            out.append(r)
            r = rng.standard_normal((G, size)) - 2.0                                                 # two keys a group that add up to nearly the same
            r[:, 0] = base + step * max(1.0, abs(base)) * rng.permutation(G)
            out.append(r.ravel())
    for p in (0.3, 0.9, 0.99):
        r = rng.standard_normal((10, E))
        out += list(np.where(rng.random((10, E)) < p, -np.inf, r))
    out += list(np.round(rng.standard_normal((20, E)) * 2) / 2) + list(rng.standard_normal((20, E)) * 30)
    out += [np.full(E, v) for v in (0.0, -math.inf, math.nan, math.inf, 1e30, -1e30)]
    return np.array(out)


@pytest.mark.parametrize("E,G,kept,k,top", [(64, 1, 1, 2, 1), (128, 8, 3, 6, 2), (128, 8, 4, 8, 1), (130, 10, 9, 3, 2), (256, 8, 4, 8, 2), (257, 1, 1, 6, 1), (512, 16, 2, 8, 2),
                                            (1024, 64, 7, 8, 2)])
@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_against_the_oracle(E, G, kept, k, top, score, dtype):
    rng = np.random.default_rng(E + k)
    x = torch.tensor(rows_for(E, G, rng)).float().to(dtype)
    n = len(x)
    times = -(-7001 // n)
    logits = x.to(DEV).repeat(times, 1)[:7001]  # each row in several places of a wave and of a batch
    at = np.arange(7001) % n
    plain = (rng.standard_normal(E) * 0.1).astype(np.float32)
    close = (rng.integers(0, 3, E) * 2.0 ** -24).astype(np.float32)
    odd = plain.copy()
    odd[::7], odd[3], odd[5] = -np.inf, np.nan, np.inf
    for bias in (None, plain, close, plain * np.float32(1e6), odd):
        for renormalize in (True, False):
            kw = dict(score=score, n_groups=G, groups_kept=kept, group_top=top, renormalize=renormalize, scale=2.5)
            idx, w = binding.moe_select_experts(logits, k, bias=None if bias is None else torch.tensor(bias, device=DEV), **kw)
            want, ww = b128.select(host(x), k, bias=bias, **kw)
            assert np.array_equal(idx.cpu().numpy(), want[at])
            assert (np.abs(host(w) - ww[at]) <= np.abs(ww[at]) * (2.0 ** -24 + 2.0 ** -40) + 2.0 ** -149).all()
