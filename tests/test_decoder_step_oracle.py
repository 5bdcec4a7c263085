"""Pins of the decoder-step oracle (no GPU): library routines written by others, special cases with known answers, hand-worked ones."""
import math

import numpy as np
import pytest
import torch

from oracle import decoder_step as od
from oracle import quant_e4m3 as oq


def empty_cache(pages, heads, page, dim):
    return dict(k=np.full((pages, heads, page, dim), 0x7F, np.uint8), v=np.full((pages, heads, page, dim), 0x7F, np.uint8),
                k_scale=np.full((pages, heads), np.nan), v_scale=np.full((pages, heads), np.nan))


def test_needed_scale_is_the_smallest_power_of_two_that_holds():
    for x in (448.0, 448.0001, 1.0, 0.875, 0.8751, 3e-5, 1e30):
        s = od.needed_scale(x)
        assert x <= 448 * s and x > 448 * s / 2
        assert s == oq.scale_of(x)
    assert od.needed_scale(0.0) == 2.0 ** -126


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_keeps_lengths_and_depends_on_distance_only(interleaved):
    rng = np.random.default_rng(0)
    q, k = rng.standard_normal((1, 32)), rng.standard_normal((1, 32))
    f = 10000.0 ** (-np.arange(8) / 8)
    near = od.rotate(q, 7, f, interleaved) @ od.rotate(k, 3, f, interleaved).T
    far = od.rotate(q, 100007, f, interleaved) @ od.rotate(k, 100003, f, interleaved).T
    assert near == pytest.approx(far, rel=1e-9)
    y = od.rotate(q, 12345, f, interleaved)
    assert np.linalg.norm(y) == pytest.approx(np.linalg.norm(q)) and np.array_equal(y[:, 16:], q[:, 16:])
    assert np.array_equal(od.rotate(q, 0, f, interleaved), q)


def test_append_by_hand():
    """A page of 4 rows: the scale grows with the second append, the first row is rounded anew, a fresh page starts over."""
    c = empty_cache(3, 1, 4, 16)
    row = lambda x: np.full((1, 1, 16), float(x))  # noqa: E731
    table = [[2, 0]]
    od.append(c, None, row(448), row(1), [], False, [0, 1], [1], table, 4)
    assert c["k_scale"][2, 0] == 1 and od.VALUES[c["k"][2, 0, 0, 0]] == 448 and c["v_scale"][2, 0] == 2.0 ** -8
    od.append(c, None, row(3 * 448), row(0), [], False, [0, 1], [2], table, 4)
    assert c["k_scale"][2, 0] == 4 and od.VALUES[c["k"][2, 0, 0, 0]] == 112 and od.VALUES[c["k"][2, 0, 1, 0]] == 320  # 336 is a tie
    assert c["v_scale"][2, 0] == 2.0 ** -8 and c["k"][2, 0, 2, 0] == 0x7F
    od.append(c, None, np.concatenate([row(2), row(3), row(5)]), np.concatenate([row(1)] * 3), [], False, [0, 3], [5], table, 4)
    assert c["k_scale"][2, 0] == 4 and c["k_scale"][0, 0] == 2.0 ** -6     # 5 <= 448 / 64
    assert od.VALUES[c["k"][0, 0, 0, 0]] * c["k_scale"][0, 0] == 5 and c["k"][0, 0, 1, 0] == 0x7F and c["k"][1, 0, 0, 0] == 0x7F


def test_attention_is_softmax_attention():
    rng = np.random.default_rng(1)
    c = empty_cache(6, 2, 4, 16)
    k, v = rng.standard_normal((11, 2, 16)), rng.standard_normal((11, 2, 16))
    table = [[5, 1, 3, -1]]
    od.append(c, None, k, v, [], False, [0, 11], [11], table, 4)
    deq = lambda n: np.concatenate([od.VALUES[c[n][p]] * c[n + "_scale"][p][:, None, None] for p in (5, 1, 3)], 1)[:, :11]  # noqa: E731
    q = rng.standard_normal((3, 4, 16))
    mask = torch.arange(11)[None] <= torch.arange(8, 11)[:, None]
    want = torch.nn.functional.scaled_dot_product_attention(torch.from_numpy(q).permute(1, 0, 2), torch.from_numpy(deq("k")).repeat_interleave(2, 0),
                                                            torch.from_numpy(deq("v")).repeat_interleave(2, 0), attn_mask=mask).permute(1, 0, 2)
    out, lse, absolute, _ = od.attend(c, q, [0, 3], [11], table, 4, 0.25)
    assert np.allclose(out, want.numpy(), atol=1e-12) and (absolute >= np.abs(out) - 1e-12).all()
    one, lse1, *_ = od.attend(c, q[2:], [0, 1], [11], table, 4, 0.25, window=1)  # sees itself only
    assert np.allclose(one[0], deq("v").repeat(2, 0)[:, 10])
    none, lse0, *_ = od.attend(c, q, [0, 3], [0], table, 4, 0.25)
    assert not none.any() and (lse0 == -np.inf).all()


def test_sampling_by_hand():
    row = np.log(np.array([0.1, 0.4, 0.2, 0.3]))
    draw = lambda u, **kw: od.sample(row, u, **kw)[0]  # noqa: E731
    assert [draw(u) for u in (0.0, 0.099, 0.101, 0.499, 0.501, 0.699, 0.701, 0.999)] == [0, 0, 1, 1, 2, 2, 3, 3]
    assert [draw(u, top_k=2) for u in (0.0, 0.57, 0.58, 0.99)] == [1, 1, 3, 3]      # 0.4 and 0.3 stay
    assert [draw(u, top_p=0.69) for u in (0.0, 0.58)] == [1, 3]
    assert [draw(u, top_p=0.71) for u in (0.45, 0.46)] == [2, 2]                  # 0.4, 0.2, 0.3 of 0.9
    assert draw(0.999, top_p=1e-9) == 1 and draw(0.999, min_p=0.8) == 1 and draw(0.999, min_p=2.0) == 1
    assert draw(0.999, temperature=0.0) == 1
    assert od.sample(row, 0.2)[1] == pytest.approx(math.log(0.4))
    ties = np.array([1.0, 3.0, 3.0, 3.0, -np.inf, np.nan])
    assert [od.sample(ties, u, top_k=2)[0] for u in (0.0, 0.49, 0.51, 0.99)] == [1, 1, 2, 2]
    assert od.sample(np.array([-np.inf, np.nan]), 0.5) == (-1, -math.inf)
    assert od.sample(np.array([0.0, np.inf, np.inf]), 0.6)[0] == 2


def test_bounds_leave_out_and_move_nothing():
    """With max_q and max_kv: the rows that are kept are those of the whole call over the keys that are kept, and appending writes a part of what the
    whole append writes."""
    rng = np.random.default_rng(2)
    table, f = [[5, 1, 3, -1]], 10000.0 ** (-np.arange(8) / 8)
    k, v, q = rng.standard_normal((11, 2, 16)), rng.standard_normal((11, 2, 16)), rng.standard_normal((11, 4, 16))
    whole, part = empty_cache(6, 2, 4, 16), empty_cache(6, 2, 4, 16)
    turned = od.append(whole, q, k, v, f, False, [0, 11], [11], table, 4)
    first = od.append(part, q, k, v, f, False, [0, 11], [11], table, 4, max_q=8)
    assert np.array_equal(first[:8], turned[:8]) and np.array_equal(first[8:], q[8:])
    for p, rows in ((5, 4), (1, 4), (3, 0)):
        assert np.array_equal(part["k"][p, :, :rows], whole["k"][p, :, :rows]) and (part["k"][p, :, rows:] == 0x7F).all()
    out, lse, *_ = od.attend(whole, turned, [0, 11], [11], table, 4, 0.25)
    few, few_lse, *_ = od.attend(part, first, [0, 11], [11], table, 4, 0.25, max_q=8)
    assert np.array_equal(few[:8], out[:8]) and not few[8:].any() and (few_lse[8:] == -np.inf).all()
    short, *_ = od.attend(whole, turned, [0, 11], [11], table, 4, 0.25, max_kv=6)
    cross, *_ = od.attend(whole, turned[6:], [0, 5], [6], table, 4, 0.25, causal=False)
    assert np.array_equal(short[:6], out[:6]) and np.allclose(short[6:], cross, atol=1e-15)
