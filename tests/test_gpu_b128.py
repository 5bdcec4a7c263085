"""Selection of experts, and products of e4m3 operands in blocks of 128, against the 64-bit oracle (oracle/b128.py).

Tolerances.  Selected experts, e4m3 bytes and scale bytes are equal.  Weights are rounded once to fp32: 2^-24 of them, and 2^-40 for the 64-bit
arithmetic in front of that.  A product's sum of K numbers in fp32 is off by less than K * 2^-24 of the sum of their absolute values (S); the
8-bit matrix instruction aligns 8 products to the largest and drops what is below 2^-14 of it or a neighbouring bit: of each of the other 7 less than
2^-13 of the largest, 7 * 2^-13 < 2^-10 of S; results are rounded to bf16 (2^-8 of them) or fp32 (2^-24).  What sums that are off by so much can move in the
feed-forward is the oracle's bound."""
import math

import numpy as np
import pytest
import torch

from oracle import b128
from paper_2303_06182_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32
DROPPED = 2.0 ** -10


def host(t):
    return t.double().cpu().numpy()


# ---- selection
def check_select(logits, k, bias=None, **kw):
    idx, w = binding.moe_select_experts(logits, k, bias=None if bias is None else torch.tensor(np.asarray(bias, np.float32), device=DEV), **kw)
    want, ww = b128.select(host(logits), k, bias=None if bias is None else np.asarray(bias, np.float32), **kw)
    assert np.array_equal(idx.cpu().numpy(), want)
    got = host(w)
    assert (np.abs(got - ww) <= np.abs(ww) * (2.0 ** -24 + 2.0 ** -40) + 2.0 ** -149).all()


@pytest.mark.parametrize("E,G,kept,k", [(1, 1, 1, 1), (2, 1, 1, 2), (8, 8, 3, 3), (20, 4, 2, 5), (63, 9, 4, 8), (64, 8, 8, 6), (128, 8, 4, 8), (130, 10, 3, 8), (256, 8, 4, 8),
                                        (510, 51, 7, 2), (512, 64, 1, 8), (1024, 1, 1, 8), (1024, 64, 5, 7), (1000, 50, 2, 8)])
@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_select(E, G, kept, k, score, dtype):
    rng = np.random.default_rng(E + G)
    x = torch.tensor(rng.standard_normal((37, E)) * 1.5, device=DEV).to(dtype)
    bias = rng.standard_normal(E) * 0.2
    check_select(x, k, score=score, n_groups=G, groups_kept=kept, group_top=1)
    check_select(x, k, bias=bias, score=score, n_groups=G, groups_kept=kept, group_top=2, scale=2.5)
    check_select(x[:1], k, bias=bias, score=score, n_groups=G, groups_kept=kept, renormalize=False)
    wide = torch.full((37, E + 3), 50.0, device=DEV, dtype=dtype)
    wide[:, 1:E + 1] = x
    check_select(wide[:, 1:E + 1], k, bias=bias, score=score, n_groups=G, groups_kept=kept, scale=-1.0)  # rows at any element


@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
def test_select_ties(score):
    """Equal keys, equal groups, keys that 32 bits cannot tell apart, scores near 1 and 0."""
    rng = np.random.default_rng(5)
    E = 128
    rows = [np.zeros(E), np.arange(E) % 3, np.full(E, 20.0), np.where(np.arange(E) % 2, 17.0, 17.0 + 2.0 ** -19), np.full(E, -100.0), np.arange(E) * -8.0,
            np.where(np.arange(E) == 100, 3e38, -3e38), np.full(E, -3.4e38), np.repeat(rng.standard_normal(16), 8), 10 + rng.integers(0, 4, E) * 2.0 ** -20]
    x = torch.tensor(np.array(rows), device=DEV).float()
    for kw in (dict(), dict(n_groups=8, groups_kept=3), dict(n_groups=16, groups_kept=2, group_top=1)):
        check_select(x, 8, score=score, **kw)
        check_select(x, 8, score=score, bias=np.arange(E) % 5 * 0.125, **kw)
        check_select(x, 8, score=score, bias=np.round(rng.standard_normal(E) * 2.0 ** 20) * 2.0 ** -44, **kw)  # far below a bit of fp32 scores


@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
def test_select_infinities_and_nan(score):
    inf, nan = math.inf, math.nan
    E = 96
    rng = np.random.default_rng(6)
    x = rng.standard_normal((12, E))
    x[0] = -inf
    x[1] = nan
    x[2, 5:] = -inf
    x[3, ::2] = nan
    x[4, 7] = inf
    x[5, 3::9] = inf
    x[6, :90] = -inf
    x[7] = inf
    x[8, 0], x[8, 1] = inf, nan
    x[9, 24:] = -inf
    x[10, :] = -inf
    x[10, 95] = -3e38
    bias = rng.standard_normal(E) * 0.1
    spoiled = bias.copy()
    spoiled[[3, 40, 41]], spoiled[50], spoiled[7] = -inf, nan, inf
    t = torch.tensor(x, device=DEV).float()
    for b in (None, bias, spoiled):
        for kw in (dict(), dict(n_groups=12, groups_kept=2), dict(n_groups=12, groups_kept=2, group_top=1), dict(renormalize=False, n_groups=4, groups_kept=3)):
            check_select(t, 8, bias=b, score=score, **kw)


@pytest.mark.parametrize("E,G,kept,k,top", [(1, 1, 1, 1, 1), (5, 1, 1, 2, 1), (16, 4, 2, 2, 2), (64, 8, 8, 6, 1), (100, 10, 3, 8, 2), (128, 8, 3, 6, 2), (128, 1, 1, 8, 1), (130, 13, 4, 3, 1),
                                                (256, 64, 9, 8, 2), (257, 1, 1, 4, 1), (512, 16, 5, 8, 2), (1024, 64, 64, 8, 1), (1023, 1, 1, 1, 1)])
@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
def test_select_many_tokens(E, G, kept, k, top, score):
    """Batches of thousands of tokens: as the same rows in small batches, which the tests above hold against the oracle; rows with ties, infinities, NaN, numbers
    far apart and a last, partly filled group of rows among them."""
    g = torch.Generator(device=DEV).manual_seed(E + k)
    T = 6157
    x = torch.randn((T, E), device=DEV, generator=g) * 1.5
    x[::7] = x[::7].bfloat16().float()                 # equal logits here and there
    x[3::11] = (x[3::11] * 2).round() / 2              # and in most places
    x[5::13] *= 40.0
    x[6::17] = x[6::17].masked_fill(torch.rand((len(range(6, T, 17)), E), device=DEV, generator=g) < 0.6, -math.inf)
    x[100], x[101], x[102], x[103], x[104] = 0.0, -math.inf, math.nan, 1e30, math.inf
    x[105, ::2], x[106, ::3], x[107, 0] = math.nan, math.inf, math.inf
    x[108:140] = x[108:109]
    bias = torch.randn(E, device=DEV, generator=g) * 0.1
    odd = bias.clone()
    odd[::5] = -math.inf
    if E > 3:
        odd[1], odd[3] = math.inf, math.nan
    kw = dict(score=score, n_groups=G, groups_kept=kept, group_top=top)
    for b in (None, bias, bias * 1e6, odd):
        for renormalize in (True, False):
            for logits in (x, x.bfloat16(), torch.cat([x, x], 1)[:, 1:E + 1]):
                idx, w = binding.moe_select_experts(logits, k, bias=b, renormalize=renormalize, **kw)
                parts = [binding.moe_select_experts(logits[i:i + 2053], k, bias=b, renormalize=renormalize, **kw) for i in range(0, T, 2053)]
                assert torch.equal(idx, torch.cat([i for i, _ in parts]))
                # sums of 64 bits in another order: the weights are the same but where they lie within 2^-45 of a border between two fp32 numbers
                other = torch.cat([v for _, v in parts])
                assert torch.allclose(w, other, rtol=2.0 ** -23, atol=0.0) and (w != other).sum() <= 4
    if E <= 16:  # and the oracle itself
        check_select(x[:160].repeat(40, 1), k, bias=host(bias), **kw)


def test_select_many_tokens_twice_and_captured():
    """More rows than the launch has waves; the same again, and from a graph, into the same tensors."""
    g = torch.Generator(device=DEV).manual_seed(1)
    x = torch.randn((300001, 16), device=DEV, generator=g)
    bias = torch.randn(16, device=DEV, generator=g) * 0.1
    idx, w = binding.moe_select_experts(x, 2, bias=bias, n_groups=4, groups_kept=2)
    key = torch.sigmoid(x.double()) + bias.double()
    best = key.view(-1, 4, 4).topk(2, dim=2).values.sum(2).topk(2, dim=1).indices
    out = torch.ones((len(x), 4), dtype=torch.bool, device=DEV).scatter_(1, best, False)
    want = key.masked_fill(out.repeat_interleave(4, 1), -math.inf).topk(2, dim=1).indices
    assert torch.equal(idx.long(), want)
    i2, w2 = torch.empty_like(idx), torch.empty_like(w)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.moe_select_experts(x, 2, bias=bias, n_groups=4, groups_kept=2, topk_idx=i2, topk_w=w2)
    for _ in range(3):
        i2.zero_(), w2.zero_()
        graph.replay()
        assert torch.equal(i2, idx) and torch.equal(w2, w)


# ---- quantisation
def check_quantize(x, block_rows):
    q, scale = binding.moe_quantize_b128(x, block_rows=block_rows)
    assert q.dtype == torch.float8_e4m3fn and q.shape == x.shape
    xs = host(x).reshape((-1,) + tuple(x.shape[-2:]))
    for m in range(len(xs)):
        number, byte = b128.quantize(xs[m], block_rows)
        assert np.array_equal(scale.cpu().numpy().reshape((-1,) + byte.shape)[m], byte)
        assert np.array_equal(host(q).reshape(xs.shape)[m], number, equal_nan=True)


@pytest.mark.parametrize("rows,cols", [(1, 16), (3, 112), (5, 128), (2, 144), (17, 512), (33, 528), (70, 1200), (130, 2000), (1, 16384)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_quantize(rows, cols, dtype):
    g = torch.Generator(device=DEV).manual_seed(rows + cols)
    x = torch.randn((rows, cols), device=DEV, generator=g) * torch.exp2(torch.randint(-20, 20, (rows, 1), device=DEV, generator=g).float())
    x[:, ::37] *= 64
    x = x.to(dtype)
    check_quantize(x, 1)
    check_quantize(x, 128)
    wide = torch.full((rows, cols + 40), 1e30, device=DEV, dtype=dtype)
    wide[:, 16:cols + 16] = x
    check_quantize(wide[:, 16:cols + 16], 1)
    check_quantize(wide[:, 16:cols + 16], 128)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_quantize_matrices(dtype):
    g = torch.Generator(device=DEV).manual_seed(3)
    x = (torch.randn((2, 3, 200, 160), device=DEV, generator=g) * 0.02).to(dtype)
    for block_rows in (1, 128):
        check_quantize(x, block_rows)
        check_quantize(x[:, :, :, 16:], block_rows)
        check_quantize(x[1], block_rows)
    with pytest.raises(ValueError):
        binding.moe_quantize_b128(x[:, :, :100])  # a gap between the matrices
    q, scale = binding.moe_quantize_b128(x[:, :, :0], block_rows=128)
    assert q.shape == (2, 3, 0, 160) and scale.shape == (2, 3, 0, 4)


def test_quantize_extremes():
    """Blocks of zeros, of the smallest and largest numbers, borders between two scales, infinities and NaN, ties."""
    inf, nan = math.inf, math.nan
    x = torch.zeros((16, 384), device=DEV)
    x[1] = 448.0
    x[2, :128], x[2, 128:256], x[2, 256:] = 448.00003, 1.75 * 2.0 ** -3, 1.7500001 * 2.0 ** -3
    x[3, 5], x[3, 200] = torch.finfo(F32).max, torch.finfo(F32).min
    x[4, 0], x[4, 130], x[4, 300] = 1e-45, 1.1754942e-38, -1.1754944e-38
    x[5, 1], x[5, 2], x[5, 140] = inf, -inf, nan
    x[6, :128], x[6, 128:] = nan, 1.0
    x[7, 0], x[7, 1:] = inf, torch.arange(383, device=DEV).float()
    x[8] = torch.arange(384, device=DEV).float() - 192.0
    x[9] = -0.0
    x[10, :128] = 448.0 * 2.0 ** -126
    x[11, :128] = 1.0 + torch.arange(128, device=DEV) / 64.0
    check_quantize(x, 1)
    check_quantize(x, 128)
    check_quantize(x.bfloat16(), 1)


def test_quantize_into_given_outputs_leaves_the_rest():
    x = torch.randn((4, 256), device=DEV)
    q = torch.full((6, 256), 99, dtype=torch.uint8, device=DEV)
    scale = torch.full((6, 4), 99, dtype=torch.uint8, device=DEV)
    binding.moe_quantize_b128(x, q=q[1:5].view(torch.float8_e4m3fn), scale=scale[1:5])
    assert (q[[0, 5]] == 99).all() and (scale[[0, 5]] == 99).all() and (scale[1:5, 2:] == 127).all() and (scale[1:5, :2] != 99).all()


# ---- products
def operands(rows, E, N, K, seed, halves=(), spread=3):
    rng = np.random.default_rng(seed)
    a = b128.e4m3(np.clip(rng.standard_normal((rows, K)) * 100, -448, 448))
    w = b128.e4m3(np.clip(rng.standard_normal((E, *halves, N, K)) * 100, -448, 448))
    sa = rng.integers(119, 119 + spread, (rows, -(-K // 512) * 4)).astype(np.uint8)
    sw = rng.integers(116, 116 + spread, (E, *halves, -(-N // 128), -(-K // 512) * 4)).astype(np.uint8)
    av = b128.value(a, sa)
    flat_w, flat_s = w.reshape(-1, N, K), sw.reshape(-1, sw.shape[-2], sw.shape[-1])
    wv = np.stack([b128.value(m, s, 128) for m, s in zip(flat_w, flat_s)]).reshape(w.shape)
    dev = lambda x: torch.tensor(x, device=DEV).float().to(torch.float8_e4m3fn)  # noqa: E731
    byte = lambda x: torch.tensor(x, device=DEV)  # noqa: E731
    return (dev(a), byte(sa), av), (dev(w), byte(sw), wv)


def split(rows, E, seed):
    """Offsets of E experts, some of them empty."""
    rng = np.random.default_rng(seed)
    cuts = np.sort(rng.integers(0, rows + 1, E - 1)) if E > 1 else np.array([], dtype=int)
    return [0] + cuts.tolist() + [rows]


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def check_sums(got, want, size, K, dtype):
    got = host(got)
    half = 2.0 ** -8 if dtype == BF16 else 2.0 ** -24
    bound = half * np.abs(want) + (K * 2.0 ** -24 + (DROPPED if dtype == BF16 else 0.0)) * size * (1 + half) + 2.0 ** -120
    assert (np.abs(got - want) <= bound).all(), float((np.abs(got - want) / bound).max())
    norm = np.sqrt(((got - want) ** 2).sum() / max((want ** 2).sum(), 1e-300))
    assert norm <= (2.0 ** -8 if dtype == BF16 else K * 2.0 ** -24), norm


@pytest.mark.parametrize("rows,E,N,K", [(1, 1, 8, 16), (1, 1, 64, 128), (3, 2, 24, 112), (16, 1, 128, 144), (17, 3, 136, 256), (40, 1, 256, 528), (65, 5, 200, 384),
                                        (100, 70, 40, 128), (130, 1, 264, 640), (257, 4, 520, 272), (300, 2, 136, 1040), (700, 3, 392, 400), (33, 9, 1640, 1200)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_gemm(rows, E, N, K, dtype):
    (a, sa, av), (w, sw, wv) = operands(rows, E, N, K, rows + N + K)
    offsets = split(rows, E, rows)
    want, size = b128.gemm(av, wv, offsets)
    check_sums(binding.moe_gemm_b128(a, sa, w, sw, offsets=ints(offsets), out_dtype=dtype), want, size, K, dtype)
    if E == 1:
        check_sums(binding.moe_gemm_b128(a, sa, w[0], sw[0], out_dtype=dtype), want, size, K, dtype)
    # rows by index: some twice, some never; those outside the array are the nearest that is in it
    pick = np.random.default_rng(K).integers(0, rows, rows + 5)
    offsets = split(rows + 5, E, rows + 1)
    want, size = b128.gemm(av, wv, offsets, pick)
    asked = pick.copy()
    asked[pick == 0] = -7
    asked[pick == rows - 1] = rows + 1000
    check_sums(binding.moe_gemm_b128(a, sa, w, sw, offsets=ints(offsets), a_rows=ints(asked), out_dtype=dtype), want, size, K, dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows", [9, 200])
def test_gemm_leaves_other_rows(dtype, rows):
    """Rows outside the experts' ranges are left as they are; offsets outside the rows are taken as the nearest inside; empty experts are not read."""
    (a, sa, av), (w, sw, wv) = operands(rows, 4, 72, 160, 1)
    w.view(torch.uint8)[2] = 0x7f
    sw[2] = 200
    out = torch.full((rows, 72), 7.0, dtype=dtype, device=DEV)
    lo, mid, hi = 2, rows // 2, rows - 3
    binding.moe_gemm_b128(a, sa, w, sw, offsets=ints([lo, lo, mid, mid, hi]), out=out)
    want, size = b128.gemm(av, wv, [lo, lo, mid, mid, hi])
    check_sums(out[lo:hi], want[lo:hi], size[lo:hi], 160, dtype)
    assert (out[:lo] == 7).all() and (out[hi:] == 7).all()
    out.fill_(7.0)
    binding.moe_gemm_b128(a, sa, w, sw, offsets=ints([-5, 3, rows + 9, rows + 7, rows + 20]), out=out)
    want, size = b128.gemm(av, wv, [0, 3, rows, rows, rows])
    check_sums(out, want, size, 160, dtype)
    out.fill_(7.0)
    binding.moe_gemm_b128(a, sa, w, sw, offsets=ints([0, 0, 0, 0, 0]), out=out)
    assert (out == 7).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows", [5, 300])
def test_gemm_nan_stays_in_its_row(dtype, rows):
    """A NaN in a row of A spoils that row, one in a row of W that column, and nothing behind the last element of a row or matrix is read into one."""
    (a, sa, av), (w, sw, wv) = operands(rows, 1, 40, 144, 2)
    want, size = b128.gemm(av, wv, [0, rows])
    a.view(torch.uint8)[3, 143] = 0x7f
    w.view(torch.uint8)[0, 17, 0] = 0xff
    got = binding.moe_gemm_b128(a, sa, w, sw, out_dtype=dtype)
    assert got[3].isnan().all() and got[:, 17].isnan().all()
    keep_r, keep_c = [r for r in range(rows) if r != 3], [c for c in range(40) if c != 17]
    check_sums(got[keep_r][:, keep_c], want[np.ix_(keep_r, keep_c)], size[np.ix_(keep_r, keep_c)], 144, dtype)


@pytest.mark.parametrize("rows,E,N,K", [(2000, 3, 512, 128), (1500, 2, 776, 112), (3000, 1, 264, 16), (900, 5, 1032, 80)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_gemm_one_block_of_k(rows, E, N, K, dtype):
    """Rows of one block and less, many of them; what stands in the scales' padding plays no part."""
    (a, sa, av), (w, sw, wv) = operands(rows, E, N, K, 5)
    sa[:, 1:] = 255
    sw[:, :, 1:] = 255
    offsets = split(rows, E, 6)
    want, size = b128.gemm(av, wv, offsets)
    check_sums(binding.moe_gemm_b128(a, sa, w, sw, offsets=ints(offsets), out_dtype=dtype), want, size, K, dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_gemm_rows_past_32_bits(dtype):
    K, N, rows = 8192, 264, 2 ** 32 // 8192 + 300
    (a, sa, av), (w, sw, wv) = operands(300, 1, N, K, 7)
    long, scales = torch.zeros((rows, K), dtype=torch.uint8, device=DEV), torch.full((rows, sa.shape[1]), 127, dtype=torch.uint8, device=DEV)
    long[-300:] = a.view(torch.uint8)
    scales[-300:] = sa
    long = long.view(torch.float8_e4m3fn)
    want, size = b128.gemm(av, wv, [0, 300])
    got = binding.moe_gemm_b128(long, scales, w[0], sw[0], out_dtype=dtype)
    assert (got[:-300] == 0).all()
    check_sums(got[-300:], want, size, K, dtype)
    pick = np.arange(rows - 1, rows - 300, -7)
    check_sums(binding.moe_gemm_b128(long, scales, w[0], sw[0], a_rows=ints(pick), out_dtype=dtype), want[pick - rows], size[pick - rows], K, dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_gemm_scales_far_apart(dtype):
    """Scale bytes over a wide range, the blocks of a row far from each other: small blocks beside large ones count as fp32 lets them."""
    (a, sa, av), (w, sw, wv) = operands(48, 2, 136, 528, 3, spread=1)
    rng = np.random.default_rng(0)
    sa2, sw2 = rng.integers(87, 160, sa.shape).astype(np.uint8), rng.integers(87, 160, sw.shape).astype(np.uint8)
    av = b128.value(host(a), sa2)
    wv = np.stack([b128.value(host(w[e]), sw2[e], 128) for e in range(2)])
    offsets = [0, 20, 48]
    want, size = b128.gemm(av, wv, offsets)
    got = host(binding.moe_gemm_b128(a, torch.tensor(sa2, device=DEV), w, torch.tensor(sw2, device=DEV), offsets=ints(offsets), out_dtype=dtype))
    bound = (2.0 ** -8 if dtype == BF16 else 2.0 ** -24) * np.abs(want) + (528 * 2.0 ** -24 + (DROPPED if dtype == BF16 else 0)) * size * 1.01
    assert (np.abs(got - want) <= bound).all()


# ---- the experts' feed-forward, and the layer
def ffn_case(T, rows, E, D, F, activation, dtype, seed):
    halves = (2,) if activation == "silu" else ()
    _, (w1, s1, v1) = operands(1, E, F, D, seed, halves)
    _, (w2, s2, v2) = operands(1, E, D, F, seed + 1)
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randn((T, D), device=DEV, generator=g)
    x[:, ::37] *= 8
    x = x.to(dtype)
    # about unit sums: 2^-7 * 100 is 0.8 a weight, so x is made small
    x = (x.float() * 2.0 ** -7 / math.sqrt(D)).to(dtype)
    src = np.random.default_rng(seed).integers(0, T, rows)
    return x, src, (w1, w2, s1, s2), (v1, v2), split(rows, E, seed)


def check_ffn(y, x, src, values, offsets, activation, dtype, K):
    xv = b128.value(*b128.quantize(host(x)))
    error = K * 2.0 ** -24 + (DROPPED if dtype == BF16 else 0.0)
    want, moved = b128.ffn(xv, values[0], values[1], offsets, activation, src, sum_error=error)
    got, half = host(y), 2.0 ** -8 if dtype == BF16 else 2.0 ** -24
    assert (np.abs(got - want) <= half * np.abs(want) + moved * (1 + half) + 2.0 ** -120).all()
    # All together: rounding (2^-8 at most) and hidden elements near a border of e4m3 that fall to the other side.  Sums that are off by 1.4e-5 of their
    # deviation do that to a few in 10^4, by a step (2^-3 of the element at most): sqrt(1e-3) * 2^-3 = 2^-8; fp32 sums (2^-22) to sqrt(2^-22 * 8) * 2^-3 = 2^-12.
    norm = np.sqrt(((got - want) ** 2).sum() / max((want ** 2).sum(), 1e-300))
    assert norm <= (2.0 ** -7 if dtype == BF16 else 2.0 ** -12), norm


@pytest.mark.parametrize("T,rows,E,D,F", [(1, 1, 1, 16, 16), (1, 4, 8, 128, 144), (5, 10, 4, 144, 128), (20, 40, 3, 272, 208), (64, 130, 70, 64, 96), (150, 300, 2, 256, 384),
                                          (300, 600, 3, 400, 272)])
@pytest.mark.parametrize("activation", ["relu", "silu"])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_ffn(T, rows, E, D, F, activation, dtype):
    x, src, weights, values, offsets = ffn_case(T, rows, E, D, F, activation, dtype, T + D)
    layer = binding.MoeLayer(max(T, rows), D, F, E, 1, "bf16" if dtype == BF16 else "f32", alloc_workspace=False)
    y = layer.moe_expert_ffn_b128(x, ints(offsets), *weights, activation=activation, src_tok=ints(src))
    check_ffn(y, x, src, values, offsets, activation, dtype, max(D, F))
    again = layer.moe_expert_ffn_b128(x, ints(offsets), *weights, activation=activation, src_tok=ints(src))
    assert torch.equal(y, again)
    # the rows themselves, as a dispatch has laid them out
    assert torch.equal(layer.moe_expert_ffn_b128(x[ints(src).long()].contiguous(), ints(offsets), *weights, activation=activation), y)


@pytest.mark.parametrize("T,E,D,F", [(600, 4, 64, 48), (400, 3, 528, 128), (500, 5, 128, 400)])
@pytest.mark.parametrize("activation", ["relu", "silu"])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_ffn_narrow(T, E, D, F, activation, dtype):
    """One block of 128 and less, of rows or of hidden elements, and rows enough for tiles."""
    test_ffn(T, T + 100, E, D, F, activation, dtype)


def test_ffn_leaves_other_rows_and_refuses():
    x, src, weights, values, _ = ffn_case(30, 40, 4, 128, 128, "silu", BF16, 1)
    layer = binding.MoeLayer(40, 128, 128, 4, 1, "bf16", alloc_workspace=False)
    offsets = [0, 9, 9, 20, 33]
    y = torch.full((40, 128), 3.0, dtype=BF16, device=DEV)
    layer.moe_expert_ffn_b128(x, ints(offsets), *weights, src_tok=ints(src), yp=y)
    check_ffn(y[:33], x, src[:33], values, offsets, "silu", BF16, 128)
    assert (y[33:] == 3).all()
    w1, w2, s1, s2 = weights
    for call in (lambda: layer.moe_expert_ffn_b128(x, ints(offsets), w1, w2, s1, s2, activation="gelu"),
                 lambda: layer.moe_expert_ffn_b128(x, ints(offsets), w1, w2, s1, s2, activation="relu"),
                 lambda: layer.moe_expert_ffn_b128(x.float(), ints(offsets), *weights), lambda: layer.moe_expert_ffn_b128(x, ints(offsets).long(), *weights),
                 lambda: layer.moe_expert_ffn_b128(x, ints(offsets), w1, w2, s1[:, :, :, :2], s2), lambda: layer.moe_expert_ffn_b128(x.cpu(), ints(offsets), *weights),
                 lambda: layer.moe_expert_ffn_b128(x, ints(offsets), *weights, src_tok=ints(src), yp=y.float())):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(binding.MoeError):
        layer.moe_expert_ffn_b128(torch.zeros((41, 128), dtype=BF16, device=DEV), ints(offsets), *weights)  # more than k * T_max
    with pytest.raises(binding.MoeError):
        binding.MoeLayer(40, 120, 128, 4, 1, "bf16", alloc_workspace=False).moe_expert_ffn_b128(x[:, :120].contiguous(), ints(offsets), *[
            t for t in (torch.zeros((4, 2, 128, 120), dtype=torch.uint8, device=DEV), torch.zeros((4, 120, 128), dtype=torch.uint8, device=DEV),
                        torch.full((4, 2, 1, 4), 127, dtype=torch.uint8, device=DEV), torch.full((4, 1, 4), 127, dtype=torch.uint8, device=DEV))])
    assert layer.moe_expert_ffn_b128(x[:0], ints([0] * 5), *weights).shape == (0, 128)


@pytest.mark.parametrize("T", [1, 7, 64, 300, 700])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("score,G,kept,activation", [("sigmoid", 4, 2, "silu"), ("softmax", 1, 1, "relu")])
def test_layer(T, dtype, score, G, kept, activation):
    """The whole layer: its logits select as moe_select_experts does, its routing is the plain one, its output the weighted sum of the experts'."""
    E, D, F, k = 24, 256, 144, 3
    x, _, weights, values, _ = ffn_case(T, 1, E, D, F, activation, dtype, T)
    g = torch.Generator(device=DEV).manual_seed(7)
    wg = (torch.randn((E, D), device=DEV, generator=g) * 40).to(dtype)
    gate_bias, select_bias = torch.randn(E, device=DEV, generator=g) * 0.1, torch.randn(E, device=DEV, generator=g) * 0.1
    layer = binding.MoeLayer(T, D, F, E, k, "bf16" if dtype == BF16 else "f32", alloc_workspace=False)
    kw = dict(score=score, n_groups=G, groups_kept=kept, scale=1.5)
    r = layer.empty_routing(T)
    y = layer.moe_layer_forward_b128(x, wg, *weights, activation=activation, gate_bias=gate_bias, select_bias=select_bias, routing_out=r, **kw)
    logits = host(r["logits"])
    want = host(x) @ host(wg).T + host(gate_bias)
    assert (np.abs(logits - want) <= D * 2.0 ** -24 * (np.abs(host(x)) @ np.abs(host(wg)).T + 1)).all()
    idx, w = b128.select(logits, k, bias=host(select_bias), **kw)
    assert np.array_equal(r["topk_idx"].cpu().numpy(), idx)
    order = np.argsort(idx.ravel(), kind="stable")
    assert np.array_equal(r["src_tok"].cpu().numpy(), order // k)
    offsets = np.concatenate([[0], np.cumsum(np.bincount(idx.ravel(), minlength=E))]).tolist()
    assert r["offsets"].cpu().tolist() == offsets
    yp = layer.moe_expert_ffn_b128(x, r["offsets"], *weights, activation=activation, src_tok=r["src_tok"])
    check_ffn(yp, x, order // k, values, offsets, activation, dtype, max(D, F))
    parts = host(yp)[r["dst_row"].cpu().numpy()]
    total, size = (parts * w[:, :, None]).sum(1), np.abs(parts * w[:, :, None]).sum(1)
    half = 2.0 ** -8 if dtype == BF16 else 2.0 ** -24
    assert (np.abs(host(y) - total) <= half * np.abs(total) + 2 * k * 2.0 ** -24 * size + 2.0 ** -120).all()
    # without the routing's outputs, and captured: the same
    assert torch.equal(layer.moe_layer_forward_b128(x, wg, *weights, activation=activation, gate_bias=gate_bias, select_bias=select_bias, **kw), y)
    out, x2 = torch.empty_like(y), x.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.moe_layer_forward_b128(x2, wg, *weights, activation=activation, gate_bias=gate_bias, select_bias=select_bias, y=out, **kw)
    for i in range(3):
        x2.copy_(x.flip(0) if i == 1 else x)
        graph.replay()
        if i == 1:
            eager = layer.moe_layer_forward_b128(x.flip(0).contiguous(), wg, *weights, activation=activation, gate_bias=gate_bias, select_bias=select_bias, **kw)
            assert torch.equal(out, eager)
        else:
            assert torch.equal(out, y)


def test_layer_without_tokens_and_refusals():
    x, _, weights, _, _ = ffn_case(4, 1, 8, 128, 128, "silu", BF16, 0)
    wg = torch.randn((8, 128), device=DEV).to(BF16)
    layer = binding.MoeLayer(4, 128, 128, 8, 2, "bf16", alloc_workspace=False)
    r = layer.empty_routing(0)
    r["counts"].fill_(9)
    assert layer.moe_layer_forward_b128(x[:0], wg, *weights, routing_out=r).shape == (0, 128)
    assert (r["counts"] == 0).all() and (r["offsets"] == 0).all()
    for kw in (dict(n_groups=3), dict(n_groups=4, groups_kept=0), dict(group_top=3)):
        with pytest.raises(binding.MoeError):
            layer.moe_layer_forward_b128(x, wg, *weights, **kw)
    for kw in (dict(score="relu"), dict(select_bias=torch.zeros(7, device=DEV)), dict(gate_bias=torch.zeros(8, dtype=torch.float64, device=DEV))):
        with pytest.raises(ValueError):
            layer.moe_layer_forward_b128(x, wg, *weights, **kw)


def test_streams_and_two_handles():
    """Calls on a side stream are in that stream's order; two handles with workspaces of their own run beside each other."""
    x, src, weights, values, offsets = ffn_case(64, 128, 8, 256, 256, "silu", BF16, 5)
    layers = [binding.MoeLayer(128, 256, 256, 8, 1, "bf16", alloc_workspace=False) for _ in range(2)]
    off, at = ints(offsets), ints(src)
    want = layers[0].moe_expert_ffn_b128(x, off, *weights, src_tok=at)
    layers[1].b128_workspace()
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(10):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i].append(layers[i].moe_expert_ffn_b128(x, off, *weights, src_tok=at))
    torch.cuda.synchronize()
    for y in got[0] + got[1]:
        assert torch.equal(y, want)
