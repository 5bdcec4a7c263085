"""Products of e4m3 operands in blocks of 128 by whole tiles, and the streamed feed-forward in several pieces of k, at sizes that are sure to come there: every
test looks up which kernel ran.  Against 64 bits; the tolerances are those of test_gpu_b128.py.

Where the feed-forward streams, both operands of both products are widened: its sums are off by K * 2^-24 of the sum of absolute values for bf16, too, so all results together by the
rounding to bf16 (2^-8 at most) and what hidden elements near a border of e4m3 move, 2^-12 as for fp32 sums there."""
import math

import numpy as np
import pytest
import torch

from oracle import b128
from paper_2303_06182_amd import binding
from test_gpu_b128 import BF16, DEV, DROPPED, F32, check_ffn, host, ints

pytestmark = pytest.mark.gpu
E4M3 = torch.float8_e4m3fn


def kernels(call):
    """What `call` launches, by name, and what it returns."""
    torch.cuda.synchronize()
    with torch.profiler.profile(activities=[torch.profiler.ProfilerActivity.CUDA]) as prof:
        out = call()
        torch.cuda.synchronize()
    return [e.key for e in prof.key_averages() if "kernel" in e.key], out


def in_tiles(dtype, call):
    names, out = kernels(call)
    want = "gemm_b128_tile_kernel<%s, 0, false>" % ("false" if dtype == BF16 else "true")
    assert any(want in n for n in names), names
    return out


def operand(shape, scale_rows, low, high, g):
    q = (torch.randn(shape, device=DEV, generator=g) * 100).clamp_(-448, 448).to(E4M3)
    return q, torch.randint(low, high, (*scale_rows, -(-shape[-1] // 512) * 4), device=DEV, generator=g, dtype=torch.uint8)


def value(q, scale, block_rows):
    """What a matrix [R, C] stands for, in 64 bits."""
    s = torch.exp2(scale.double() - 127).repeat_interleave(block_rows, 0)[:q.shape[0]].repeat_interleave(128, 1)[:, :q.shape[1]]
    return q.double() * s


class Product:
    def __init__(self, count, E, N, K, seed=0, bytes_a=(119, 122), bytes_w=(116, 119)):
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.a, self.sa = operand((count, K), (count,), *bytes_a, g)
        self.w, self.sw = operand((E, N, K), (E, -(-N // 128)), *bytes_w, g)
        self.E, self.N, self.K = E, N, K

    def __call__(self, offsets, **kw):
        return binding.moe_gemm_b128(self.a, self.sa, self.w, self.sw, offsets=ints(offsets), **kw)

    def exact(self, offsets, pick=None):
        """64-bit results and sums of absolute values; NaN in rows that no expert has."""
        av = value(self.a, self.sa, 1)
        rows = len(av) if pick is None else len(pick)
        at = torch.arange(rows, device=DEV) if pick is None else torch.tensor(pick, device=DEV)
        want, size = (torch.full((rows, self.N), math.nan, dtype=torch.float64, device=DEV) for _ in range(2))
        for e in range(self.E):
            lo, hi = offsets[e], offsets[e + 1]
            if lo < hi:
                x, wv = av[at[lo:hi]], value(self.w[e], self.sw[e], 128).t().contiguous()
                want[lo:hi], size[lo:hi] = torch.mm(x, wv), torch.mm(x.abs(), wv.abs())
        return want, size

    def check(self, got, offsets, pick=None, norm=True):
        want, size = self.exact(offsets, pick)
        live = ~want.isnan()
        bf16 = got.dtype == BF16
        half = 2.0 ** -8 if bf16 else 2.0 ** -24
        off = (got.double() - want).abs()
        bound = half * want.abs() + (self.K * 2.0 ** -24 + (DROPPED if bf16 else 0.0)) * size * (1 + half) + 2.0 ** -120
        assert (off <= bound)[live].all(), float((off / bound)[live].max())
        if norm:
            assert off[live].norm() <= (2.0 ** -8 if bf16 else self.K * 2.0 ** -24) * want[live].norm()


def ends(counts):
    return np.concatenate([[0], np.cumsum(counts)]).tolist()


def ragged(rows, E, seed, empty=()):
    """Offsets of E experts, the ones named and a few others without rows."""
    rng = np.random.default_rng(seed)
    weight = rng.random(E) ** 3 * (rng.random(E) < 0.9)
    weight[list(empty)] = 0
    weight[E - 1 if E - 1 not in empty else 0] += 0.5
    return ends(rng.multinomial(rows, weight / weight.sum()))


@pytest.mark.parametrize("rows,E,N,K", [(3000, 2, 1032, 272), (4000, 3, 1640, 400), (5003, 5, 1400, 528), (6000, 4, 1288, 640), (3000, 4, 2056, 144), (6000, 5, 1640, 1040),
                                        (5000, 3, 1640, 1200), (2500, 2, 2056, 2064), (4001, 1, 1640, 1552)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_gemm(rows, E, N, K, dtype):
    """2 to 17 blocks of k, the last one short; ragged experts, rows in order and by index, and the same bits again."""
    p = Product(rows, E, N, K, seed=K)
    offsets = ragged(rows, E, K, empty=[1] if E > 3 else [])
    got = in_tiles(dtype, lambda: p(offsets, out_dtype=dtype))
    p.check(got, offsets)
    assert torch.equal(p(offsets, out_dtype=dtype), got)
    pick = np.random.default_rng(K).integers(0, rows, rows + 77)
    offsets = ragged(rows + 77, E, K + 1)
    asked = pick.copy()
    asked[pick == 0], asked[pick == rows - 1] = -7, rows + 1000
    p.check(in_tiles(dtype, lambda: p(offsets, a_rows=ints(asked), out_dtype=dtype)), offsets, pick)


@pytest.mark.parametrize("counts", [[256, 257, 64, 63, 1, 0, 512, 700], [0, 0, 1, 65, 128, 129, 192, 193, 255, 320, 31, 32, 33, 0], [2049]])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_gemm_tile_heights(counts, dtype):
    """Experts whose rows end at, before and behind the end of a tile or of a block of 32 rows."""
    p = Product(sum(counts), len(counts), 1992, 1104)
    p.check(in_tiles(dtype, lambda: p(ends(counts), out_dtype=dtype)), ends(counts))


@pytest.mark.parametrize("rows,E,N,K,empty", [(4001, 65, 520, 272, ()), (9000, 130, 520, 400, range(64, 128)), (9000, 130, 776, 272, range(0, 128)), (12000, 200, 264, 528, range(10, 150)),
                                              (26000, 1024, 264, 144, range(300, 700)), (40000, 70, 2056, 144, range(1, 69))])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_gemm_more_than_64_experts(rows, E, N, K, empty, dtype):
    """Windows of 64 experts, some with no row at all."""
    p = Product(rows, E, N, K, seed=E)
    offsets = ragged(rows, E, E, empty)
    out = torch.full((rows + 1, N), 7.0, dtype=dtype, device=DEV)
    in_tiles(dtype, lambda: p(offsets, out=out[:rows]))
    p.check(out[:rows], offsets)
    assert (out[rows] == 7).all()


@pytest.mark.parametrize("rows,E,empty", [(20000, 7, (0, 3)), (30000, 80, range(5, 70)), (33000, 1, ()), (21000, 6, (1, 2, 3, 4))])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_gemm_more_than_1024_tiles(rows, E, empty, dtype):
    """Output tiles that are dealt to the XCDs by what they cost: every one of them once."""
    N, K = 4104, 272
    assert rows // 256 * -(-N // 256) > 1024
    p = Product(rows, E, N, K, seed=E)
    offsets = ragged(rows, E, E + 1, empty)
    out = torch.full((rows, N), math.nan, dtype=dtype, device=DEV)
    in_tiles(dtype, lambda: p(offsets, out=out))
    p.check(out, offsets)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_gemm_leaves_other_rows_and_keeps_nan(dtype):
    """Rows outside every expert's are left as they are, an expert without rows is not read, a NaN stays in its row or column, also where rows come by index."""
    rows, N, K = 4000, 1640, 400
    p = Product(rows, 4, N, K, seed=1)
    offsets = [130, 1900, 1900, 3100, 3977]
    p.w.view(torch.uint8)[1] = 0x7f
    p.sw[1] = 254
    clean = torch.full((rows, N), 7.0, dtype=dtype, device=DEV)
    in_tiles(dtype, lambda: p(offsets, out=clean))
    p.check(clean, offsets)
    assert (clean[:130] == 7).all() and (clean[3977:] == 7).all()
    p.a.view(torch.uint8)[[131, 2050, 3976], [0, 399, 130]] = 0x7f
    p.w.view(torch.uint8)[2, 1639, 399] = 0xff
    spoiled = torch.zeros((rows, N), dtype=torch.bool, device=DEV)
    spoiled[[131, 2050, 3976]], spoiled[1900:3100, 1639] = True, True
    got = torch.full_like(clean, 7.0)
    in_tiles(dtype, lambda: p(offsets, out=got))
    assert torch.equal(got.isnan(), spoiled) and torch.equal(got[~spoiled], clean[~spoiled])
    back = torch.arange(rows - 1, -1, -1, device=DEV, dtype=torch.int32)
    turned = [rows - o for o in offsets[::-1]]
    q = binding.moe_gemm_b128(p.a, p.sa, p.w.flip(0).contiguous(), p.sw.flip(0).contiguous(), offsets=ints(turned), a_rows=back, out_dtype=dtype)
    assert torch.equal(q.flip(0)[130:3977][~spoiled[130:3977]], clean[130:3977][~spoiled[130:3977]]) and torch.equal(q.flip(0)[130:3977].isnan(), spoiled[130:3977])


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_gemm_scales_far_apart(dtype):
    """Ten blocks of k with scales of their own, 2^72 apart: each block counts by its own scale and no neighbour's."""
    p = Product(4000, 3, 1640, 1168, seed=3, bytes_a=(87, 160), bytes_w=(87, 160))
    offsets = [0, 1500, 1501, 4000]
    p.check(in_tiles(dtype, lambda: p(offsets, out_dtype=dtype)), offsets, norm=False)
    # and one block alone: the others are zeros with the largest scales
    p.a.view(torch.uint8)[:, :768] = 0
    p.a.view(torch.uint8)[:, 896:] = 0
    p.check(in_tiles(dtype, lambda: p(offsets, out_dtype=dtype)), offsets, norm=False)


# ---- the feed-forward
class Experts:
    """Weights of E experts; what those with rows stand for, on the host."""

    def __init__(self, E, D, F, activation, dtype, T_max, seed=0):
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.halves = (2,) if activation == "silu" else ()
        self.w1, self.s1 = operand((E, *self.halves, F, D), (E, *self.halves, -(-F // 128)), 116, 119, g)
        self.w2, self.s2 = operand((E, D, F), (E, -(-D // 128)), 116, 119, g)
        self.E, self.D, self.F, self.activation, self.dtype, self.g = E, D, F, activation, dtype, g
        self.layer = binding.MoeLayer(T_max, D, F, E, 1, "bf16" if dtype == BF16 else "f32", alloc_workspace=False)

    def rows(self, T):
        x = torch.randn((T, self.D), device=DEV, generator=self.g)
        x[:, ::37] *= 8
        return (x * 2.0 ** -7 / math.sqrt(self.D)).to(self.dtype)

    def __call__(self, x, offsets, src, **kw):
        return self.layer.moe_expert_ffn_b128(x, ints(offsets), self.w1, self.w2, self.s1, self.s2, activation=self.activation, src_tok=ints(src), **kw)

    def some(self, offsets, most, seed=0):
        """(rows, at most `most` of them, the first and last of every expert among them; offsets of those; values of the weights of the experts that have some)"""
        rng, keep, counts, w1, w2 = np.random.default_rng(seed), [], [], [], []
        active = [e for e in range(self.E) if offsets[e] < offsets[e + 1]]
        for e in active:
            lo, hi = offsets[e], offsets[e + 1]
            r = np.unique(np.concatenate([[lo, hi - 1], rng.integers(lo, hi, max(0, most // len(active) - 2))]))
            keep.append(r)
            counts.append(len(r))
            w1.append(np.stack([host(value(m, s, 128)) for m, s in zip(self.w1[e].view(-1, self.F, self.D), self.s1[e].view(-1, *self.s1.shape[-2:]))]))
            w2.append(host(value(self.w2[e], self.s2[e], 128)))
        w1 = np.stack(w1)
        return np.concatenate(keep), ends(counts), (w1 if self.halves else w1[:, 0], np.stack(w2))


@pytest.mark.parametrize("T,rows,E,D,F", [(1500, 5000, 3, 1040, 1200), (3000, 4000, 70, 272, 528), (2000, 20000, 6, 272, 1328)])
@pytest.mark.parametrize("activation", ["relu", "silu"])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_ffn(T, rows, E, D, F, activation, dtype):
    """Both products in tiles: many blocks of k, more than 64 experts, more than 1024 tiles; a row with a NaN beside the others."""
    m = Experts(E, D, F, activation, dtype, rows, seed=D)
    x = m.rows(T)
    src, offsets = np.random.default_rng(E).integers(0, T, rows), ragged(rows, E, E, [2] if E < 10 else range(20, 66))
    names, y = kernels(lambda: m(x, offsets, src))
    first = "gemm_b128_tile_kernel<true, %d, %s>" % (2 if activation == "silu" else 1, "false" if dtype == BF16 else "true")
    assert any(first in n for n in names), names
    if E < 10:
        assert any("gemm_b128_tile_kernel<%s, 0, false>" % ("false" if dtype == BF16 else "true") in n for n in names), names
    keep, at, values = m.some(offsets, 200)
    check_ffn(y[torch.tensor(keep, device=DEV)], x, src[keep], values, at, activation, dtype, max(D, F))
    x[T // 2, D - 1] = math.nan
    spoiled = torch.tensor(src == T // 2, device=DEV)
    z = m(x, offsets, src)
    assert z[spoiled].isnan().all() and torch.equal(z[~spoiled], y[~spoiled])


def check_streamed(y, x, src, values, offsets, activation, dtype, K):
    want, moved = b128.ffn(b128.value(*b128.quantize(host(x))), values[0], values[1], offsets, activation, src, sum_error=K * 2.0 ** -24)
    got, half = host(y), 2.0 ** -8 if dtype == BF16 else 2.0 ** -24
    assert (np.abs(got - want) <= half * np.abs(want) + moved * (1 + half) + 2.0 ** -120).all()
    norm = np.sqrt(((got - want) ** 2).sum() / (want ** 2).sum())
    assert norm <= (2.0 ** -8 if dtype == BF16 else 0.0) + 2.0 ** -12, norm


@pytest.mark.parametrize("E,D,F,counts,ks", [
    (64, 2176, 1040, {3: 40, 7: 16, 8: 17, 63: 33, 20: 1}, {"silu": (1, 1), "relu": (2, 1)}),
    (40, 2064, 1040, {0: 50, 39: 30}, {"silu": (2, 2), "relu": (4, 2)}),
    (8, 4240, 2176, {2: 50, 5: 14}, {"silu": (4, 4), "relu": (8, 4)}),
    (2, 8208, 2192, {1: 16}, {"silu": (8, 8), "relu": (8, 8)}),
    (16, 4112, 4112, {4: 128}, {"silu": (1, 2), "relu": (2, 2)}),
])
@pytest.mark.parametrize("activation", ["relu", "silu"])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_ffn_streams_long_rows(E, D, F, counts, ks, activation, dtype):
    """Rows that LDS holds a piece of at a time, up to 8 of them an expert on average, and all of them one expert's; one, two, four and eight waves on the same weights."""
    per = [counts.get(e, 0) for e in range(E)]
    rows = sum(per)
    m = Experts(E, D, F, activation, dtype, max(rows, 8), seed=D)
    x = m.rows(rows // 2 + 1)
    src, offsets = np.random.default_rng(E).integers(0, len(x), rows), ends(per)
    names, y = kernels(lambda: m(x, offsets, src))
    for what in ("gemm_b128_stream_kernel<%d, %d, %d>" % (1 if dtype == BF16 else 2, 2 if activation == "silu" else 1, ks[activation][0]),
                 "gemm_b128_stream_kernel<2, 0, %d>" % ks[activation][1]):
        assert any(what in n for n in names), names
    keep, at, values = m.some(offsets, 10 ** 6)
    keep = torch.arange(rows) if len(keep) == rows else torch.tensor(keep)
    check_streamed(y[keep.to(DEV)], x, src[keep.numpy()], values, at, activation, dtype, max(D, F))
    assert torch.equal(m(x, offsets, src), y)


@pytest.mark.parametrize("activation", ["relu", "silu"])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_ffn_streams_what_tiles_cannot_address(activation, dtype):
    """A handle whose rows by index pass 32-bit offsets: any number of rows is streamed, with a workspace for that."""
    D, F, T = 16400, 144, 300
    m = Experts(2, D, F, activation, dtype, 2 ** 18, seed=1)
    assert 2 ** 18 * D > 0xfc000000
    x = m.rows(T)
    src, offsets = np.random.default_rng(0).integers(0, T, 700), [0, 213, 700]
    names, y = kernels(lambda: m(x, offsets, src))
    assert sum("gemm_b128_stream_kernel" in n for n in names) == 2 and not any("tile_kernel" in n for n in names), names
    keep, at, values = m.some(offsets, 120)
    check_streamed(y[torch.tensor(keep, device=DEV)], x, src[keep], values, at, activation, dtype, D)
    assert torch.equal(m(x, offsets, src), y)


@pytest.mark.parametrize("activation", ["relu", "silu"])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_layer_prefill(activation, dtype):
    """A whole batch: the selection of many tokens, more than 64 experts, tiles, the weighted sum; a token that is not finite spoils itself alone; captured, the same."""
    T, E, k, D, F = 7001, 96, 4, 272, 400
    m = Experts(E, D, F, activation, dtype, T, seed=5)
    layer = binding.MoeLayer(T, D, F, E, k, "bf16" if dtype == BF16 else "f32", alloc_workspace=False)
    x = m.rows(T)
    wg = (torch.randn((E, D), device=DEV, generator=m.g) * 40).to(dtype)
    bias = torch.randn(E, device=DEV, generator=m.g) * 0.1
    kw = dict(activation=activation, select_bias=bias, n_groups=8, groups_kept=3, scale=2.0)
    run = lambda x, **more: layer.moe_layer_forward_b128(x, wg, m.w1, m.w2, m.s1, m.s2, **kw, **more)  # noqa: E731
    r = layer.empty_routing(T)
    names, y = kernels(lambda: run(x, routing_out=r))
    assert any("select_many_kernel" in n for n in names) and any("gemm_b128_tile_kernel<true" in n for n in names), names
    idx, w = b128.select(host(r["logits"]), k, bias=host(bias), n_groups=8, groups_kept=3, scale=2.0)
    assert np.array_equal(r["topk_idx"].cpu().numpy(), idx)
    order = np.argsort(idx.ravel(), kind="stable")
    offsets = ends(np.bincount(idx.ravel(), minlength=E))
    assert np.array_equal(r["src_tok"].cpu().numpy(), order // k) and r["offsets"].cpu().tolist() == offsets
    yp = layer.moe_expert_ffn_b128(x, r["offsets"], m.w1, m.w2, m.s1, m.s2, activation=activation, src_tok=r["src_tok"])
    keep, at, values = m.some(offsets, 200)
    check_ffn(yp[torch.tensor(keep, device=DEV)], x, (order // k)[keep], values, at, activation, dtype, max(D, F))
    parts = host(yp)[r["dst_row"].cpu().numpy()].reshape(T, k, D)
    total, size = (parts * w[:, :, None]).sum(1), np.abs(parts * w[:, :, None]).sum(1)
    half = 2.0 ** -8 if dtype == BF16 else 2.0 ** -24
    assert (np.abs(host(y) - total) <= half * np.abs(total) + 2 * k * 2.0 ** -24 * size + 2.0 ** -120).all()
    out, x2 = torch.empty_like(y), x.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(x2, y=out)
    x2[77, 5], x2[T - 1, 0] = math.nan, math.inf
    others = torch.ones(T, dtype=torch.bool, device=DEV)
    others[[77, T - 1]] = False
    for spoiled in (True, False, True):
        if not spoiled:
            x2.copy_(x)
        else:
            x2[77, 5], x2[T - 1, 0] = math.nan, math.inf
        graph.replay()
        assert torch.equal(out[others], y[others])
        assert out[~others].isnan().any(1).all() if spoiled else torch.equal(out, y)
