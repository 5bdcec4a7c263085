"""moe_sample against the 64-bit oracle: tokens are equal; the log-probability is rounded once to fp32 (2^-24 of it), the weights' sum
holds whole numbers of 2^-43 or less (1e-7 of the sum at the largest vocabulary)."""
import math

import numpy as np
import pytest
import torch

from oracle import decoder_step as od
from paper_2303_06182_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def f32(v):
    return None if v is None else torch.tensor(np.asarray(v, dtype=np.float32), device=DEV)


def check(logits, u, temperature=None, top_k=None, top_p=None, min_p=None):
    """logits [B, V] on the device (maybe strided)."""
    B = logits.shape[0]
    token, logprob = binding.moe_sample(logits, f32(u), f32(temperature), None if top_k is None else torch.tensor(top_k, dtype=torch.int32, device=DEV),
                                        f32(top_p), f32(min_p))
    token, logprob, rows = token.cpu().tolist(), logprob.double().cpu().tolist(), logits.double().cpu().numpy()
    at = lambda v, b, other: other if v is None else float(np.float32(v[b]))  # noqa: E731
    for b in range(B):
        want, lp = od.sample(rows[b], at(u, b, 0), at(temperature, b, 1.0), 0 if top_k is None else top_k[b], at(top_p, b, 1.0), at(min_p, b, 0.0))
        assert token[b] == want, (b, token[b], want)
        assert logprob[b] == lp or abs(logprob[b] - lp) <= 2.0 ** -24 * abs(lp) + 1e-7, (b, logprob[b], lp)


def logits_of(B, V, dtype, seed, sharp=1.0):
    rng = np.random.default_rng(seed)
    x = -sharp * np.log(np.argsort(rng.random((B, V)), 1) + 1.0) + rng.standard_normal((B, V)) * 0.7
    return torch.from_numpy(x).to(dtype).to(DEV), rng


@pytest.mark.parametrize("V", [1, 2, 63, 64, 1000, 4097, 20011])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_filters(V, dtype):
    """Every filter alone and all together; bf16 logits have many ties, at the borders too."""
    B = 24
    x, rng = logits_of(B, V, dtype, V)
    u = rng.random(B).astype(np.float32)
    check(x, u)                                     # rows at any element
    check(x[1:], u[1:])
    for kw in (dict(top_p=rng.choice([0.5, 0.9, 0.95], B)), dict(top_k=[int(k) for k in rng.choice([1, 2, 5, 50, 1000, V, V + 1], B)]),
               dict(min_p=rng.choice([0.01, 0.1, 1.0, 2.0], B)), dict(temperature=rng.choice([0.0, 0.3, 1.0, 1.7], B)),
               dict(top_p=rng.choice([0.5, 0.9, 1.0], B), top_k=[int(k) for k in rng.choice([0, 3, 50, 700], B)], min_p=rng.choice([0.0, 0.05], B),
                    temperature=rng.choice([0.0, 0.7, 1.3], B))):
        check(pad(x), u, **kw)


def pad(x):
    """The same rows at a stride of a multiple of 16 bytes."""
    B, V = x.shape
    wide = torch.full((B, (V + 15) // 8 * 8), 99.0, dtype=x.dtype, device=DEV)
    wide[:, :V] = x
    return wide[:, :V]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_ties_and_flat_rows(dtype):
    """Rows of one value, of two, and of a ramp: every border lies among ties."""
    V, B = 3000, 12
    x = torch.zeros((B, V), dtype=dtype, device=DEV)
    x[1::3] = (torch.arange(V, device=DEV) % 2).to(dtype)
    x[2::3] = (torch.arange(V, device=DEV) // 100 * 0.25).to(dtype)
    u = np.linspace(0.0, 0.9999, B)
    check(x, u)
    check(x, u, top_k=[7] * B)
    check(x, u, top_p=[0.37] * B)
    check(x, u, top_p=[0.37] * B, top_k=[2100] * B)
    check(x, u, top_p=[1e-6] * B)
    check(x, u, min_p=[0.4] * B)


def test_infinities_and_nan():
    V, inf = 500, math.inf
    x = torch.full((9, V), -inf, device=DEV)
    x[1, 17] = -3.0
    x[2] = math.nan
    x[3, ::2], x[3, 1::2] = math.nan, 0.5
    x[4, 100:200] = inf
    x[5] = torch.finfo(torch.float32).min
    x[6], x[6, 3] = torch.finfo(torch.float32).min, 0.0
    x[7, :4] = torch.tensor([-0.0, 0.0, -0.0, 0.0], device=DEV)
    x[8, 5], x[8, 6] = inf, 1.0
    u = np.full(9, 0.6)
    for kw in ({}, dict(top_p=[0.5] * 9), dict(top_k=[3] * 9), dict(min_p=[0.2] * 9), dict(temperature=[0.0] * 9), dict(temperature=[1e-3] * 9),
               dict(temperature=[1e3] * 9), dict(top_k=[2] * 9, top_p=[0.9] * 9, min_p=[0.1] * 9)):
        check(x, u, **kw)


@pytest.mark.parametrize("B,V", [(1, 128000), (3, 1 << 19), (130, 9001), (5, 50001), (40, 33000)])
def test_sizes(B, V):
    x, rng = logits_of(B, V, torch.float32, B)
    u = rng.random(B).astype(np.float32)
    check(pad(x), u, top_p=[0.9] * B)
    check(pad(x), u)
    check(pad(x), u, top_k=[20000] * B, temperature=[2.0] * B)


def test_spread_and_crowded_values():
    """Logits hundreds apart, and a vocabulary inside one small step of the selection."""
    rng = np.random.default_rng(5)
    B, V = 6, 9000
    x = rng.standard_normal((B, V)) * 300
    x[3:] = 20 + rng.random((3, V)) * 1e-3
    x = torch.from_numpy(x).float().to(DEV)
    u = rng.random(B).astype(np.float32)
    for kw in ({}, dict(top_k=[4000] * B), dict(top_p=[0.6] * B), dict(top_p=[0.999] * B, top_k=[8000] * B), dict(temperature=[50.0] * B, top_p=[0.8] * B)):
        check(x, u, **kw)


def test_draws_follow_the_probabilities():
    """4096 rows alike, u spread evenly: counts are the probabilities, up to the one token that a border can move."""
    p = np.array([0.05, 0.0, 0.4, 0.25, 0.3])
    B = 4096
    with np.errstate(divide="ignore"):
        x = torch.from_numpy(np.tile(np.log(p), (B, 1))).float().to(DEV)
    u = (np.arange(B) + 0.5) / B
    token, _ = binding.moe_sample(pad(x), f32(u))
    assert (np.abs(np.bincount(token.cpu().numpy(), minlength=5) - p * B) <= 1).all()


def test_same_result_every_time_and_in_a_graph():
    x, rng = logits_of(16, 30000, torch.bfloat16, 1)
    u = f32(rng.random(16))
    top_p, workspace = f32([0.95] * 16), torch.empty(binding.moe_sample_workspace_bytes(16, 30000), dtype=torch.uint8, device=DEV)
    token, logprob = binding.moe_sample(x, u, top_p=top_p, workspace=workspace)
    t2, l2 = token.clone(), logprob.clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.moe_sample(x, u, top_p=top_p, token=t2, logprob=l2, workspace=workspace)
    for i in range(3):
        if i:
            u.copy_(f32(rng.random(16)))
        workspace.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        got = t2.clone(), l2.clone()
        token, logprob = binding.moe_sample(x, u, top_p=top_p, workspace=workspace)
        torch.cuda.synchronize()
        assert torch.equal(got[0], token) and torch.equal(got[1], logprob)


@pytest.mark.parametrize("V", [300, 30000])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_min_p_that_is_no_number_leaves_the_first(V, dtype):
    """No weight is at least NaN, and the first of the order always stays; alone, with the other filters, and on a row whose last tokens are masked."""
    B = 4
    x, rng = logits_of(B, V, dtype, 3)
    x[:, V // 2:] = -math.inf
    u = rng.random(B).astype(np.float32)
    for kw in ({}, dict(top_k=[5] * B), dict(top_p=[0.9] * B), dict(temperature=[0.7] * B)):
        check(x, u, min_p=[math.nan] * B, **kw)


@pytest.mark.parametrize("V", [300, 30000])
def test_infinite_logits_and_infinite_temperature(V):
    """Where the largest logit is +infinity its tokens have w = 1 and the others none, at every temperature; with finite ones an infinite temperature
    makes all of them equal."""
    x = torch.full((4, V), -1.0, device=DEV)
    x[0, 7], x[1, 40:60], x[2, ::2], x[3, 5] = math.inf, math.inf, -math.inf, 3.0
    u = np.array([0.9, 0.3, 0.77, 0.5])
    for t in (math.inf, 3e38, 1e30):
        for kw in ({}, dict(min_p=[0.5] * 4), dict(top_k=[30] * 4), dict(top_p=[0.6] * 4)):
            check(x, u, temperature=[t] * 4, **kw)


@pytest.mark.parametrize("V", [20000, 40000])
@pytest.mark.parametrize("top_p", [0.3, 0.99])
def test_borders_around_what_is_sorted(V, top_p):
    """Rows shared by several blocks, about as many likely tokens as are still sorted together (512), and as by count (3891): the blocks that gather
    and the one that goes on agree about them."""
    B = 24
    rng = np.random.default_rng(V)
    for least, step, kw in ((500, 1, dict(top_p=[top_p] * B)), (3860, 3, dict(top_k=[3700] * B, top_p=[top_p] * B))):
        x = rng.random((B, V)) * 4 - 30
        for b in range(B):
            x[b, rng.choice(V, least + step * b, replace=False)] = 2.0 + rng.random(least + step * b) * 0.01
        check(torch.from_numpy(x).float().to(DEV), rng.random(B).astype(np.float32), **kw)


@pytest.mark.parametrize("V", [20000, 40001])
def test_infinities_and_nan_of_rows_shared_by_blocks(V):
    """As above, in vocabularies that several blocks share."""
    inf = math.inf
    x = torch.full((9, V), -inf, device=DEV)
    x[1, V - 3] = -3.0
    x[2] = math.nan
    x[3, ::2], x[3, 1::2] = math.nan, 0.5
    x[4, 8100:8300] = inf
    x[5] = torch.finfo(torch.float32).min
    x[6], x[6, V // 2] = torch.finfo(torch.float32).min, 0.0
    x[7, 9000:9004] = torch.tensor([-0.0, 0.0, -0.0, 0.0], device=DEV)
    x[8, 17000], x[8, 6] = inf, 1.0
    u = np.full(9, 0.6)
    for kw in ({}, dict(top_p=[0.5] * 9), dict(top_k=[3] * 9), dict(min_p=[0.2] * 9), dict(temperature=[0.0] * 9), dict(temperature=[1e-3] * 9),
               dict(temperature=[1e3] * 9), dict(top_k=[2] * 9, top_p=[0.9] * 9, min_p=[0.1] * 9)):
        check(x, u, **kw)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_ties_and_flat_rows_shared_by_blocks(dtype):
    """Borders among ties, in steps of more tokens than are sorted: by weight first, by count first, both."""
    V, B = 20000, 6
    x = torch.zeros((B, V), dtype=dtype, device=DEV)
    x[1::3] = (torch.arange(V, device=DEV) % 2).to(dtype)
    x[2::3] = (torch.arange(V, device=DEV) // 700 * 0.25).to(dtype)
    u = np.linspace(0.0, 0.9999, B)
    for kw in ({}, dict(top_k=[7] * B), dict(top_k=[6000] * B), dict(top_p=[0.37] * B), dict(top_p=[0.37] * B, top_k=[9100] * B), dict(top_p=[1e-6] * B),
               dict(min_p=[0.4] * B)):
        check(x, u, **kw)


def test_spread_and_crowded_values_of_rows_shared_by_blocks():
    rng = np.random.default_rng(6)
    B, V = 4, 20000
    x = rng.standard_normal((B, V)) * 300
    x[2:] = 20 + rng.random((2, V)) * 1e-3
    x = torch.from_numpy(x).float().to(DEV)
    u = rng.random(B).astype(np.float32)
    for kw in ({}, dict(top_k=[9000] * B), dict(top_p=[0.6] * B), dict(top_p=[0.999] * B, top_k=[18000] * B), dict(temperature=[50.0] * B, top_p=[0.8] * B)):
        check(x, u, **kw)


@pytest.mark.parametrize("V", [6500, 20000])
def test_more_tokens_in_a_step_than_their_weight_says(V):
    """A temperature below the normal range: 6000 tokens lie in the step of the largest logit and weigh nothing beside it, so the guess of how many there
    are, which goes by weight, is far off."""
    x = torch.full((3, V), -5.0, device=DEV)
    x[:, :6000] = torch.arange(6000, device=DEV, dtype=torch.float64).mul(-1e-43).float().roll(11)
    check(x, np.array([0.0, 0.5, 0.99]), temperature=[1e-45] * 3, top_p=[0.9] * 3)


def test_outputs_and_settings_that_do_not_fit_are_refused():
    x, rng = logits_of(3, 40, torch.float32, 0)
    u = f32(rng.random(3))
    for kw in (dict(token=torch.empty(3, dtype=torch.int64, device=DEV)), dict(token=torch.empty(2, dtype=torch.int32, device=DEV)),
               dict(token=torch.empty(3, dtype=torch.int32)), dict(logprob=torch.empty(4, device=DEV)), dict(logprob=torch.empty(3, dtype=torch.float64, device=DEV)),
               dict(workspace=torch.empty(4096, dtype=torch.uint8)), dict(workspace=torch.empty(4096, device=DEV)), dict(top_p=torch.ones(3))):
        with pytest.raises(ValueError):
            binding.moe_sample(x, u, **kw)
    with pytest.raises(ValueError):
        binding.moe_sample(x, u.cpu())
    with pytest.raises(ValueError):
        binding.moe_sample(x.cpu(), u.cpu())
    check(x, u.cpu().numpy())


def test_more_rows_than_2_32_threads():
    """4.2 million rows of three tokens: a block each."""
    B = (1 << 22) + 1000
    gen = torch.Generator(device=DEV).manual_seed(4)
    x = torch.empty((B, 3), device=DEV).normal_(0, 1, generator=gen)
    u = torch.rand(B, device=DEV, generator=gen)
    token, logprob = binding.moe_sample(x, u, token=torch.full((B,), -7, dtype=torch.int32, device=DEV))
    p = torch.softmax(x.double(), 1)
    c = p.cumsum(1)
    want = (u.double()[:, None] >= c[:, :2]).sum(1)
    near = ((u.double()[:, None] - c[:, :2]).abs() < 1e-9).any(1)            # sums of another order
    assert ((token.long() == want) | near).all()
    # log(p) is rounded once to fp32, 2^-24 of it; both sides' 64-bit weights 1e-12
    lp = torch.log(torch.gather(p, 1, token.long()[:, None]))[:, 0]
    assert ((logprob.double() - lp).abs() <= 2.0 ** -24 * lp.abs() + 1e-11).all()
