"""The MoE layer with its experts' products in 8 bits, over the range a user of this library meets.

Four operators: ``moe_select_experts`` (sigmoid or softmax scores, a bias for balance, groups of experts, top-k),
``moe_quantize_b128`` (e4m3 bytes with a power of two as scale for each block of 128, of a row or of 128 rows), ``moe_gemm_b128``
(product of such operands, grouped by expert or plain) and ``moe_expert_ffn_b128`` (the experts' feed-forward on them: rows quantised,
first product, gated SiLU or ReLU, quantised again, second product).  Sizes are the layers' of this repository (1024 -> 4096,
2048 -> 8192, 16 to 512 experts) and generic ones.

A case is one call:

    op                      "select", "quantize", "gemm" or "ffn"
    select                  T tokens, E experts, k of them, G groups of which `kept` stay by the sum of their `top` best, score
                            "sigmoid" or "softmax", bias, renorm, dtype "f32" or "bf16" of the logits
    quantize                matrices of rows x cols, `matrices` of them (block_rows 128: weights) or one (block_rows 1: rows), dtype
    gemm                    rows over E experts (1: a plain product), N columns, a contraction of K, `skew` of the experts' popularity,
                            gather (rows by index, of half as many), dtype of the result
    ffn                     T tokens of which each has k experts of E, D -> F -> D, `act` "silu" (gated) or "relu", skew, dtype of x and y
"""
from __future__ import annotations

import math
import random
import zlib

import numpy as np
import torch

own = False


def _select(name, T, E, k, G, kept, top, score, bias, renorm, dtype):
    return dict(name=name, op="select", T=T, E=E, k=k, G=G, kept=kept, top=top, score=score, bias=bias, renorm=renorm, dtype=dtype)


def _quantize(name, matrices, rows, cols, block_rows, dtype):
    return dict(name=name, op="quantize", matrices=matrices, rows=rows, cols=cols, block_rows=block_rows, dtype=dtype)


def _gemm(name, rows, E, N, K, skew, gather, dtype):
    return dict(name=name, op="gemm", rows=rows, E=E, N=N, K=K, skew=skew, gather=gather, dtype=dtype)


def _ffn(name, T, k, E, D, F, act, skew, dtype):
    return dict(name=name, op="ffn", T=T, k=k, E=E, D=D, F=F, act=act, skew=skew, dtype=dtype)


def listed():
    return [
        # one token being decoded: latency alone
        _select("select_1", 1, 128, 8, 8, 4, 2, "sigmoid", True, True, "f32"),
        # a decoder step over many experts, softmax scores, no groups
        _select("select_64", 64, 512, 2, 1, 1, 1, "softmax", False, False, "bf16"),
        # a whole prefill batch: bound by the logits and the selection's arithmetic
        _select("select_64k", 65536, 128, 6, 8, 3, 2, "sigmoid", True, True, "f32"),
        # a decoder step's rows
        _quantize("quantize_64", 1, 64, 2048, 1, "bf16"),
        # a prefill batch's rows, of a length that ends inside a block
        _quantize("quantize_64k", 1, 65536, 2000, 1, "bf16"),
        # a layer's weights, laid out once
        _quantize("quantize_weights", 16, 8192, 2048, 128, "bf16"),
        # few rows of a plain product: bound by reading the weights
        _gemm("gemm_17", 17, 1, 8192, 2048, 0.0, False, "f32"),
        # ragged experts, odd sizes, rows gathered by index
        _gemm("gemm_ragged", 5003, 24, 1640, 1200, 1.0, True, "bf16"),
        # a large plain product: bound by the matrix cores
        _gemm("gemm_8k", 8192, 1, 8192, 8192, 0.0, False, "bf16"),
        # one token's eight experts
        _ffn("ffn_1", 1, 8, 64, 2048, 1024, "silu", 0.0, "bf16"),
        # a decoder step of 64 tokens: most experts are active with a few rows each
        _ffn("ffn_64", 64, 8, 128, 2048, 1024, "silu", 0.5, "bf16"),
        # an encoder's batch over 16 experts, the repository's own layer
        _ffn("ffn_16k", 16384, 2, 16, 2048, 8192, "relu", 0.5, "bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _log_multiple(rng, of, lo, hi):
    """A multiple of `of`; now and then a rounder one."""
    step = of * rng.choice([1, 1, 8])
    return max(of, _log_int(rng, lo, hi) // step * step)


def draw(rng: random.Random):
    """One more case (without a name)."""
    op = rng.choice(["select", "select", "quantize", "gemm", "gemm", "gemm", "ffn", "ffn", "ffn"])
    if op == "select":
        G = rng.choice([1, 1, 2, 4, 8, 16])
        size = max(2, _log_int(rng, max(8, 2 * G), 512) // G)
        kept = rng.randint(1, G)
        c = _select("", _log_int(rng, 1, 65536), G * size, rng.randint(1, min(8, kept * size)), G, kept, rng.choice([1, 2]),
                    rng.choice(["sigmoid", "softmax"]), rng.random() < 0.6, rng.random() < 0.7, rng.choice(["f32", "bf16"]))
        c["T"] = min(c["T"], 65536 * 128 // c["E"])
    elif op == "quantize":
        dtype = rng.choice(["bf16", "bf16", "f32"])
        if rng.random() < 0.6:
            cols = _log_multiple(rng, 16, 64, 16384)
            c = _quantize("", 1, min(_log_int(rng, 1, 65536), (1 << 27) // cols), cols, 1, dtype)
        else:
            rows, cols = _log_multiple(rng, 8, 64, 8192), _log_multiple(rng, 16, 64, 8192)
            c = _quantize("", min(_log_int(rng, 1, 64), max(1, (1 << 27) // rows // cols)), rows, cols, 128, dtype)
    elif op == "gemm":
        E = rng.choice([1, 1, _log_int(rng, 2, 128)])
        N, K = _log_multiple(rng, 8, 64, 8192), _log_multiple(rng, 16, 64, 8192)
        E = max(1, min(E, (1 << 29) // (N * K)))
        rows = min(_log_int(rng, 1, 16384), int(5e11 / N / K))
        c = _gemm("", rows, E, N, K, rng.choice([0.0, 0.5, 1.0]), rng.random() < 0.4, rng.choice(["bf16", "bf16", "f32"]))
    else:
        D, F = _log_multiple(rng, 16, 256, 4096), _log_multiple(rng, 16, 256, 8192)
        act = rng.choice(["silu", "silu", "relu"])
        E = max(2, min(_log_int(rng, 4, 256), 800000000 // (D * F * (3 if act == "silu" else 2))))
        k = rng.randint(1, min(8, E))
        T = max(1, min(_log_int(rng, 1, 16384), int(2.5e11 / D / F / k)))
        c = _ffn("", T, k, E, D, F, act, rng.choice([0.0, 0.5, 1.0]), rng.choice(["bf16", "bf16", "bf16", "f32"]))
    del c["name"]
    return c


def _counts(case):
    """Rows of every expert, from the case alone (work() needs them too): popularity falls with a power of the rank."""
    E, skew = case["E"], case["skew"]
    most, rows = (case["T"], case["T"] * case["k"]) if case["op"] == "ffn" else (case["rows"], case["rows"])
    r = np.random.default_rng(zlib.crc32(repr(sorted((k, v) for k, v in case.items() if k != "name")).encode()))
    weight = (1.0 + r.permutation(E)) ** -skew
    counts = np.zeros(E, dtype=np.int64)
    while counts.sum() < rows:  # an expert has a token once at most
        free = counts < most
        counts = np.minimum(most, counts + r.multinomial(rows - counts.sum(), weight * free / (weight * free).sum()))
    return counts.tolist()


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _normal(shape, std, dtype, gen):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=gen)


def _blocks(n):
    return -(-n // 128)


def _scale_columns(cols):
    """Scale bytes of a row: one for each block of 128, in groups of four."""
    return -(-cols // 512) * 4


def _operand(shape, scale_rows, low, gen):
    """e4m3 values and scale bytes (low, low + 1 or low + 2), as a quantisation leaves them."""
    q = _normal(shape, 100.0, torch.bfloat16, gen).clamp_(-448, 448).to(torch.float8_e4m3fn)
    scale = torch.randint(low, low + 3, scale_rows + (_scale_columns(shape[-1]),), device="cuda", generator=gen, dtype=torch.uint8)
    scale[..., _blocks(shape[-1]):] = 127
    return q, scale


def _rows_of_tokens(counts, tokens, gen):
    """For every expert's rows the tokens they come from: ascending, each once."""
    return torch.cat([torch.randperm(tokens, generator=gen, device="cuda")[:n].sort()[0] for n in counts if n]).int()


def prepare(case, seed):
    """Logits and bias; or values to be quantised; or quantised operands, the experts' offsets and the rows' tokens."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    op, s = case["op"], dict(case=case)
    if op == "select":
        s["logits"] = _normal((case["T"], case["E"]), 1.5, _dtype(case), gen)
        # what balancing has added up for every expert
        s["bias"] = _normal((case["E"],), 0.1, torch.float32, gen) if case["bias"] else None
        return s
    if op == "quantize":
        shape = (case["rows"], case["cols"]) if case["block_rows"] == 1 else (case["matrices"], case["rows"], case["cols"])
        s["x"] = _normal(shape, 1.0 if case["block_rows"] == 1 else 0.02, _dtype(case), gen)
        # a few columns that are much larger, as activations have them
        s["x"][..., ::97] *= 16.0
        return s
    s["counts"] = _counts(case)
    ends = np.cumsum([0] + s["counts"]).tolist()
    s["offsets"] = torch.tensor(ends, dtype=torch.int32, device="cuda")
    if op == "gemm":
        E, N, K, rows = case["E"], case["N"], case["K"], case["rows"]
        held = max(1, rows // 2) if case["gather"] else rows
        s["a"], s["a_scale"] = _operand((held, K), (held,), 119, gen)
        s["w"], s["w_scale"] = _operand((E, N, K), (E, _blocks(N)), 114, gen)
        s["a_rows"] = torch.randint(0, held, (rows,), device="cuda", generator=gen, dtype=torch.int32) if case["gather"] else None
        return s
    E, D, F = case["E"], case["D"], case["F"]
    s["x"] = _normal((case["T"], D), 1.0, _dtype(case), gen)
    s["x"][..., ::97] *= 16.0
    s["src_tok"] = _rows_of_tokens(s["counts"], case["T"], gen)
    gated = case["act"] == "silu"
    s["w1"], s["w1_scale"] = _operand((E, 2, F, D) if gated else (E, F, D), (E, 2, _blocks(F)) if gated else (E, _blocks(F)), 114, gen)
    s["w2"], s["w2_scale"] = _operand((E, D, F), (E, _blocks(D)), 114, gen)
    if own:  # the handle that a program keeps for its layers
        from paper_2303_06182_amd import binding
        s["layer"] = binding.MoeLayer(case["T"], D, F, E, case["k"], case["dtype"], alloc_workspace=False)
    return s


def _power_of_two(byte):
    """2^(byte - 127) in 32 bits, 1 <= byte <= 254."""
    return (byte.int() << 23).view(torch.float32)


def _select_plain(s):
    c = s["case"]
    T, E, G, k = c["T"], c["E"], c["G"], c["k"]
    logits = s["logits"].double()
    score = 1 / (1 + torch.exp(-logits))
    if c["score"] == "softmax":
        e = torch.exp(logits - logits.amax(1, keepdim=True))
        score = e / e.sum(1, keepdim=True)
    key = score + s["bias"].double() if c["bias"] else score
    if c["kept"] < G:
        best = torch.sort(key.view(T, G, E // G), dim=2, descending=True)[0][..., :c["top"]].sum(2)
        order = torch.sort(best, dim=1, descending=True, stable=True)[1]
        out = torch.ones((T, G), dtype=torch.bool, device="cuda").scatter_(1, order[:, :c["kept"]], False)
        key = key.masked_fill(out.repeat_interleave(E // G, 1), -math.inf)
    idx = torch.sort(key, dim=1, descending=True, stable=True)[1][:, :k]
    w = torch.gather(score, 1, idx)
    if c["renorm"]:
        w = w / w.sum(1, keepdim=True)
    return {"idx": idx.int(), "w": (w * 2.5).float()}


def _quantized(x, block_rows):
    """x [M, R, C] in 32 bits -> e4m3 [M, R, C] and scale bytes [M, R or blocks of rows, columns in groups of four]."""
    M, R, C = x.shape
    rb, cb = -(-R // block_rows), _blocks(C)
    whole = torch.nn.functional.pad(x, (0, cb * 128 - C, 0, rb * block_rows - R)).view(M, rb, block_rows, cb, 128)
    largest = whole.abs().amax((2, 4))
    mantissa, exponent = torch.frexp(largest)
    byte = torch.where(largest > 0, torch.where(mantissa <= 0.875, exponent - 9, exponent - 8).clamp(min=-126) + 127, 127)
    q = (whole / _power_of_two(byte)[:, :, None, :, None]).view(M, rb * block_rows, cb * 128)[:, :R, :C].to(torch.float8_e4m3fn)
    return q, torch.nn.functional.pad(byte, (0, _scale_columns(C) - cb), value=127).to(torch.uint8)


def _value(q, scale, block_rows):
    """e4m3 [R, C] times its scales, in 32 bits."""
    R, C = q.shape
    s = _power_of_two(scale).repeat_interleave(block_rows, 0)[:R].repeat_interleave(128, 1)[:, :C]
    return q.float() * s


def _products(a, counts, w, w_scale):
    """Rows of every expert, in 32 bits, times that expert's weights."""
    out, at = [], 0
    for e, n in enumerate(counts):
        if n:
            out.append(a[at:at + n] @ _value(w[e], w_scale[e], 128).T)
        at += n
    return torch.cat(out)


def _gemm_plain(s):
    a = _value(s["a"], s["a_scale"], 1)
    if s["a_rows"] is not None:
        a = a[s["a_rows"].long()]
    return _products(a, s["counts"], s["w"], s["w_scale"]).to(_dtype(s["case"]))


def _ffn_plain(s):
    c = s["case"]
    q, scale = _quantized(s["x"].float()[None], 1)
    a = _value(q[0], scale[0], 1)[s["src_tok"].long()]
    if c["act"] == "silu":
        g, u = (_products(a, s["counts"], s["w1"][:, i], s["w1_scale"][:, i]) for i in (0, 1))
        h = g / (1 + torch.exp(-g)) * u
    else:
        h = _products(a, s["counts"], s["w1"], s["w1_scale"]).clamp(min=0)
    q, scale = _quantized(h[None], 1)
    return _products(_value(q[0], scale[0], 1), s["counts"], s["w2"], s["w2_scale"]).to(_dtype(c))


def _quantize_plain(s):
    x = s["x"].float()
    q, scale = _quantized(x if x.dim() == 3 else x[None], s["case"]["block_rows"])
    return {"q": q.view(x.shape), "scale": scale if x.dim() == 3 else scale[0]}


def run(s):
    """One pass through an operator."""
    c = s["case"]
    op = c["op"]
    if not own:
        return {"select": _select_plain, "quantize": _quantize_plain, "gemm": _gemm_plain, "ffn": _ffn_plain}[op](s)
    from paper_2303_06182_amd import binding
    if op == "select":
        idx, w = binding.moe_select_experts(s["logits"], c["k"], bias=s["bias"], score=c["score"], n_groups=c["G"], groups_kept=c["kept"],
                                            group_top=c["top"], renormalize=c["renorm"], scale=2.5)
        return {"idx": idx, "w": w}
    if op == "quantize":
        q, scale = binding.moe_quantize_b128(s["x"], block_rows=c["block_rows"])
        return {"q": q, "scale": scale}
    if op == "gemm":
        return binding.moe_gemm_b128(s["a"], s["a_scale"], s["w"], s["w_scale"], offsets=s["offsets"] if c["E"] > 1 else None, a_rows=s["a_rows"],
                                     out_dtype=_dtype(c))
    return s["layer"].moe_expert_ffn_b128(s["x"], s["offsets"], s["w1"], s["w2"], s["w1_scale"], s["w2_scale"], activation=c["act"],
                                          src_tok=s["src_tok"])


def work(case):
    """Selecting: logits in, indices and weights out, about ten operations a logit.  Quantising: values in, bytes and scales out.
    Products: the rows that are read, the active experts' weights, each with its scales, and the result; two operations a product."""
    op, es = case["op"], 2 if case["dtype"] == "bf16" else 4
    if op == "select":
        return {"bytes": float(case["T"] * (case["E"] * es + 8 * case["k"])), "flops": 10.0 * case["T"] * case["E"]}
    if op == "quantize":
        n = case["matrices"] * case["rows"] * case["cols"]
        return {"bytes": n * (es + 1.0) + n / (128.0 * case["block_rows"]), "flops": 3.0 * n}
    counts = _counts(case)
    active, rows = sum(1 for n in counts if n), sum(counts)
    if op == "gemm":
        N, K = case["N"], case["K"]
        held = max(1, rows // 2) if case["gather"] else rows
        return {"bytes": float(held * K * 129 / 128 + active * N * K + rows * N * es), "flops": 2.0 * rows * N * K}
    D, F, T = case["D"], case["F"], case["T"]
    matrices = 3 if case["act"] == "silu" else 2
    return {"bytes": float(min(T, rows) * D * es + active * matrices * D * F + rows * D * es), "flops": 2.0 * rows * D * F * matrices}


def _two_to(n):
    """2^n in 64 bits, exactly."""
    return ((n.long() + 1023) << 52).view(torch.float64)


def _e4m3(x):
    """x in 64 bits, |x| <= 448: the nearest e4m3 value, ties to even."""
    step = _two_to(torch.frexp(x)[1].clamp(min=-5) - 4)
    return torch.round(x / step) * step


def _exact_select(s):
    c = s["case"]
    E, G, k, size = c["E"], c["G"], c["k"], c["E"] // c["G"]
    logits = s["logits"].double().cpu().numpy()
    bias = s["bias"].double().cpu().numpy() if c["bias"] else np.zeros(E)
    if c["score"] == "sigmoid":
        score = 1.0 / (1.0 + np.exp(-logits))
    else:
        score = np.exp(logits - logits.max(1, keepdims=True))
        score /= score.sum(1, keepdims=True)
    key = score + bias
    idx, w = np.empty((c["T"], k), dtype=np.int32), np.empty((c["T"], k))
    for t in range(c["T"]):
        groups = key[t].reshape(G, size)
        best = np.partition(groups, size - min(c["top"], size), 1)[:, size - min(c["top"], size):].sum(1)
        allowed = np.sort(np.argsort(-best, kind="stable")[:c["kept"]])
        experts = (allowed[:, None] * size + np.arange(size)).ravel()
        idx[t] = experts[np.argsort(-key[t, experts], kind="stable")[:k]]
        w[t] = score[t, idx[t]]
    if c["renorm"]:
        w /= w.sum(1, keepdims=True)
    return {"idx": torch.from_numpy(idx), "w": torch.from_numpy(2.5 * w)}


def _exact_rows(x):
    """x [R, C] in 64 bits -> the values that its quantised rows stand for, the e4m3 numbers and the scales' exponents."""
    value, number, exponents = torch.empty_like(x), torch.empty_like(x), []
    for at in range(0, x.shape[1], 128):
        b = x[:, at:at + 128]
        n = _exponent(b.abs().amax(1))
        number[:, at:at + 128] = _e4m3(b / _two_to(n)[:, None])
        value[:, at:at + 128] = number[:, at:at + 128] * _two_to(n)[:, None]
        exponents.append(n)
    return value, number, torch.stack(exponents, 1)


def _exponent(largest):
    """The smallest n >= -126 with largest <= 448 * 2^n; 0 where largest is 0."""
    n = torch.floor(torch.log2((largest / 448).clamp(min=2.0 ** -126))) - 1
    for _ in range(3):
        n = n + (largest > 448 * _two_to(n))
    return torch.where(largest > 0, n.clamp(min=-126), torch.zeros_like(n)).long()


def _exact_quantize(s):
    c = s["case"]
    x = s["x"].double()
    x = x if x.dim() == 3 else x[None]
    number = torch.empty_like(x)
    scale = torch.full((x.shape[0], -(-c["rows"] // c["block_rows"]), _scale_columns(c["cols"])), 127, dtype=torch.uint8, device="cuda")
    for m in range(x.shape[0]):
        if c["block_rows"] == 1:
            _, number[m], n = _exact_rows(x[m])
            scale[m, :, :n.shape[1]] = n + 127
            continue
        for r in range(0, c["rows"], 128):
            tile = x[m, r:r + 128]
            n = torch.stack([_exponent(b.abs().amax()) for b in tile.split(128, 1)])
            scale[m, r // 128, :n.numel()] = n + 127
            number[m, r:r + 128] = _e4m3(tile / _two_to(n).repeat_interleave(128)[:c["cols"]])
    shape = s["x"].shape
    return {"q": number.view(shape), "scale": scale if len(shape) == 3 else scale[0]}


def _exact_weights(q, scale):
    """[N, K] in 64 bits."""
    w = q.double()
    factor = _two_to(scale.long() - 127)
    for n in range(0, w.shape[0], 128):
        w[n:n + 128] *= factor[n // 128].repeat_interleave(128)[:w.shape[1]]
    return w


def _exact_gemm(s):
    c = s["case"]
    a = s["a"].double() * _two_to(s["a_scale"].long() - 127).repeat_interleave(128, 1)[:, :c["K"]]
    ends, out = s["offsets"].tolist(), torch.empty((c["rows"], c["N"]), dtype=torch.float64, device="cuda")
    for e in range(c["E"]):
        if ends[e] < ends[e + 1]:
            rows = torch.arange(ends[e], ends[e + 1], device="cuda")
            rows = rows if s["a_rows"] is None else s["a_rows"][rows].long()
            out[ends[e]:ends[e + 1]] = torch.mm(a[rows], _exact_weights(s["w"][e], s["w_scale"][e]).T)
    return out


def _exact_ffn(s):
    c = s["case"]
    x = _exact_rows(s["x"].double())[0]
    ends, y = s["offsets"].tolist(), torch.empty((s["src_tok"].numel(), c["D"]), dtype=torch.float64, device="cuda")
    for e in range(c["E"]):
        if ends[e] == ends[e + 1]:
            continue
        rows = x[s["src_tok"][ends[e]:ends[e + 1]].long()]
        if c["act"] == "silu":
            g, u = (torch.mm(rows, _exact_weights(s["w1"][e, i], s["w1_scale"][e, i]).T) for i in (0, 1))
            h = g * torch.sigmoid(g) * u
        else:
            h = torch.relu(torch.mm(rows, _exact_weights(s["w1"][e], s["w1_scale"][e]).T))
        y[ends[e]:ends[e + 1]] = torch.mm(_exact_rows(h)[0], _exact_weights(s["w2"][e], s["w2_scale"][e]).T)
    return y


def exact(case, seed):
    """The outputs of run() on prepare(case, seed), from the definitions in 64 bits."""
    s = prepare(case, seed)
    return {"select": _exact_select, "quantize": _exact_quantize, "gemm": _exact_gemm, "ffn": _exact_ffn}[case["op"]](s)
