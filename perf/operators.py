"""The attention half of a decoder step and the choice of its next token, over the range a user of this library meets.

Three operators: ``moe_kv_append`` (position rotation of new queries and keys, new keys and values into a paged cache of
e4m3 bytes with one power-of-two scale per page and head), ``moe_attn_forward`` (attention over that cache) and
``moe_sample`` (temperature, top-k, top-p and min-p from given random numbers).  Head layouts follow the repository's own
layers (1024 = 16 x 64, 2048 = 16 x 128) and generic groupings of query heads over fewer key heads; vocabularies are generic.

A case of the first two is one layer and one batch of sequences:

    op                  "append" or "attend"
    B, q_min, q_max     sequences, and the range of their new tokens (1, 1: a decoder step)
    kv_min, kv_max      range of their lengths in the cache, the new tokens among them (spread over the logarithm)
    Hq, Hkv, Dh, page   query heads, key heads, head dimension, tokens of a page
    dtype               "bf16" or "f32": queries, new keys and values, and the output
    causal, window      attend: causal mask, and how many tokens a query sees at most (0: all)
    rot, interleaved    append: rotated dimensions of a head, and whether pairs are neighbours or half of them apart

A case of ``moe_sample`` is a batch of B rows of logits over V tokens, dtype "bf16" or "f32", and which filters its rows use:
"none", "top_p", "top_k" or "mixed" (every request with its own, greedy ones and masked vocabularies among them).
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False


def _kv(name, op, B, q_min, q_max, kv_min, kv_max, Hq, Hkv, Dh, page=64, dtype="bf16", causal=True, window=0, rot=0, interleaved=False):
    c = dict(name=name, op=op, B=B, q_min=q_min, q_max=q_max, kv_min=kv_min, kv_max=kv_max, Hq=Hq, Hkv=Hkv, Dh=Dh, page=page, dtype=dtype)
    c.update(dict(causal=causal, window=window) if op == "attend" else dict(rot=rot or Dh, interleaved=interleaved))
    return c


def _sample(name, B, V, dtype, filters):
    return dict(name=name, op="sample", B=B, V=V, dtype=dtype, filters=filters)


def listed():
    return [
        # one sequence being decoded: a token's keys and values, latency alone
        _kv("append_1", "append", 1, 1, 1, 900, 900, 16, 16, 64, page=16),
        # a served batch's step; pages of 64 tokens, grouped heads, positions up to some thousands
        _kv("append_256", "append", 256, 1, 1, 1, 2000, 32, 8, 128),
        # prefill chunks of many sequences that begin and end inside pages
        _kv("append_prefill", "append", 24, 1, 2047, 1, 6000, 16, 16, 128, page=32, rot=64, interleaved=True),
        # one sequence being decoded: few keys, latency alone
        _kv("decode_1", "attend", 1, 1, 1, 900, 900, 16, 16, 64, page=16),
        # a served batch's step, lengths from one token to long ones
        _kv("decode_64", "attend", 64, 1, 1, 1, 16384, 32, 4, 128),
        # two long contexts: all of the chip on few sequences
        _kv("decode_long", "attend", 2, 1, 1, 120001, 131072, 16, 2, 128),
        # cross attention of a decoder step over encoder memory, several drafts a sequence, in fp32
        _kv("cross_f32", "attend", 32, 1, 5, 1, 1111, 16, 16, 64, page=16, dtype="f32", causal=False),
        # prefill of one long prompt: bound by the matrix cores
        _kv("prefill_8k", "attend", 1, 8192, 8192, 8192, 8192, 16, 16, 128),
        # prefill chunks of several sequences behind their histories, odd lengths, a sliding window
        _kv("prefill_chunks", "attend", 7, 100, 1500, 100, 9000, 24, 4, 128, page=32, window=4000),
        # one request's next token
        _sample("sample_1", 1, 128000, "f32", "top_p"),
        # a served batch, every request with filters of its own
        _sample("sample_64", 64, 51201, "bf16", "mixed"),
        # the largest batch and vocabulary
        _sample("sample_256", 256, 128000, "f32", "mixed"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    """One more case (without a name)."""
    kind = rng.choice(["append", "append", "decode", "decode", "decode", "prefill", "prefill", "sample", "sample", "sample"])
    if kind == "sample":
        c = _sample("", _log_int(rng, 1, 256), _log_int(rng, 500, 128000), rng.choice(["bf16", "f32"]), rng.choice(["none", "top_p", "top_k", "mixed", "mixed"]))
        del c["name"]
        return c
    Hkv = rng.choice([1, 2, 4, 8, 16])
    Hq = Hkv * rng.choice([g for g in (1, 2, 3, 4, 6, 8, 16) if 4 <= Hkv * g <= 48])
    Dh, page = rng.choice([64, 128, 128, 256]), rng.choice([16, 32, 64, 64, 128])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    width = Hkv * Dh / 1024.0
    if kind == "append":
        if rng.random() < 0.5:
            B, q_max = _log_int(rng, 1, 256), rng.choice([1, 1, 4])
        else:
            B, q_max = _log_int(rng, 1, 24), _log_int(rng, 16, 2047)
        kv_max = max(q_max, _log_int(rng, 100, max(101, min(6000, int(250000 / B / max(1.0, width))))))
        c = _kv("", "append", B, min(q_max, rng.choice([1, q_max])), q_max, 1, kv_max, Hq, Hkv, Dh, page, dtype,
                rot=rng.choice([Dh, Dh, Dh // 2]), interleaved=rng.random() < 0.4)
    elif kind == "decode":
        B, q_max = _log_int(rng, 1, 128), rng.choice([1, 1, 1, 2, 5])
        kv_max = _log_int(rng, 64, max(65, min(131072, int(400000 / B / max(1.0, width)))))
        c = _kv("", "attend", B, 1, q_max, rng.choice([1, max(1, kv_max // 2)]), kv_max, Hq, Hkv, Dh, page, dtype,
                causal=rng.random() < 0.8, window=rng.choice([0, 0, 0, _log_int(rng, 1, 4096)]))
    else:
        B, q_max = _log_int(rng, 1, 8), _log_int(rng, 17, 2000)
        kv_max = q_max + rng.choice([0, _log_int(rng, 10, 8000)])
        while 4.0 * B * q_max * kv_max * Hq * Dh > 2.7e11:  # as much as the largest listed one
            B, q_max, kv_max = (B + 1) // 2, max(17, q_max * 7 // 8), max(17, kv_max * 7 // 8)
        c = _kv("", "attend", B, rng.choice([1, q_max]), q_max, rng.choice([q_max, kv_max]), kv_max, Hq, Hkv, Dh, page, dtype,
                causal=rng.random() < 0.8, window=rng.choice([0, 0, 0, _log_int(rng, 16, 4096)]))
    del c["name"]
    return c


def _lengths(case):
    """New tokens and cached tokens of every sequence, from the case alone (work() needs them too).  The first is the longest."""
    rng = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    n, kv = [], []
    for b in range(case["B"]):
        top = case["kv_max"] if b == 0 else _log_int(rng, case["kv_min"], case["kv_max"])
        n.append(min(top, case["q_max"] if b == 0 else rng.randint(case["q_min"], case["q_max"])))
        kv.append(top)
    return n, kv


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _normal(shape, std, dtype, gen):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=gen)


def _power_of_two(n):
    """2^n in 32 bits, -126 <= n <= 127, from its bit pattern (a library's exp2 may be a rounding off)."""
    return ((n.int() + 127) << 23).view(torch.float32)


def _prepare_sample(case, gen, seed):
    B, V = case["B"], case["V"]
    rng = random.Random(seed)
    # a model's logits: probabilities that fall with a power of the rank, noise, and a sharpness of each row's own
    rank = torch.argsort(torch.rand((B, V), device="cuda", generator=gen), dim=1).float()
    sharp = torch.rand((B, 1), device="cuda", generator=gen) * 1.2 + 0.6
    logits = -sharp * torch.log(rank + 1.0) + _normal((B, V), 0.7, torch.float32, gen) + 3.0
    filters = case["filters"]
    if filters == "mixed":  # vocabularies masked by a grammar
        logits[::5].masked_fill_(torch.rand((len(range(0, B, 5)), V), device="cuda", generator=gen) < 0.5, float("-inf"))
    temperature = [rng.choice([0.6, 0.8, 1.0, 1.0, 1.3]) for _ in range(B)]
    top_k, top_p, min_p = [0] * B, [1.0] * B, [0.0] * B
    for b in range(B):
        if filters in ("top_p", "mixed"):
            top_p[b] = rng.choice([0.8, 0.9, 0.95, 1.0 if filters == "mixed" else 0.99])
        if filters in ("top_k", "mixed"):
            top_k[b] = rng.choice([1, 20, 50, 1000] + [0, 0] * (filters == "mixed"))
        if filters == "mixed":
            min_p[b] = rng.choice([0.0, 0.0, 0.02, 0.1])
            temperature[b] = rng.choice([temperature[b]] * 7 + [0.0])
    floats = lambda v: torch.tensor(v, dtype=torch.float32, device="cuda")  # noqa: E731
    return dict(case=case, logits=logits.to(torch.bfloat16 if case["dtype"] == "bf16" else torch.float32),
                u=torch.rand((B,), device="cuda", generator=gen), temperature=floats(temperature), top_k=_ints(top_k), top_p=floats(top_p),
                min_p=floats(min_p))


def prepare(case, seed):
    """One batch: the queries, keys and values of its new tokens (appending) or its rotated queries (attending), the cache as the
    steps before left it, the page table and the lengths; or one batch of logits, random numbers and each request's filters."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    if case["op"] == "sample":
        return _prepare_sample(case, gen, seed)
    B, Hq, Hkv, Dh, page = (case[n] for n in ("B", "Hq", "Hkv", "Dh", "page"))
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    n, kv = _lengths(case)
    T = sum(n)
    held = [max(1, -(-v // page)) for v in kv]
    pages, max_pages = sum(held) + 3, max(held)
    order = random.Random(seed).sample(range(pages), pages)
    table, at = [], 0
    for h in held:
        table.append(order[at:at + h] + [-1] * (max_pages - h))
        at += h
    offsets = [0]
    for v in n:
        offsets.append(offsets[-1] + v)
    s = dict(case=case, T=T, max_pages=max_pages, q_offsets=_ints(offsets), kv_len=_ints(kv), page_table=_ints(table), max_q=max(n), max_kv=max(kv))
    # what the steps before wrote: keys of about unit size (the scale is the smallest power of two that holds a page's largest one)
    for name in ("k", "v"):
        s[name + "_cache"] = _normal((pages, Hkv, page, Dh), 100.0, torch.bfloat16, gen).clamp_(-448, 448).to(torch.float8_e4m3fn)
        s[name + "_scale"] = _power_of_two(torch.randint(-8, -5, (pages, Hkv), device="cuda", generator=gen))
    if case["op"] == "append":
        # one projection's output holds the three: the views are strided
        qkv = _normal((T, (Hq + 2 * Hkv) * Dh), 1.0, dt, gen)
        # a head's keys and values have sizes of their own, and now and then a token's are large
        qkv[:, Hq * Dh:] *= _power_of_two(torch.randint(-3, 3, (2 * Hkv, 1), device="cuda", generator=gen)).to(dt).expand(-1, Dh).reshape(-1)
        qkv[::37] *= 4
        s["q"] = qkv[:, :Hq * Dh].view(T, Hq, Dh)
        s["k"] = qkv[:, Hq * Dh:(Hq + Hkv) * Dh].view(T, Hkv, Dh)
        s["v"] = qkv[:, (Hq + Hkv) * Dh:].view(T, Hkv, Dh)
        half = case["rot"] // 2
        s["inv_freq"] = 10000.0 ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half)
    else:
        s["q"] = _normal((T, Hq, Dh), 1.5, dt, gen)
        s["scale"] = 1.0 / math.sqrt(Dh)
    if own:  # the handle and the workspace that a program keeps for its layers
        from paper_2303_06182_amd import binding
        s["attention"] = binding.PagedAttention(B, T, Hq, Hkv, Dh, page, pages, max_pages, case["dtype"], rot_dim=case.get("rot", 0),
                                                interleaved=case.get("interleaved", False))
        s["cache"] = binding.KvCache(s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"])
    return s


def _tokens(s):
    """For each new token: its sequence and its position."""
    t = torch.arange(s["T"], dtype=torch.int32, device="cuda")
    b = torch.searchsorted(s["q_offsets"], t, right=True) - 1
    n = s["q_offsets"][1:] - s["q_offsets"][:-1]
    return b, (s["kv_len"] - n)[b].long() + (t - s["q_offsets"][:-1][b])


def _rotated(x, pos, inv_freq, interleaved):
    """x [T, H, Dh] at positions pos: rotated in 64 bits, rounded to 32."""
    half = inv_freq.numel()
    angle = pos.double()[:, None, None] * inv_freq
    c, w = torch.cos(angle), torch.sin(angle)
    y = x.double()
    a, b = (y[..., 0:2 * half:2], y[..., 1:2 * half:2]) if interleaved else (y[..., :half], y[..., half:2 * half])
    turned = torch.stack((a * c - b * w, b * c + a * w), -1).flatten(-2) if interleaved else torch.cat((a * c - b * w, b * c + a * w), -1)
    return torch.cat((turned, y[..., 2 * half:]), -1).float()


def _needed(largest):
    """The smallest power of two s, at least 2^-126, with largest <= 448 s."""
    mantissa, exponent = torch.frexp(largest)
    n = torch.where(mantissa <= 0.875, exponent - 9, exponent - 8)
    return _power_of_two(torch.where(largest > 0, n, -126).clamp(min=-126))


def _append_plain(s):
    c = s["case"]
    P, half_pages = c["page"], -(-s["max_q"] // c["page"]) + 1
    b, pos = _tokens(s)
    q = _rotated(s["q"], pos, s["inv_freq"], c["interleaved"]).to(s["q"].dtype)
    new = {"k": _rotated(s["k"], pos, s["inv_freq"], c["interleaved"]), "v": s["v"].float()}
    # the pages that a sequence's new tokens touch; further ones are the last of them again, with the same contents
    n = s["q_offsets"][1:] - s["q_offsets"][:-1]
    start = (s["kv_len"] - n).long()
    last = (s["kv_len"].long() - 1).clamp(min=0) // P
    at = torch.minimum(start[:, None] // P + torch.arange(half_pages, device="cuda"), last[:, None])
    ids = torch.gather(s["page_table"].long(), 1, at)
    row = at[..., None] * P + torch.arange(P, device="cuda")                      # positions [B, pages, P]
    is_new = (row >= start[:, None, None]) & (row < s["kv_len"].long()[:, None, None])
    token = (s["q_offsets"][:-1].long()[:, None, None] + row - start[:, None, None]).clamp(0, s["T"] - 1)
    is_new, is_old = is_new[:, :, None, :, None], (row < start[:, None, None])[:, :, None, :, None]
    fresh = (at * P >= start[:, None])[..., None]
    for name in ("k", "v"):
        cache, scale = s[name + "_cache"], s[name + "_scale"]
        x = new[name][token].permute(0, 1, 3, 2, 4)                                # [B, pages, H, P, Dh]
        held, before = cache[ids].float(), scale[ids]
        largest = torch.where(is_new, x.abs(), torch.zeros_like(x)).amax((-1, -2))
        after = torch.where(fresh, _needed(largest), torch.maximum(before, _needed(largest)))
        kept = torch.where(is_old, held * (before / after)[..., None, None], held).to(torch.float8_e4m3fn).float()
        written = torch.where(is_new, torch.where(is_new, x, torch.zeros_like(x)) / after[..., None, None], kept)
        cache[ids] = written.to(torch.float8_e4m3fn)
        scale[ids] = after
    return {"q": q, "k": s["k_cache"], "v": s["v_cache"], "k_scale": s["k_scale"], "v_scale": s["v_scale"]}


def _attend_plain(s):
    c = s["case"]
    B, Hq, Hkv, Dh, P = (c[n] for n in ("B", "Hq", "Hkv", "Dh", "page"))
    G, Q, L = Hq // Hkv, s["max_q"], s["max_pages"] * c["page"]
    b, pos = _tokens(s)
    first = s["q_offsets"][:-1].long()
    n = s["q_offsets"][1:].long() - first
    kv_len = s["kv_len"].long()
    key = torch.arange(L, device="cuda")
    held = (key < kv_len[:, None])[:, None, :, None]
    ids = s["page_table"].long().clamp(min=0)
    zero = torch.zeros((), device="cuda")
    k, v = (torch.where(held, (s[x + "_cache"][ids].float() * s[x + "_scale"][ids][..., None, None]).permute(0, 2, 1, 3, 4).reshape(B, Hkv, L, Dh), zero)
            for x in ("k", "v"))
    i = torch.arange(Q, device="cuda")
    rows = (first[:, None] + i).clamp(max=s["T"] - 1)
    q = s["q"].float()[rows].view(B, Q, Hkv, G, Dh).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * Q, Dh)
    at = (kv_len - n)[:, None] + i                                                 # [B, Q]
    see = (key < kv_len[:, None])[:, None, :].expand(B, Q, L)
    if c["causal"]:
        see = see & (key <= at[..., None])
    if c["window"]:
        see = see & (at[..., None] - key < c["window"])
    see = see[:, None, None]
    score = (torch.matmul(q, k.transpose(-1, -2)) * s["scale"]).view(B, Hkv, G, Q, L)
    score = torch.where(see, score, zero - math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(top == -math.inf, zero, top))
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p.view(B, Hkv, G * Q, L), v).view(B, Hkv, G, Q, Dh) / torch.where(total == 0, zero + 1, total)
    lse = (top + torch.log(total))[..., 0]
    t = torch.arange(s["T"], device="cuda") - first[b]
    return {"out": out.permute(0, 3, 1, 2, 4)[b, t].reshape(-1, Hq, Dh).to(s["q"].dtype), "lse": lse.permute(0, 3, 1, 2)[b, t].reshape(-1, Hq)}


def _sample_plain(s):
    logits = s["logits"].double()
    logits = torch.where(torch.isnan(logits), torch.full_like(logits, -math.inf), logits)
    V = logits.shape[1]
    ordered, index = torch.sort(logits, dim=1, descending=True, stable=True)
    top = ordered[:, :1]
    greedy = s["temperature"][:, None] <= 0
    z = (ordered - top) / torch.where(greedy, torch.ones_like(top), s["temperature"].double()[:, None])
    w = torch.where(ordered == top, torch.ones_like(z), torch.exp(z))
    w = torch.where(ordered == -math.inf, torch.zeros_like(z), w)
    place = torch.arange(V, device="cuda")
    k = torch.where(s["top_k"] <= 0, V, s["top_k"])[:, None]
    w = torch.where((place < torch.where(greedy, 1, k)), w, torch.zeros_like(w))
    before = torch.cumsum(w, 1) - w
    p = s["top_p"].double()[:, None]
    keep = (p >= 1) | (before < p * w.sum(1, keepdim=True)) | (place == 0)
    keep &= w >= s["min_p"].double()[:, None]
    w = torch.where(keep | (place == 0), w, torch.zeros_like(w))
    kept = torch.zeros_like(w).scatter(1, index, w)                                # vocabulary order
    total = kept.sum(1, keepdim=True)
    reached = torch.cumsum(kept, 1) > s["u"].double()[:, None] * total
    # rounding may leave the last sums short of the total: the last token kept is the answer then
    reached |= place == torch.where(kept > 0, place, torch.zeros_like(place)).amax(1, keepdim=True)
    token = torch.argmax((reached & (kept > 0)).int(), 1)
    none = top[:, 0] == -math.inf
    logprob = torch.log(torch.gather(kept, 1, token[:, None]) / total)[:, 0]
    return {"token": torch.where(none, -1, token).int(), "logprob": torch.where(none, torch.full_like(logprob, -math.inf), logprob).float()}


def run(s):
    """One pass through an operator."""
    op = s["case"]["op"]
    if not own:
        return {"append": _append_plain, "attend": _attend_plain, "sample": _sample_plain}[op](s)
    if op == "append":
        q = s["attention"].moe_kv_append(s["cache"], s["q"], s["k"], s["v"], s["inv_freq"], s["q_offsets"], s["kv_len"], s["page_table"], s["max_q"])
        return {"q": q, "k": s["k_cache"], "v": s["v_cache"], "k_scale": s["k_scale"], "v_scale": s["v_scale"]}
    if op == "attend":
        out, lse = s["attention"].moe_attn_forward(s["cache"], s["q"], s["q_offsets"], s["kv_len"], s["page_table"], s["max_q"], s["max_kv"],
                                                   scale=s["scale"], causal=s["case"]["causal"], window=s["case"]["window"])
        return {"out": out, "lse": lse}
    from paper_2303_06182_amd import binding
    token, logprob = binding.moe_sample(s["logits"], s["u"], s["temperature"], s["top_k"], s["top_p"], s["min_p"])
    return {"token": token, "logprob": logprob}


def _visible(case, n, kv):
    """Keys that are seen by all the queries of a sequence together, and by any of them."""
    total, first, i = 0, kv, np.arange(n, dtype=np.int64) + kv - n
    high = i + 1 if case["causal"] else np.full(n, kv, dtype=np.int64)
    low = np.maximum(0, i - case["window"] + 1) if case["window"] else np.zeros(n, dtype=np.int64)
    total = int(np.maximum(0, np.minimum(high, kv) - low).sum())
    first = int(low.min()) if n else kv
    return total, max(0, kv - first)


def work(case):
    """Appending: queries in and out, new keys and values in, their bytes and the scales of their pages out.  Attending: queries in,
    outputs out, the keys and values that are seen, once for each sequence and key head, and two products for each visible pair.
    Sampling: the logits, and a handful of operations for each."""
    es = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "sample":
        return {"bytes": float(case["B"] * case["V"] * es + 28 * case["B"]), "flops": 4.0 * case["B"] * case["V"]}
    Hq, Hkv, Dh = case["Hq"], case["Hkv"], case["Dh"]
    n, kv = _lengths(case)
    T = sum(n)
    if case["op"] == "append":
        pages = sum(-(-v // case["page"]) - (v - x) // case["page"] for x, v in zip(n, kv))
        return {"bytes": float(T * Dh * es * (2 * Hq + 2 * Hkv) + 2 * T * Hkv * Dh + 8 * pages * Hkv), "flops": 3.0 * T * case["rot"] * (Hq + Hkv)}
    seen = [_visible(case, x, v) for x, v in zip(n, kv)]
    return {"bytes": float(2 * T * Hq * Dh * es + 4 * T * Hq + sum(2 * x[1] * Hkv * Dh for x in seen)), "flops": 4.0 * Hq * Dh * sum(x[0] for x in seen)}


def _two_to(n):
    """2^n in 64 bits, exactly."""
    return ((n.long() + 1023) << 52).view(torch.float64)


def _e4m3(x):
    """x in 64 bits, |x| <= 448: the nearest e4m3 value, ties to even."""
    step = _two_to(torch.frexp(x)[1].clamp(min=-5) - 4)
    return torch.round(x / step) * step


def _exact_append(s):
    c = s["case"]
    P, half = c["page"], c["rot"] // 2
    offsets, kv, table = s["q_offsets"].tolist(), s["kv_len"].tolist(), s["page_table"].tolist()
    angle = torch.arange(s["max_kv"], dtype=torch.float64, device="cuda")[:, None] * s["inv_freq"]
    turn = torch.polar(torch.ones_like(angle), angle)                              # as complex numbers

    def rotated(x, begin):
        x, z = x.double().clone(), turn[begin:begin + x.shape[0], None, :]
        if c["interleaved"]:
            x[..., :2 * half] = torch.view_as_real(torch.view_as_complex(x[..., :2 * half].reshape(*x.shape[:-1], half, 2).contiguous()) * z).flatten(-2)
        else:
            y = torch.complex(x[..., :half].contiguous(), x[..., half:2 * half].contiguous()) * z
            x[..., :half], x[..., half:2 * half] = y.real, y.imag
        return x

    q = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    cache = {m: s[m + "_cache"].double() for m in "kv"}
    scale = {m: s[m + "_scale"].double() for m in "kv"}
    for b in range(c["B"]):
        lo, hi = offsets[b], offsets[b + 1]
        begin = kv[b] - (hi - lo)
        if hi == lo:
            continue
        q[lo:hi] = rotated(s["q"][lo:hi], begin)
        fresh = {"k": rotated(s["k"][lo:hi], begin).float().double(), "v": s["v"][lo:hi].double()}
        for page in range(begin // P, (kv[b] - 1) // P + 1):
            first, end = max(begin, page * P), min(kv[b], (page + 1) * P)
            r, pid = first - page * P, table[b][page]
            for m in "kv":
                x = fresh[m][first - begin:end - begin].transpose(0, 1)            # [H, rows, Dh]
                largest = x.abs().amax((1, 2))
                n = torch.floor(torch.log2((largest / 448).clamp(min=2.0 ** -126))) - 1
                n = n + (largest > 448 * _two_to(n))
                n = n + (largest > 448 * _two_to(n))
                need = _two_to((n + (largest > 448 * _two_to(n))).clamp(min=-126))
                if r:
                    need = torch.maximum(need, scale[m][pid])
                    cache[m][pid, :, :r] = _e4m3(cache[m][pid, :, :r] * (scale[m][pid] / need)[:, None, None])
                scale[m][pid] = need
                cache[m][pid, :, r:r + end - first] = _e4m3(x / need[:, None, None])
    return {"q": q, "k": cache["k"], "v": cache["v"], "k_scale": scale["k"], "v_scale": scale["v"]}


def _exact_attend(s):
    c = s["case"]
    Hq, Hkv, Dh = c["Hq"], c["Hkv"], c["Dh"]
    offsets, kv, table = s["q_offsets"].tolist(), s["kv_len"].tolist(), s["page_table"].tolist()
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full((s["T"], Hq), -math.inf, dtype=torch.float64, device="cuda")
    for b in range(c["B"]):
        lo, hi, n = offsets[b], offsets[b + 1], kv[b]
        if hi == lo or n == 0:
            continue
        ids = torch.tensor(table[b][:-(-n // c["page"])], device="cuda")
        pos, key = torch.arange(n - (hi - lo), n, device="cuda")[:, None], torch.arange(n, device="cuda")[None]
        hidden = torch.zeros((hi - lo, n), dtype=torch.bool, device="cuda")
        if c["causal"]:
            hidden |= key > pos
        if c["window"]:
            hidden |= key <= pos - c["window"]
        for h in range(Hkv):
            k, v = ((s[m + "_cache"][ids, h].double() * s[m + "_scale"][ids, h].double()[:, None, None]).reshape(-1, Dh)[:n] for m in "kv")
            for j in range(h * (Hq // Hkv), (h + 1) * (Hq // Hkv)):
                score = (s["q"][lo:hi, j].double() @ k.T * s["scale"]).masked_fill_(hidden, -math.inf)
                lse[lo:hi, j] = torch.logsumexp(score, 1)
                out[lo:hi, j] = torch.nan_to_num(torch.exp(score - lse[lo:hi, j, None])) @ v
    return {"out": out, "lse": lse}


def _exact_sample(s):
    logits, u = s["logits"].double().cpu().numpy(), s["u"].double().cpu().numpy()
    settings = [s[n].double().cpu().numpy() for n in ("temperature", "top_k", "top_p", "min_p")]
    token, logprob = [], []
    for row, r, t, k, p, m in zip(logits, u, *settings):
        order = np.argsort(-row, kind="stable")
        order = order[row[order] > -np.inf]
        if not len(order):
            token.append(-1)
            logprob.append(-math.inf)
            continue
        order = order[:1] if t <= 0 else order[:int(k)] if k > 0 else order
        w = np.exp((row[order] - row[order[0]]) / (t if t > 0 else 1.0))
        if p < 1:
            mass = np.cumsum(w)
            cut = max(1, int(np.searchsorted(mass, p * mass[-1], side="left")) + 1)
            order, w = order[:cut], w[:cut]
        order, w = order[:max(1, int((w >= m).sum()))], w[:max(1, int((w >= m).sum()))]
        by_index = np.argsort(order)
        order, w = order[by_index], w[by_index]
        mass = np.cumsum(w)
        at = min(int(np.searchsorted(mass, r * mass[-1], side="right")), len(order) - 1)
        token.append(int(order[at]))
        logprob.append(math.log(w[at] / mass[-1]))
    return {"token": torch.tensor(token, dtype=torch.int32), "logprob": torch.tensor(logprob, dtype=torch.float64)}


def exact(case, seed):
    """The outputs of run() on prepare(case, seed), from the definitions in 64 bits."""
    s = prepare(case, seed)
    return {"append": _exact_append, "attend": _exact_attend, "sample": _exact_sample}[case["op"]](s)
