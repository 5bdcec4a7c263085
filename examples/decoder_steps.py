"""A small decoder generating text-shaped nonsense: prefill of a batch of prompts, then one step a token, on this library's operators.

Every layer is  x += W_o attention(rotated q, cache)  and  x += moe_layer(norm(x)):  moe_kv_append and moe_attn_forward for the
attention half, moe_layer_forward for the expert half; the next tokens come from moe_sample.  Projections, norms and the embedding are
plain torch.  Weights are random, so the tokens mean nothing; what it shows is how the calls fit together: one PagedAttention handle and one
workspace for all layers, a cache a layer, one page table, lengths that live on the device, and a decoder step that is captured into a graph
and replayed with nothing but the random numbers and the lengths changing.

    python examples/decoder_steps.py [--layers 4 --batch 8 --prompt 200 --steps 32 --graph]
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2303_06182_amd import binding  # noqa: E402


class Decoder:
    def __init__(self, layers=4, d_model=1024, d_ff=4096, experts=16, n_heads=16, n_kv_heads=4, vocab=32000, batch=8, max_tokens=4096, page=64,
                 max_new=4096, seed=0, device="cuda:0"):
        self.n_heads, self.n_kv_heads, self.head_dim, self.d, self.vocab = n_heads, n_kv_heads, d_model // n_heads, d_model, vocab
        self.batch, self.device = batch, torch.device(device)
        g = torch.Generator(device=device)
        g.manual_seed(seed)

        def weight(*shape, std):
            return torch.empty(shape, dtype=torch.bfloat16, device=device).normal_(0.0, std, generator=g)

        kv = n_kv_heads * self.head_dim
        self.embedding = weight(vocab, d_model, std=1.0)
        self.head = weight(vocab, d_model, std=2.0 * d_model ** -0.5)
        self.layers = [dict(qkv=weight(d_model + 2 * kv, d_model, std=d_model ** -0.5), o=weight(d_model, d_model, std=d_model ** -0.5),
                            gate=weight(experts, d_model, std=d_model ** -0.5), w1=weight(experts, d_ff, d_model, std=d_model ** -0.5),
                            w2=weight(experts, d_model, d_ff, std=d_ff ** -0.5)) for _ in range(layers)]
        self.moe = binding.MoeLayer(max_new, d_model, d_ff, experts, 2, "bf16", device=device)
        per_seq = -(-max_tokens // page)
        self.attention = binding.PagedAttention(batch, max_new, n_heads, n_kv_heads, self.head_dim, page, batch * per_seq, per_seq, "bf16",
                                                rot_dim=self.head_dim, device=device)
        self.caches = [self.attention.new_cache() for _ in range(layers)]
        # every sequence has its pages from the beginning; a server hands them out as sequences grow
        self.page_table = torch.randperm(batch * per_seq, generator=g, device=device).int().view(batch, per_seq).contiguous()
        half = self.head_dim // 2
        self.inv_freq = 10000.0 ** (-torch.arange(half, dtype=torch.float64, device=device) / half)
        self.kv_len = torch.zeros(batch, dtype=torch.int32, device=device)
        self.max_tokens = max_tokens

    @staticmethod
    def _norm(x):
        return (x * torch.rsqrt(x.pow(2).mean(-1, keepdim=True) + 1e-6)).bfloat16()

    def forward(self, tokens, q_offsets, max_q, max_kv):
        """tokens [T] of all sequences, of which kv_len already counts them; -> logits [batch, vocab] of every sequence's last token."""
        x = self.embedding[tokens].float()
        T, h, hk, dim = x.shape[0], self.n_heads, self.n_kv_heads, self.head_dim
        for w, cache in zip(self.layers, self.caches):
            qkv = torch.nn.functional.linear(self._norm(x), w["qkv"])
            q = qkv[:, :h * dim].view(T, h, dim)
            k = qkv[:, h * dim:(h + hk) * dim].view(T, hk, dim)
            v = qkv[:, (h + hk) * dim:].view(T, hk, dim)
            q = self.attention.moe_kv_append(cache, q, k, v, self.inv_freq, q_offsets, self.kv_len, self.page_table, max_q)
            a, _ = self.attention.moe_attn_forward(cache, q, q_offsets, self.kv_len, self.page_table, max_q, max_kv, want_lse=False)
            x = x + torch.nn.functional.linear(a.view(T, h * dim), w["o"]).float()
            x = x + self.moe.moe_layer_forward(self._norm(x), w["gate"], w["w1"], w["w2"]).float()
        last = x[(q_offsets[1:] - 1).long()]
        return torch.nn.functional.linear(self._norm(last), self.head)

    def prefill(self, prompts):
        """prompts: a list of token lists -> logits of each one's last token."""
        n = [len(p) for p in prompts]
        offsets = torch.tensor([0] + n, device=self.device).cumsum(0).int()
        self.kv_len.copy_(torch.tensor(n, dtype=torch.int32))
        tokens = torch.tensor([t for p in prompts for t in p], device=self.device)
        return self.forward(tokens, offsets, max(n), max(n))

    def generate(self, prompts, steps, temperature=0.8, top_k=50, top_p=0.95, seed=1, graph=False):
        """-> tokens [batch, steps]; with graph, the step is captured once and replayed."""
        B = self.batch
        g = torch.Generator(device=self.device)
        g.manual_seed(seed)
        u = torch.rand((steps, B), device=self.device, generator=g)
        settings = [torch.full((B,), v, dtype=t, device=self.device) for v, t in ((temperature, torch.float32), (top_k, torch.int32), (top_p, torch.float32))]
        room = torch.empty(binding.moe_sample_workspace_bytes(B, self.vocab), dtype=torch.uint8, device=self.device)
        offsets = torch.arange(B + 1, dtype=torch.int32, device=self.device)
        token, now = torch.empty(B, dtype=torch.int32, device=self.device), torch.empty(B, device=self.device)
        out = torch.empty((steps, B), dtype=torch.int32, device=self.device)

        def choose(logits):
            binding.moe_sample(logits, now, *settings, token=token, workspace=room)

        def step():
            self.kv_len.add_(1)
            choose(self.forward(token.long(), offsets, 1, self.max_tokens))

        now.copy_(u[0])
        choose(self.prefill(prompts))
        out[0] = token
        captured = None
        if graph:  # captured on a copy of what a step changes: warming up and capturing leave no trace
            held, first = self.kv_len.clone(), token.clone()
            side = torch.cuda.Stream(self.device)
            side.wait_stream(torch.cuda.current_stream(self.device))
            with torch.cuda.stream(side):
                step()
            torch.cuda.current_stream(self.device).wait_stream(side)
            self.kv_len.copy_(held)
            token.copy_(first)
            captured = torch.cuda.CUDAGraph()
            with torch.cuda.graph(captured):
                step()
        for i in range(1, steps):
            now.copy_(u[i])
            captured.replay() if captured is not None else step()
            out[i] = token
        return out.T


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("layers", 4), ("batch", 8), ("prompt", 200), ("steps", 32)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--graph", action="store_true")
    a = ap.parse_args()
    model = Decoder(layers=a.layers, batch=a.batch, max_tokens=a.prompt + a.steps + 64, max_new=a.batch * a.prompt)
    g = torch.Generator()
    g.manual_seed(0)
    prompts = [torch.randint(0, model.vocab, (a.prompt - 7 * b % a.prompt,), generator=g).tolist() for b in range(a.batch)]
    model.generate(prompts, 2, graph=a.graph)
    torch.cuda.synchronize()
    began = time.perf_counter()
    tokens = model.generate(prompts, a.steps, graph=a.graph)
    torch.cuda.synchronize()
    s = time.perf_counter() - began
    print("%d sequences, %d tokens each in %.1f ms (prefill among it): %.0f tokens/s" % (a.batch, a.steps, s * 1e3, a.batch * a.steps / s))
    print(tokens[:, :8].tolist())


if __name__ == "__main__":
    main()
