"""One transformer layer from a prompt to decoded tokens: the prompt in bf16 and mini-sequences, the cache and the decoded tokens in four bits.

    python examples/decode_four_bits.py [--prompt 8192] [--tokens 32] [--hidden 4096] [--intermediate 14336]

Prompt: keys and values of a chunk go to the paged cache with the rotation on the way (mom_mx_kv_append), the chunk attends over the cache
(mom_mx_attention), the MLP runs in mini-sequences (mom_mlp_prefill) while the pages that the chunk filled leave for page-locked memory
(mom_kv_offload).  Decoding: the pages come back (mom_kv_reload), and each token is four products with four-bit weights (mom_mx_matvec,
mom_mx_gateup), one append and one attention.  Weights and inputs are synthetic; norms and the prompt's projections are torch's.
"""
import argparse
import math
import os
import sys
import time

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
from paper_2504_12526_amd import binding  # noqa: E402


def rms_norm(x):
    y = x.float()
    return (y * torch.rsqrt(y.pow(2).mean(-1, keepdim=True) + 1e-5)).to(torch.bfloat16)


class FourBits:
    """A weight [N, K] bf16 in four bits."""

    def __init__(self, w):
        n, k = w.shape
        self.codes = torch.empty((n, k // 2), dtype=torch.uint8, device=w.device)
        self.scales = torch.empty((n, k // 32), dtype=torch.uint8, device=w.device)
        binding.mom_mx_quantize(w, self.codes, self.scales)

    def values(self):
        """What it stands for, exactly, as bf16."""
        table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], device=self.codes.device)
        v = table[torch.stack((self.codes & 15, self.codes >> 4), -1).flatten(-2).long()].unflatten(-1, (-1, 32))
        return (v * torch.exp2(self.scales.float() - 127).unsqueeze(-1)).flatten(-2).to(torch.bfloat16)


class Layer:
    """Weights, cache and buffers of one layer and one sequence of up to `most` tokens."""

    def __init__(self, hidden, intermediate, heads, kv_heads, head_dim, most, page_tokens=64, rope_base=500000.0, seed=0, device="cuda"):
        gen = torch.Generator(device=device).manual_seed(seed)

        def weight(n, k):
            return (torch.randn((n, k), generator=gen, device=device) / math.sqrt(k)).to(torch.bfloat16)

        self.heads, self.kv_heads, self.d, self.page, self.most = heads, kv_heads, head_dim, page_tokens, most
        width = (heads + 2 * kv_heads) * head_dim
        self.four = {n: FourBits(weight(*s)) for n, s in (("qkv", (width, hidden)), ("out", (hidden, heads * head_dim)), ("gate", (intermediate, hidden)),
                                                          ("up", (intermediate, hidden)), ("down", (hidden, intermediate)))}
        # the prompt runs on the same weights, as bf16
        self.w = {n: q.values() for n, q in self.four.items()}
        pages = -(-most // page_tokens)
        self.cache = torch.zeros((pages, kv_heads, binding.mom_mx_block_bytes(head_dim, page_tokens)), dtype=torch.uint8, device=device)
        self.table = torch.arange(pages, dtype=torch.int32, device=device)[None]
        self.inv_freq = (rope_base ** (-torch.arange(0, head_dim, 2, dtype=torch.float64, device=device) / head_dim)).float()
        # a decoded token: everything at its place beforehand, so that a step is launches alone (and can be captured)
        bf = dict(dtype=torch.bfloat16, device=device)
        self.qkv, self.h = torch.empty((1, width), **bf), torch.empty((1, intermediate), **bf)
        self.q, self.o = (torch.empty((1, heads, head_dim), **bf) for _ in range(2))
        self.place = torch.zeros(1, dtype=torch.int32, device=device)
        self.slot, self.length = torch.zeros(1, dtype=torch.int64, device=device), torch.zeros(1, dtype=torch.int32, device=device)
        self.workspace = torch.empty(binding.mom_mx_attention_workspace_bytes(1, 1, heads, kv_heads, head_dim, most), dtype=torch.uint8, device=device)

    def _split(self, qkv):
        t = qkv.view(qkv.shape[0], -1, self.d)
        return t[:, :self.heads], t[:, self.heads:self.heads + self.kv_heads], t[:, self.heads + self.kv_heads:]

    def prompt(self, x, chunk=2048, mini_seq=1024, offload=None):
        """The layer's output for the tokens x [S, H] bf16, a chunk at a time.  offload: (page-locked uint8 tensor of the cache's size, side
        stream): the pages of a chunk leave under its MLP."""
        S, H = x.shape
        out = torch.empty_like(x)
        for lo in range(0, S, chunk):
            hi = min(S, lo + chunk)
            q, k, v = self._split(rms_norm(x[lo:hi]) @ self.w["qkv"].t())
            at = torch.arange(lo, hi, device=x.device)
            rotated, o = (torch.empty((hi - lo, self.heads, self.d), dtype=torch.bfloat16, device=x.device) for _ in range(2))
            binding.mom_mx_kv_append(k, v, at, self.cache, self.page, positions=at.to(torch.int32), inv_freq=self.inv_freq, q=q, q_out=rotated)
            ws = torch.empty(binding.mom_mx_attention_workspace_bytes(hi - lo, 1, self.heads, self.kv_heads, self.d, hi), dtype=torch.uint8, device=x.device)
            binding.mom_mx_attention(rotated, self.cache, self.page, self.table, torch.tensor([hi], dtype=torch.int32, device=x.device), hi, o, ws)
            if offload:
                # whole pages as they lie, two halves of the bytes as k and v
                host, side = offload
                first, last = lo // self.page, -(-hi // self.page)
                each = self.cache[0].numel()
                moved = self.cache[first:last].view(-1)
                half = moved.numel() // 2
                order = torch.cuda.Event()
                order.record()
                binding.mom_kv_offload(moved[:half], moved[half:], host[first * each:last * each], side, producer_stream=torch.cuda.current_stream(), order_event=order)
            y = x[lo:hi] + o.view(hi - lo, -1) @ self.w["out"].t()
            mlp = torch.empty_like(y)
            mws = torch.empty(binding.mom_mlp_workspace_bytes(hi - lo, H, self.w["gate"].shape[0], mini_seq), dtype=torch.uint8, device=x.device)
            binding.mom_mlp_prefill(rms_norm(y), self.w["gate"], self.w["up"], self.w["down"], mini_seq, mlp, mws)
            out[lo:hi] = y + mlp
        return out

    def restore(self, host, stream):
        """The cache back from page-locked memory before decoding."""
        flat = self.cache.view(-1)
        half = flat.numel() // 2
        binding.mom_kv_reload(host, flat[:half], flat[half:], stream)

    def set_place(self, position):
        self.place.fill_(position)
        self.slot.fill_(position)                     # the pages of this sequence lie in order
        self.length.fill_(position + 1)

    def token(self, x):
        """The layer's output for one token x [1, H] at the place that set_place said: launches on the current stream alone."""
        four = self.four
        binding.mom_mx_matvec(rms_norm(x), four["qkv"].codes, four["qkv"].scales, self.qkv)
        q, k, v = self._split(self.qkv)
        binding.mom_mx_kv_append(k, v, self.slot, self.cache, self.page, positions=self.place, inv_freq=self.inv_freq, q=q, q_out=self.q)
        binding.mom_mx_attention(self.q, self.cache, self.page, self.table, self.length, self.most, self.o, self.workspace)
        y = torch.empty_like(x)
        binding.mom_mx_matvec(self.o.view(1, -1), four["out"].codes, four["out"].scales, y, residual=x)
        binding.mom_mx_gateup(rms_norm(y), four["gate"].codes, four["gate"].scales, four["up"].codes, four["up"].scales, self.h)
        binding.mom_mx_matvec(self.h, four["down"].codes, four["down"].scales, y, residual=y)
        return y


def main():
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--prompt", type=int, default=8192)
    p.add_argument("--tokens", type=int, default=32)
    p.add_argument("--hidden", type=int, default=4096)
    p.add_argument("--intermediate", type=int, default=14336)
    p.add_argument("--heads", type=int, default=32)
    p.add_argument("--kv-heads", type=int, default=8)
    a = p.parse_args()
    if a.prompt < 1 or a.tokens < 1:
        p.error("--prompt and --tokens are at least 1")
    layer = Layer(a.hidden, a.intermediate, a.heads, a.kv_heads, 128, a.prompt + a.tokens)
    x = torch.randn((a.prompt, a.hidden), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(torch.bfloat16)
    host, side = torch.empty(layer.cache.numel(), dtype=torch.uint8, pin_memory=True), torch.cuda.Stream()
    y = layer.prompt(x, offload=(host, side))
    torch.cuda.current_stream().wait_stream(side)
    layer.cache.zero_()
    layer.restore(host, torch.cuda.current_stream())
    t = y[-1:].contiguous()
    step_in = t.clone()
    layer.set_place(a.prompt)
    layer.token(step_in)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step_out = layer.token(step_in)
    begun = time.perf_counter()
    for i in range(a.tokens):
        layer.set_place(a.prompt + i)
        step_in.copy_(t)
        graph.replay()
        t = step_out.clone()
    torch.cuda.synchronize()
    each = (time.perf_counter() - begun) / a.tokens
    print(f"{a.prompt} tokens of prompt, {a.tokens} decoded: {each * 1e6:.1f} us a token of one layer; last token rms {t.float().pow(2).mean().sqrt().item():.3f}")


if __name__ == "__main__":
    main()
