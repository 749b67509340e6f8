"""One decoder layer and an output projection on the library's operators, prompts and single tokens.

    python examples/decoder_layer.py

The layer's projections are MosaicQuant weights (W4A8 behind the norms, whose 8-bit output is their
operand, W4A4 for the others), the output projection is an 8-bit weight, and keys and values live in the
paged 4-bit cache.  With ``fp8`` the projection is in e4m3 with scales for blocks of 128, and the cache in e4m3 with
scales for blocks of 32 tokens.  Tokens are drawn from the logits.  Positions are left out; weights and tokens are
random.
"""
from __future__ import annotations

import os
import sys
from dataclasses import dataclass

import torch

if __name__ == "__main__":
    sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2606_15652_amd as mq

EPS = 1e-5


@dataclass
class Layer:
    heads: int
    kv_heads: int
    head_dim: int
    norm1: torch.Tensor
    norm2: torch.Tensor
    norm3: torch.Tensor
    qkv: mq.PackedWeight
    o: mq.PackedWeight
    gate_up: mq.PackedWeight
    down: mq.PackedWeight
    out: mq.PackedWeight8 | mq.PackedWeightFP8


def random_layer(hidden: int, heads: int, kv_heads: int, head_dim: int, ffn: int, vocab: int, seed: int = 0,
                 fp8: bool = False) -> Layer:
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def weight(n, k):
        return torch.randn((n, k), generator=gen, device="cuda") / k ** 0.5

    def packed(n, k):
        return mq.prepare_weight(weight(n, k), (n // 128) * (k // 128) // 10)       # a tenth of the blocks with a residual

    def gamma():
        return (1.0 + 0.1 * torch.randn(hidden, generator=gen, device="cuda")).half()

    return Layer(heads, kv_heads, head_dim, gamma(), gamma(), gamma(),
                 packed((heads + 2 * kv_heads) * head_dim, hidden), packed(hidden, heads * head_dim),
                 packed(2 * ffn, hidden), packed(hidden, ffn),
                 (mq.quantize_weight_fp8 if fp8 else mq.quantize_weight8)(weight(vocab, hidden)))


class Batch:
    """Sequences in a paged cache: which pages each has, and how many tokens."""

    def __init__(self, layer: Layer, sequences: int, most_tokens: int, page: int = 64, fp8: bool = False):
        per = -(-most_tokens // page)
        self.page = page
        self.cache = (mq.kv8_cache if fp8 else mq.kv4_cache)(sequences * per, page, layer.kv_heads, layer.head_dim)
        # pages of a sequence need not be neighbours
        self.table = torch.randperm(sequences * per, device="cuda").int().reshape(sequences, per)
        self.lens = [0] * sequences

    def add(self, counts):
        """Slots of the next counts[b] tokens of each sequence, and the lengths with them."""
        slots = []
        for b, n in enumerate(counts):
            t = torch.arange(self.lens[b], self.lens[b] + n, device="cuda")
            slots.append(self.table[b, t // self.page].long() * self.page + t % self.page)
            self.lens[b] += n
        return torch.cat(slots), torch.tensor(self.lens, dtype=torch.int32, device="cuda")


def forward(layer: Layer, batch: Batch, x: torch.Tensor, counts) -> torch.Tensor:
    """x [tokens, hidden]: the next counts[b] tokens of each sequence, one after the other -> logits in fp32."""
    slots, lens = batch.add(counts)
    starts = torch.tensor([0, *counts], device="cuda").cumsum(0).int()
    d, hq, hk = layer.head_dim, layer.heads, layer.kv_heads

    codes, scale = mq.rms_norm_quantize8(x, layer.norm1, EPS, layout="a8")
    qkv = mq.fused_gemm_a8(codes, scale, layer.qkv).view(-1, hq + 2 * hk, d)
    single = max(counts) == 1 and min(counts) == 1
    if isinstance(batch.cache, mq.KVCache8):
        mq.kv8_append(batch.cache, qkv[:, hq:hq + hk], qkv[:, hq + hk:], batch.table, lens, cu_new=None if single else starts)
        attend = mq.attention_kv8
    else:
        mq.kv4_append(batch.cache, qkv[:, hq:hq + hk], qkv[:, hq + hk:], slots)
        attend = mq.attention_kv4
    attended = attend(qkv[:, :hq], batch.cache, batch.table, lens, cu_q=None if single else starts, max_q=max(counts),
                      max_kv=max(batch.lens))
    y = mq.linear(attended.view(-1, hq * d), layer.o)

    codes, scale, x = mq.rms_norm_quantize8(y, layer.norm2, EPS, residual=x, layout="a8")
    gate, up = mq.fused_gemm_a8(codes, scale, layer.gate_up).chunk(2, dim=1)
    y = mq.linear(torch.nn.functional.silu(gate) * up, layer.down)

    if isinstance(layer.out, mq.PackedWeightFP8):
        x = torch.nn.functional.rms_norm(x.float() + y.float(), (x.shape[1],), layer.norm3.float(), EPS).to(x.dtype)
        return mq.gemm_fp8(*mq.quantize_rows_fp8(x), layer.out, out_dtype=torch.float32)
    codes, scale, x = mq.rms_norm_quantize8(y, layer.norm3, EPS, residual=x)
    return mq.gemm_w8a8(codes, scale, layer.out, out_dtype=torch.float32)


def draw(logits: torch.Tensor, gen: torch.Generator, temperature=0.8, top_k=50, top_p=0.95) -> torch.Tensor:
    """A token for each row, from the generator's numbers."""
    u = torch.rand(logits.shape[0], generator=gen, device=logits.device)
    return mq.sample(logits, u, temperature, top_k=top_k, top_p=top_p)[0]


def main():
    for fp8 in (False, True):
        layer = random_layer(hidden=1024, heads=16, kv_heads=4, head_dim=64, ffn=2048, vocab=10007, fp8=fp8)
        counts = [100, 37, 64]
        batch = Batch(layer, len(counts), 256, fp8=fp8)
        gen = torch.Generator(device="cuda")
        gen.manual_seed(0)
        x = torch.randn((sum(counts), 1024), device="cuda").half()
        logits = forward(layer, batch, x, counts)
        print("8-bit floating point" if fp8 else "integers", "- prompts of", counts, "tokens: logits", tuple(logits.shape))
        for step in range(4):
            logits = forward(layer, batch, torch.randn((len(counts), 1024), device="cuda").half(), [1] * len(counts))
            print("token", step + 1, "lengths", batch.lens, "drawn", draw(logits, gen).tolist())


if __name__ == "__main__":
    main()
