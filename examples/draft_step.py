"""A decoder's step with drafted tokens, and a tuning step, on one GPU.

`Decoder` is a small stack in the shape of the paper's spiking decoder (Sec.
2.1): an embedding table, blocks of a continuous feed-forward up projection
(bias, GELU), spikes where its output passes a threshold, the spike-gated down
projection back to the residual width and an output projection added to the
residual stream, and a vocabulary head.  All weights are INT8 codes with one
FP32 scale per output, exported from random FP32 weights on the GPU.

`Decoder.verify` runs the drafted tokens of several sequences through it at
once and checks them against the head's logits; `tune` fits the embedding table
and an up projection's bias to given outputs through the frozen INT8 weights.

    python examples/draft_step.py
"""
from __future__ import annotations

import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2606_03026_amd import _binding as sp  # noqa: E402


def export(g, M, K, layout=sp.SPIKE_LAYOUT_ROW_MAJOR):
    """INT8 codes and scales of a random [M][K] weight of size 1 / sqrt(K)."""
    W = torch.randn((M, K), device="cuda", generator=g) / math.sqrt(K)
    Q = torch.empty((M, K) if layout == sp.SPIKE_LAYOUT_ROW_MAJOR else (K, M), dtype=torch.int8, device="cuda")
    scale = torch.empty(M, device="cuda")
    sp.spike_quantize_int8(W, layout, Q, scale)
    return Q, scale


def pack_spikes(bits):
    """bool [B, K] -> the library's bitmask, int64 [B, ceil(K / 64)]."""
    B, K = bits.shape
    full = torch.zeros((B, (K + 63) // 64 * 64), dtype=torch.int64, device=bits.device)
    full[:, :K] = bits
    place = torch.ones(64, dtype=torch.int64, device=bits.device) << torch.arange(64, device=bits.device)
    return (full.view(B, -1, 64) * place).sum(dim=2)


class Decoder:
    def __init__(self, vocab=2048, width=256, blocks=2, max_rows=512, seed=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.vocab, self.width, self.hidden = vocab, width, 4 * width
        self.table = torch.randn((vocab, width), device="cuda", generator=g) / math.sqrt(width)
        self.blocks = []
        for _ in range(blocks):
            up = export(g, self.hidden, width)
            out = export(g, width, width)
            down = export(g, width, self.hidden, sp.SPIKE_LAYOUT_COL_MAJOR)
            self.blocks.append({
                "up": sp.dense_fused_create(*up), "up_bias": torch.randn(self.hidden, device="cuda", generator=g) * 0.1,
                "down": sp.spike_proj_create_reserved(*down, max_rows),
                "out": sp.dense_fused_create(*out), "out_bias": torch.zeros(width, device="cuda")})
        self.head = export(g, vocab, width)

    def logits(self, ids, blocks=None):
        """Logits [rows, vocab] of token rows; `blocks`: only that many (a drafter made of the first ones)."""
        rows = ids.numel()
        x = torch.empty((rows, self.width), device="cuda")
        sp.spike_embed_forward(self.table, ids.reshape(-1).contiguous(), x, scale=math.sqrt(self.width))
        up = torch.empty((rows, self.hidden), device="cuda")
        down = torch.empty((rows, self.width), device="cuda")
        for b in self.blocks[:blocks]:
            sp.dense_fused_forward(b["up"], x, up, bias=b["up_bias"], act=sp.DENSE_ACT_GELU)
            sp.spike_proj_forward(b["down"], pack_spikes(up > 0.5), rows, down)
            sp.dense_fused_forward(b["out"], down, x, bias=b["out_bias"], residual=x)  # the residual stream, in place
        y = torch.empty((rows, self.vocab), device="cuda")
        sp.dense_proj_forward(*self.head, x, rows, y)
        return y

    def verify(self, last, temperature, n_drafts, g):
        """One speculative step of S sequences from their last tokens: the
        drafter (the first block) samples n_drafts tokens one by one, the whole
        decoder then checks them together.  Returns tokens [S, n_drafts + 1]
        (accepted drafts, the next token, -1) and how many were accepted."""
        S, G = last.numel(), n_drafts
        hot = temperature.clamp_min(1e-6)[:, None]
        drafts, dist, ids = [], [], last
        for _ in range(G):
            q = self.logits(ids, blocks=1)
            race = torch.empty_like(q).exponential_(generator=g).log_()
            ids = (q / hot - race).argmax(dim=1)
            drafts.append(ids)
            dist.append(q)
        drafts = torch.stack(drafts, dim=1)
        rows = torch.cat([last[:, None], drafts], dim=1)
        target = self.logits(rows).view(S, G + 1, self.vocab)
        tokens = torch.empty((S, G + 1), dtype=torch.int32, device="cuda")
        accepted = torch.empty(S, dtype=torch.int32, device="cuda")
        sp.head_draft_verify(target, torch.stack(dist, dim=1), drafts.to(torch.int32),
                             torch.rand((S, G), device="cuda", generator=g),
                             torch.empty((S, self.vocab), device="cuda").exponential_(generator=g).clamp_min_(1e-30),
                             tokens, accepted, temperature=temperature)
        return tokens, accepted


def tune(table, up, bias, ids, wanted, steps=20, rate=0.5):
    """Gradient steps on the embedding table and the bias, in place, of half the
    mean squared difference between GELU(up(embedding) + bias) and `wanted`,
    through frozen INT8 weights (`up` created with backward=True).  Returns the
    loss before each step."""
    T, D = ids.numel(), table.shape[1]
    x, dx = torch.empty((T, D), device="cuda"), torch.empty((T, D), device="cuda")
    y, pre = torch.empty_like(wanted), torch.empty_like(wanted)
    dtable, dbias = torch.empty_like(table), torch.empty_like(bias)
    losses = []
    for _ in range(steps):
        sp.spike_embed_forward(table, ids, x)
        sp.dense_fused_forward(up, x, y, bias=bias, act=sp.DENSE_ACT_GELU, pre=pre)
        dy = (y - wanted) / T
        losses.append(0.5 * float(((y - wanted) ** 2).sum()) / T)
        sp.dense_fused_backward(up, dy, dx=dx, dbias=dbias, pre=pre, act=sp.DENSE_ACT_GELU)
        sp.spike_embed_backward(dx, ids, dtable)
        table -= rate * dtable
        bias -= rate * dbias
    return losses


def main():
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    decoder = Decoder()
    last = torch.randint(0, decoder.vocab, (16,), device="cuda", generator=g)
    temperature = torch.full((16,), 0.8, device="cuda")
    tokens, accepted = decoder.verify(last, temperature, 4, g)
    print("accepted drafts per sequence:", accepted.tolist())
    print("tokens of the first:", tokens[0].tolist())
    Q, scale = export(g, 512, 128)
    up = sp.dense_fused_create(Q, scale, backward=True)
    table, bias = torch.randn((1000, 128), device="cuda", generator=g), torch.zeros(512, device="cuda")
    ids = torch.randint(0, 1000, (600,), device="cuda", generator=g)
    losses = tune(table, up, bias, ids, torch.randn((600, 512), device="cuda", generator=g).abs())
    print("loss before and after tuning:", round(losses[0], 3), round(losses[-1], 3))


if __name__ == "__main__":
    main()
