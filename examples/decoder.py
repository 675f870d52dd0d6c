"""A small decoder of linear-attention and gated blocks: trained on one packed row of
sequences (a few patterns over and over), then prompted and continued a token at a time.

    python examples/decoder.py [--steps 60] [--width 512] [--layers 4] [--blocks ag] [--rotary 32]

Tokens enter through ``embedding``.  An attention block ("a") is ``residual_norm`` (the
norm with the residual addition), one projection to q, k, v, the gate z and the decays,
``head_norm`` of q and k (with ``rotary``, turned by their positions), ``linear_attn`` and
``gated_norm`` over each head; q, k, v and z stay slices of the projection's rows.  A
gated block ("g") projects to x, its gates and z and runs ``gated_scan`` in place of
attention, a group of its norm for each ``head`` channels.  ``blocks`` is the pattern the
layers repeat.  Training runs the operators' autograd functions, ``prompt`` the packed
forward, which leaves every sequence's state, and ``decode`` the one-token step on a pool
of those states.
"""
import argparse
import os
import sys

import torch
from torch import nn
from torch.nn import functional as F

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2606_00601_amd as sw  # noqa: E402


class Block(nn.Module):
    """Heads of ``head`` columns, every ``share`` of them on one q and k."""

    def __init__(self, width, head=64, share=2, rotary=0):
        super().__init__()
        self.H, self.Hk, self.head = width // head, width // head // share, head
        self.cols = [self.Hk * head, self.Hk * head, self.H * head, self.H * head, self.H]
        self.norm = nn.Parameter(torch.ones(width))
        self.out_norm = nn.Parameter(torch.ones(width))
        self.res_scale = nn.Parameter(torch.ones(width))
        self.rate = nn.Parameter(torch.linspace(-4.0, 0.0, self.H))  # log of the decays' rates
        self.inp = nn.Linear(width, sum(self.cols), bias=False, dtype=torch.bfloat16)
        self.out = nn.Linear(width, width, bias=False, dtype=torch.bfloat16)
        freq = 1000.0 ** (-torch.arange(0, rotary, 2) / rotary) if rotary else None
        self.register_buffer("freq", freq, persistent=False)

    def _project(self, y, positions, head_norm):
        """(..., width) -> q, k (..., Hk, head), v (..., H, head), z (..., width), g (..., H).
        The norms leave q and k head ** 0.5 long: ``scale`` takes that back."""
        q, k, v, z, d = self.inp(y).split(self.cols, dim=-1)
        q, k = head_norm(*(t.unflatten(-1, (self.Hk, self.head)) for t in (q, k)),
                         positions=positions if self.freq is not None else None, inv_freq=self.freq)
        g = -F.softplus(d.float()) * self.rate.exp()
        return q, k, v.unflatten(-1, (self.H, self.head)), z, g

    def forward(self, x, res, cu, positions, last_state=False):
        """x, the block before's output, joins the residual stream res; (1, L, width)
        rows of packed sequences.  Returns (output, stream, the sequences' last states)."""
        norm, attn, gate = sw.residual_norm_fn, sw.linear_attn_fn, sw.gated_norm_fn
        y, res = norm(x, self.norm, res, res_scale=self.res_scale)
        q, k, v, z, g = self._project(y, positions, sw.head_norm_fn)
        how = dict(scale=1.0 / self.head, cu_seqlens=cu)
        o, state = attn(q, k, v, g, return_last_state=True, **how) if last_state else \
            (attn(q, k, v, g, **how), None)
        y = gate(o.flatten(-2), z, self.out_norm, group=self.head)
        return self.out(y), res, state

    def step(self, x, res, pool, slots, positions):
        """One token of each sequence: (B, width), the states pool[slots] in place."""
        y, res = sw.residual_norm_fwd(x, self.norm, res, res_scale=self.res_scale)
        q, k, v, z, g = self._project(y, positions, sw.head_norm_fwd)
        o = sw.linear_attn_step(q, k, v, g, pool, scale=1.0 / self.head, slots=slots)
        return self.out(sw.gated_norm_fwd(o.flatten(-2), z, self.out_norm, group=self.head)), res


class GatedBlock(nn.Module):
    """The gated recurrence of ``width`` channels in place of attention."""

    def __init__(self, width, head=64):
        super().__init__()
        self.width, self.head = width, head
        self.norm = nn.Parameter(torch.ones(width))
        self.out_norm = nn.Parameter(torch.ones(width))
        self.res_scale = nn.Parameter(torch.ones(width))
        # an open gate's decay from 0.9 to 0.999: c softplus(lam) is minus its logarithm
        decay = torch.linspace(0.9, 0.999, width)
        self.lam = nn.Parameter(torch.log(torch.expm1(-decay.log() / 8.0)))
        self.inp = nn.Linear(width, 4 * width, bias=False, dtype=torch.bfloat16)
        self.out = nn.Linear(width, width, bias=False, dtype=torch.bfloat16)

    def forward(self, x, res, cu, positions, last_state=False):
        y, res = sw.residual_norm_fn(x, self.norm, res, res_scale=self.res_scale)
        x, r, i, z = self.inp(y).split(self.width, dim=-1)
        h, state = sw.gated_scan_fn(x, r, i, self.lam, cu_seqlens=cu, return_last_state=True) \
            if last_state else (sw.gated_scan_fn(x, r, i, self.lam, cu_seqlens=cu), None)
        return self.out(sw.gated_norm_fn(h, z, self.out_norm, group=self.head)), res, state

    def step(self, x, res, pool, slots, positions):
        y, res = sw.residual_norm_fwd(x, self.norm, res, res_scale=self.res_scale)
        x, r, i, z = self.inp(y).split(self.width, dim=-1)
        h = sw.gated_scan_step(x, r, i, self.lam, pool, slots=slots)
        return self.out(sw.gated_norm_fwd(h, z, self.out_norm, group=self.head)), res


class Decoder(nn.Module):
    def __init__(self, vocab=256, width=512, layers=4, blocks="a", rotary=0):
        super().__init__()
        self.embed = nn.Embedding(vocab, width)
        kinds = {"a": lambda: Block(width, rotary=rotary), "g": lambda: GatedBlock(width)}
        self.blocks = nn.ModuleList(kinds[blocks[n % len(blocks)]]() for n in range(layers))
        self.norm = nn.Parameter(torch.ones(width))
        self.head = nn.Linear(width, vocab, bias=False, dtype=torch.bfloat16)

    def _start(self, tokens, embedding):
        x = embedding(tokens, self.embed.weight, dtype=torch.bfloat16)
        return x, torch.zeros(x.shape, device=x.device)  # the residual stream is fp32

    @staticmethod
    def _positions(tokens, cu):
        """Of packed rows (1, L): each sequence's from 0 on."""
        at = torch.arange(tokens.shape[1], device=tokens.device, dtype=torch.int32)
        n = torch.searchsorted(cu[1:].contiguous(), at, right=True).clamp_(max=cu.numel() - 2)
        return (at - cu[n])[None]

    def forward(self, tokens, cu):
        """Logits (1, L, vocab) of packed rows of tokens (1, L)."""
        x, res = self._start(tokens, sw.embedding_fn)
        positions = self._positions(tokens, cu)
        for b in self.blocks:
            x, res, _ = b(x, res, cu, positions)
        y, _ = sw.residual_norm_fn(x, self.norm, res)
        return self.head(y)

    @torch.no_grad()
    def prompt(self, tokens, cu):
        """(logits of every step, the blocks' states after each sequence)."""
        x, res = self._start(tokens, sw.embedding_fwd)
        positions = self._positions(tokens, cu)
        states = []
        for b in self.blocks:
            x, res, s = b(x, res, cu, positions, last_state=True)
            states.append(s)
        y, _ = sw.residual_norm_fwd(x, self.norm, res)
        return self.head(y), states

    @torch.no_grad()
    def decode(self, tokens, pools, slots, positions=None):
        """Logits (B, vocab) after one more token (B,) of each sequence, at ``positions``
        (B,), which only rotary blocks need."""
        x, res = self._start(tokens, sw.embedding_fwd)
        for b, pool in zip(self.blocks, pools):
            x, res = b.step(x, res, pool, slots, positions)
        y, _ = sw.residual_norm_fwd(x, self.norm, res)
        return self.head(y)


def packed(lens, patterns, gen, device):
    """A packed row of sequences, each one of the patterns (n, period) over and over."""
    rows, period = [], patterns.shape[1]
    for n in lens:
        pattern = patterns[torch.randint(0, len(patterns), (), generator=gen)]
        rows.append(pattern.repeat((n + period - 1) // period)[:n])
    cu = torch.tensor([0] + list(lens)).cumsum(0).to(torch.int32)
    return torch.cat(rows)[None].to(device), cu.to(device)


def train(model, patterns, steps, gen, lens=(700, 129, 1, 512, 64), log=print):
    opt = torch.optim.AdamW(model.parameters(), lr=1e-3)
    losses = []
    for i in range(steps):
        tokens, cu = packed(lens, patterns, gen, "cuda")
        target = tokens[0].roll(-1).clone()
        target[(cu[1:] - 1).long()] = -100  # a sequence's last token has no successor
        loss = F.cross_entropy(model(tokens, cu)[0].float(), target)
        opt.zero_grad()
        loss.backward()
        opt.step()
        losses.append(loss.item())
        if log and (i % 10 == 0 or i == steps - 1):
            log(f"step {i}: loss {losses[-1]:.3f}", flush=True)
    return losses


def generate(model, tokens, cu, steps):
    """Greedy continuations (n, steps) of n packed prompts, none of them empty."""
    logits, states = model.prompt(tokens, cu)
    slots = torch.arange(len(cu) - 1, dtype=torch.int32, device=tokens.device)
    token = logits[0, (cu[1:] - 1).long()].argmax(-1)
    out = [token]
    lengths = cu[1:] - cu[:-1]
    for i in range(steps - 1):
        token = model.decode(token, states, slots, lengths + i).argmax(-1)
        out.append(token)
    return torch.stack(out, dim=1)


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--width", type=int, default=512)
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--blocks", default="a", help="pattern of attention (a) and gated (g) blocks")
    ap.add_argument("--rotary", type=int, default=0, help="columns of q and k turned by position")
    args = ap.parse_args()
    torch.manual_seed(0)
    gen = torch.Generator().manual_seed(0)
    model = Decoder(width=args.width, layers=args.layers, blocks=args.blocks, rotary=args.rotary).cuda()
    patterns = torch.randint(0, 256, (8, 12), generator=gen)
    train(model, patterns, args.steps, gen)
    tokens, cu = packed((36, 50, 24), patterns, gen, "cuda")
    got = generate(model, tokens, cu, 12)
    for n in range(3):
        row = tokens[0, int(cu[n]):int(cu[n + 1])].tolist()
        want = [row[(len(row) + i) % 12] for i in range(12)]
        hit = sum(a == b for a, b in zip(got[n].tolist(), want))
        print(f"prompt of {len(row)}: {hit} of 12 tokens continue its pattern")


if __name__ == "__main__":
    main()
