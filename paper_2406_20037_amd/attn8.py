"""An attention layer that answers from an 8-bit cache: y = attend(x Wq, x Wk, x Wv) Wo^T.

The operators around attention as a program uses them together, with the 8-bit products of the
feed-forward layer's: tokens of several sequences go through one product for queries, keys and values, the
queries and keys are turned by their positions, keys and values go to the sequences' pages, and the
queries attend to what the pages hold.  A call takes any number of new tokens of each sequence: a whole prompt, a
chunk of one, or one token.

    python -m paper_2406_20037_amd.attn8 --width 1024 --heads 16 --kv-heads 4 --dim 64 --prompt 2000 --tokens 32

reads prompts of several sequences in chunks, then answers token by token, and prints one JSON line of times and of
how far the chunks' last outputs are from those of the prompts read at once.
"""
from __future__ import annotations

import argparse
import json
import math
import sys
import time

import torch

from . import _lib as L


def rotary_freqs(dim, base=10000.0, *, factor=1.0, trained=None, slow=1.0, fast=32.0):
    """The table of ds_rotary for `dim` turned values: base ** (-2 i / dim).  factor > 1 is for texts that much longer than
    the ``trained`` length: frequencies that make less than ``slow`` turns over it are divided by factor, those that
    make more than ``fast`` stay, and between them the change is linear in the turns; without ``trained`` all are divided."""
    f = base ** (torch.arange(0, dim, 2, dtype=torch.float64) / -dim)
    if factor != 1.0:
        if trained is None:
            f = f / factor
        else:
            keep = ((trained * f / (2 * math.pi) - slow) / (fast - slow)).clamp(0, 1)
            f = f * keep + f / factor * (1 - keep)
    return f.float()


class Attention8:
    """width -> heads of dim over kv_heads of a cache -> width, for up to ``seqs`` sequences of up to ``most`` tokens.
    w [(heads + 2 kv_heads) dim, width] holds the rows of queries, keys and values, wo [width, heads dim]."""

    def __init__(self, width, heads, kv_heads, dim, *, seqs, most, page=64, turn=None, pairs=False, window=0, freqs=None,
                 dtype=torch.float8_e4m3fn, scale=None, seed=0, device="cuda"):
        if window < 0 or most < 1:
            raise ValueError(f"window {window}, up to {most} tokens")
        freqs = rotary_freqs(dim if turn is None else turn) if freqs is None else freqs
        if 2 * freqs.numel() > dim:
            raise ValueError(f"{2 * freqs.numel()} turned values of {dim}")
        self.width, self.heads, self.kv_heads, self.dim = width, heads, kv_heads, dim
        self.seqs, self.window, self.pairs, self.device = seqs, window, pairs, device
        self.page, self.cols = page, -(-most // page)
        scale = scale or torch.float8_e8m0fnu
        gen = torch.Generator(device=device).manual_seed(seed)
        w = torch.randn((heads + 2 * kv_heads) * dim, width, generator=gen, device=device) / width ** 0.5
        wo = torch.randn(width, heads * dim, generator=gen, device=device) / (heads * dim) ** 0.5
        self.q, self.qo = (L.Q8(*m.shape, scale=scale, block_rows=L.DS_Q8_BLOCK, device=device) for m in (w, wo))
        L.ds_q8_quantize(w, self.q)
        L.ds_q8_quantize(wo, self.qo)
        self.act_scale = scale
        self.freqs = freqs.to(device)
        self.cache = L.Cache8(seqs * self.cols, kv_heads, dim, page, dtype, scale=scale, device=device)
        # pages are given out as sequences grow, the lowest free one first
        self.free = list(range(seqs * self.cols - 1, -1, -1))
        self.lengths = [0] * seqs
        self.held = [[] for _ in range(seqs)]
        self.table = torch.zeros(seqs, self.cols, dtype=torch.int32)

    def forget(self, seq):
        """The sequence begins anew; its pages are free."""
        self.free += reversed(self.held[seq])
        self.held[seq], self.lengths[seq] = [], 0

    def _grow(self, new):
        """Chunk and positions of so many new tokens of each sequence, their lengths with them and the pages that each
        takes more, which are theirs once _grown says that their rows are written."""
        if len(new) != self.seqs or min(new) < 0:
            raise ValueError(f"new tokens of {self.seqs} sequences, not {list(new)}")
        for seq, n in enumerate(new):
            if self.lengths[seq] + n > self.cols * self.page:
                raise ValueError(f"sequence {seq} would have {self.lengths[seq] + n} tokens, of {self.cols * self.page}")
        pos, starts = [], [0]
        lengths, more, taken = [], [], 0
        for seq, (first, n) in enumerate(zip(self.lengths, new)):
            lengths.append(first + n)
            more.append([])
            for col in range(len(self.held[seq]), -(-lengths[seq] // self.page)):
                taken += 1
                more[seq].append(self.free[-taken])
                self.table[seq, col] = self.free[-taken]         # (past what the sequence has, where nobody looks yet)
            pos.append(torch.arange(first, first + n, dtype=torch.int32))
            starts.append(starts[-1] + n)
        lists = (torch.tensor(starts, dtype=torch.int32), torch.tensor(lengths, dtype=torch.int32), self.table)
        return L.Chunk(*(t.to(self.device) for t in lists)), torch.cat(pos).to(self.device), lengths, more

    def _grown(self, lengths, more):
        self.lengths = lengths
        for held, pages in zip(self.held, more):
            held += pages
            del self.free[len(self.free) - len(pages):]

    def forward(self, x, new):
        """y [tokens, width] in bf16 of x [tokens, width], new[b] tokens of sequence b after another."""
        if tuple(x.shape) != (sum(new), self.width):
            raise ValueError(f"x of shape {tuple(x.shape)}, not ({sum(new)}, {self.width})")
        tokens, heads, kv = x.shape[0], self.heads, self.kv_heads

        def room(cols):
            return torch.empty(tokens, cols, dtype=torch.bfloat16, device=self.device)

        def eight(t):
            m = L.Q8(*t.shape, scale=self.act_scale, device=self.device)
            L.ds_q8_quantize(t, m)
            return m
        qkv = room((heads + 2 * kv) * self.dim)
        L.ds_q8_matmul(eight(x), self.q, qkv)
        chunk, pos, lengths, more = self._grow(new)
        qkv = qkv.view(tokens, heads + 2 * kv, self.dim)
        q, k, v = qkv.split([heads, kv, kv], 1)
        L.ds_rotary(qkv[:, :heads + kv], pos, self.freqs, pairs=self.pairs)
        L.ds_cache8_write(self.cache, chunk, k, v)
        out = torch.empty(tokens, heads, self.dim, dtype=torch.bfloat16, device=self.device)
        L.ds_attn8(q, self.cache, chunk, out, window=self.window, max_len=max(1, *lengths))
        y = room(self.width)
        L.ds_q8_matmul(eight(out.view(tokens, heads * self.dim)), self.qo, y)
        self._grown(lengths, more)
        return y


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--width", type=int, default=1024)
    ap.add_argument("--heads", type=int, default=16)
    ap.add_argument("--kv-heads", type=int, default=4)
    ap.add_argument("--dim", type=int, default=64)
    ap.add_argument("--seqs", type=int, default=4)
    ap.add_argument("--prompt", type=int, default=2000, help="tokens of the longest prompt")
    ap.add_argument("--chunk", type=int, default=512)
    ap.add_argument("--tokens", type=int, default=32, help="tokens answered")
    ap.add_argument("--window", type=int, default=0)
    args = ap.parse_args(argv)
    for name, least in dict(width=1, heads=1, kv_heads=1, dim=1, seqs=1, prompt=0, chunk=1, tokens=0, window=0).items():
        if getattr(args, name) < least:
            ap.error(f"--{name.replace('_', '-')} {getattr(args, name)}: {least} or more")

    def layer():
        return Attention8(args.width, args.heads, args.kv_heads, args.dim, seqs=args.seqs,
                          most=args.prompt + args.tokens, window=args.window, seed=1)
    gen = torch.Generator(device="cuda").manual_seed(2)
    # prompts of unequal length
    left = [max(1, args.prompt * (s + 1) // args.seqs) for s in range(args.seqs)]
    prompts = [torch.randn(n, args.width, generator=gen, device="cuda", dtype=torch.bfloat16) for n in left]
    whole = layer().forward(torch.cat(prompts), left)
    ends = torch.tensor(left).cumsum(0) - 1
    chunked, at, last = layer(), [0] * args.seqs, [None] * args.seqs
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    while any(a < n for a, n in zip(at, left)):
        new = [min(args.chunk, n - a) for a, n in zip(at, left)]
        y = chunked.forward(torch.cat([p[a:a + n] for p, a, n in zip(prompts, at, new)]), new)
        row = 0
        for s, n in enumerate(new):
            at[s], row = at[s] + n, row + n
            if n:
                last[s] = y[row - 1]
    torch.cuda.synchronize()
    prompt_ms = (time.perf_counter() - t0) * 1e3
    off = float((torch.stack(last).float() - whole[ends.cuda()].float()).norm() / whole[ends.cuda()].float().norm())
    x = torch.stack(last)
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    for _ in range(args.tokens):
        x = chunked.forward(x, [1] * args.seqs)
    torch.cuda.synchronize()
    print(json.dumps({"seqs": args.seqs, "prompt": args.prompt, "chunk": args.chunk, "prompt_ms": round(prompt_ms, 3),
                      "token_us": round((time.perf_counter() - t0) * 1e6 / max(1, args.tokens), 2), "chunks_off": off,
                      "finite": bool(torch.isfinite(x).all())}))


if __name__ == "__main__":
    sys.exit(main())
