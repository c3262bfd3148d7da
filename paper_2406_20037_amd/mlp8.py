"""A gated feed-forward layer that computes in 8 bits: y = (silu(x Wg^T) * (x Wu^T)) W2^T.

The 8-bit operators as a program uses them together: activations quantized in blocks
of 128 with their transposes for the weights' gradients, both weights held in 8
bits with one scale a 128x128 square (masters in fp32), the gated unit's inputs kept
in 8 bits for the backward pass, gradients in e5m2, and a token at a time through
the same layer when it answers.

    python -m paper_2406_20037_amd.mlp8 --tokens 2048 --width 1024 --hidden 2816 --steps 20

trains the layer towards a fixed one of the same shape and prints one JSON line of
losses and times.
"""
from __future__ import annotations

import argparse
import json
import sys
import time

import torch

from . import _lib as L

E4M3, E5M2 = torch.float8_e4m3fn, torch.float8_e5m2
SETS = 4      # sets of buffers kept for training passes, and for others: of the latest token counts


def _up(n):
    return (n + L.DS_Q8_BLOCK - 1) // L.DS_Q8_BLOCK * L.DS_Q8_BLOCK


class Mlp8:
    """width -> hidden (gated) -> width.  w1 [up + hidden, width] holds the gate's rows, zeros up
    to ``up`` (a multiple of 128), then the other factor's; w2 [width, hidden]."""

    def __init__(self, width, hidden, *, scale=None, seed=0, device="cuda"):
        self.width, self.hidden, self.up = width, hidden, _up(hidden)
        self.scale = scale or torch.float8_e8m0fnu
        self.device = device
        gen = torch.Generator(device=device).manual_seed(seed)
        self.w1 = torch.randn(self.up + hidden, width, generator=gen, device=device) / width ** 0.5
        self.w1[hidden:self.up] = 0
        self.w2 = torch.randn(width, hidden, generator=gen, device=device) / hidden ** 0.5
        self.q1, self.q1_t = self._pair(*self.w1.shape, block_rows=L.DS_Q8_BLOCK)
        self.q2, self.q2_t = self._pair(*self.w2.shape, block_rows=L.DS_Q8_BLOCK)
        self._buffers = {True: {}, False: {}}
        self.requantize()

    def _q8(self, rows, cols, dtype=E4M3, block_rows=1):
        return L.Q8(rows, cols, dtype, scale=self.scale, block_rows=block_rows, device=self.device)

    def _pair(self, rows, cols, dtype=E4M3, block_rows=1):
        return self._q8(rows, cols, dtype, block_rows), self._q8(cols, rows, dtype, block_rows)

    def requantize(self):
        """The 8-bit weights, and their transposes, from the fp32 ones."""
        L.ds_q8_quantize(self.w1, self.q1, self.q1_t)
        L.ds_q8_quantize(self.w2, self.q2, self.q2_t)

    def _room(self, tokens, train):
        """What a pass over so many tokens writes, kept from pass to pass for the latest token counts."""
        sets = self._buffers[train]
        b = sets.pop(tokens, None)
        if b is None:
            if len(sets) == SETS:
                del sets[next(iter(sets))]                 # the one used longest ago
            wide, new = self.up + self.hidden, lambda r, c: torch.empty(r, c, dtype=torch.bfloat16,
                                                                        device=self.device)
            b = {"x": self._q8(tokens, self.width), "gu": new(tokens, wide),
                 "h": self._q8(tokens, self.hidden), "y": new(tokens, self.width)}
            if train:
                b["x_t"] = self._q8(self.width, tokens)
                b["saved"] = self._q8(tokens, wide)
                b["dy"], b["dy_t"] = self._pair(tokens, self.width, E5M2)
                b["dgu"], b["dgu_t"] = self._pair(tokens, wide, E5M2)
                b["h_t"] = self._q8(self.hidden, tokens)
                b["dh"], b["dx"] = new(tokens, self.hidden), new(tokens, self.width)
                b["dw1"], b["dw2"] = torch.empty_like(self.w1), torch.empty_like(self.w2)
        sets[tokens] = b
        return b

    def forward(self, x, train=False):
        """y [tokens, width] in bf16, in a buffer that the next call of as many tokens uses again;
        train keeps what backward needs."""
        b = self._room(x.shape[0], train)
        L.ds_q8_quantize(x, b["x"], b.get("x_t"))
        L.ds_q8_matmul(b["x"], self.q1, b["gu"])
        L.ds_swiglu8(b["gu"], b["h"], b.get("saved"))
        L.ds_q8_matmul(b["h"], self.q2, b["y"])
        return b["y"]

    def backward(self, dy):
        """(dx in bf16, dw1, dw2 in fp32) after forward(x, train=True) of as many tokens, among the latest
        SETS token counts of such calls."""
        b = self._buffers[True].get(dy.shape[0])
        if b is None:
            raise ValueError(f"no forward pass of {dy.shape[0]} tokens is kept")
        L.ds_q8_quantize(dy, b["dy"], b["dy_t"])
        L.ds_q8_matmul(b["dy"], self.q2_t, b["dh"])
        L.ds_swiglu8_grad(b["saved"], b["dh"], b["dgu"], b["dgu_t"], b["h_t"])
        L.ds_q8_matmul(b["dy_t"], b["h_t"], b["dw2"])
        L.ds_q8_matmul(b["dgu"], self.q1_t, b["dx"])
        L.ds_q8_matmul(b["dgu_t"], b["x_t"], b["dw1"])
        return b["dx"], b["dw1"], b["dw2"]

    def step(self, x, target, rate):
        """One step of gradient descent on the mean squared error; the loss before it, on the device."""
        diff = (self.forward(x, train=True) - target).float()
        _, dw1, dw2 = self.backward((diff * (2.0 / diff.numel())).to(torch.bfloat16))
        self.w1.sub_(dw1, alpha=rate)
        self.w2.sub_(dw2, alpha=rate)
        self.requantize()
        return diff.square().mean()


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--tokens", type=int, default=2048)
    ap.add_argument("--width", type=int, default=1024)
    ap.add_argument("--hidden", type=int, default=2816)
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--rate", type=float, default=None, help="default: 0.2 times the width")
    ap.add_argument("--scale", choices=["pow2", "f32"], default="pow2")
    args = ap.parse_args(argv)
    scale = torch.float8_e8m0fnu if args.scale == "pow2" else torch.float32
    layer = Mlp8(args.width, args.hidden, scale=scale, seed=1)
    teacher = Mlp8(args.width, args.hidden, scale=scale, seed=2)
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(args.tokens, args.width, generator=gen, device="cuda", dtype=torch.bfloat16)
    target = teacher.forward(x).clone()
    rate = args.rate if args.rate is not None else 0.2 * args.width
    losses = [layer.step(x, target, rate)]
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    losses += [layer.step(x, target, rate) for _ in range(args.steps - 1)]
    torch.cuda.synchronize()
    step_ms = (time.perf_counter() - t0) * 1e3 / max(1, args.steps - 1)
    token = x[:1]
    layer.forward(token)
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    for _ in range(100):
        layer.forward(token)
    torch.cuda.synchronize()
    print(json.dumps({"tokens": args.tokens, "width": args.width, "hidden": args.hidden, "scale": args.scale,
                      "loss": [round(float(v), 5) for v in losses], "step_ms": round(step_ms, 3),
                      "token_us": round((time.perf_counter() - t0) * 1e4, 2)}))


if __name__ == "__main__":
    sys.exit(main())
