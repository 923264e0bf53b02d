"""A packed matrix repaired by low-rank adapters, and served with them: what comes after a plan, on synthetic inputs.

    python -m paper_2605_26660_amd.adapt [--rows R --cols C --chunk G --steps K --tokens T --rank r]

One matrix is fitted and packed at a mix of treatments of about 2 bits.  Adapters of a few requests' kinds are then trained through
the frozen packed weights, each on activations of its own kind, towards the unquantised product (windq_project, windq_project_grad,
windq_adamw with moments in 8 bits), and a decoding batch of mixed requests, some without an adapter, is served with them.
Prints the mean squared error before and after for every kind."""
from __future__ import annotations

import argparse

import torch

from . import synth
from .binding import (ADAMW_BLOCK, Adapters, AdamwItems, Packed, n_units, project_workspace, windq_adamw, windq_apply_plan,
                      windq_fit_score_all_bits, windq_plan_layout, windq_project, windq_project_grad)

SERVED = 24                                       # requests of the decoding step
MIX = (2, 4, 5, 5, 6, 6, 4, 5, 6, 5)              # treatments of the units in turn: 2.0 bits a weight with the scales left out


def pack(W: torch.Tensor, s: torch.Tensor, chunk_w: int, unit_rows: int = 0) -> Packed:
    """W at the treatments of MIX, clip indices as the fit chose them."""
    U, R_u = n_units(W.shape[0], W.shape[1], chunk_w, unit_rows)
    action = torch.tensor([MIX[u % len(MIX)] for u in range(U)], dtype=torch.uint8)
    grid = synth.clip_grid(20)
    clip = windq_fit_score_all_bits(W, s, chunk_w, unit_rows, grid)[1]
    off = windq_plan_layout(action, R_u, chunk_w).to(W.device)
    action = action.to(W.device)
    codes, scale, offset = windq_apply_plan(W, chunk_w, unit_rows, action, clip, grid, off)
    return Packed(W, chunk_w, unit_rows, action, off, codes, scale, offset)


class Trainer:
    """Adapters of n kinds beside a packed matrix: fp32 parameters, bfloat16 working copies (what the products read), 8-bit moments."""

    def __init__(self, packed: Packed, n: int, rank: int, tokens: int, seed: int = 0):
        dev = packed.W.device
        g = torch.Generator(device=dev).manual_seed(seed)
        a = torch.randn(n, rank, packed.cols, generator=g, device=dev) / packed.cols ** 0.5
        self.params = [a, torch.zeros(n, packed.rows, rank, device=dev)]
        self.copies = [p.to(torch.bfloat16) for p in self.params]
        self.grads = [torch.empty_like(p) for p in self.params]
        bytes_of = lambda: [torch.zeros(p.shape, dtype=torch.float8_e4m3fn, device=dev) for p in self.params]
        scales = lambda: [torch.zeros((p.numel() + ADAMW_BLOCK - 1) // ADAMW_BLOCK, device=dev) for p in self.params]
        self.items = AdamwItems(self.params, self.grads, bytes_of(), bytes_of(), scales(), scales(), self.copies)
        self.packed, self.adapters = packed, Adapters(*self.copies, alpha=torch.ones(n, device=dev))
        like = torch.empty(tokens, packed.cols, dtype=torch.bfloat16, device=dev)
        serving = torch.empty(max(tokens, SERVED), packed.cols, dtype=torch.bfloat16, device=dev)
        self.ws = project_workspace(packed, serving, self.adapters)
        self.ws_grad = project_workspace(packed, like, self.adapters, grad=True)
        self.h = torch.empty(tokens, rank, device=dev)
        self.step_no = 0

    def step(self, X: torch.Tensor, of: torch.Tensor, target: torch.Tensor, lr: float) -> torch.Tensor:
        """One step on the mean squared error towards target (the gradient reaches the adapters alone). -> errors [tokens]"""
        h = self.h[: X.shape[0]]
        Y = windq_project(self.packed, X, self.adapters, of, h=h, ws=self.ws)
        off = Y.float() - target
        windq_project_grad(self.packed, (off * (2.0 / off.numel())).to(torch.bfloat16), X, self.adapters, of, h=h, ws=self.ws_grad,
                           outs=(None, *self.grads), want_dx=False)
        self.step_no += 1
        windq_adamw(self.items, self.step_no, lr)
        return off.square().mean(1)


def run(rows: int = 4096, cols: int = 4096, chunk_w: int = 128, steps: int = 60, tokens: int = 2048, rank: int = 16, kinds: int = 3,
        lr: float = 2e-3, seed: int = 0, device: str = "cuda:0"):
    """-> (errors of every kind before the first step [kinds], after the last [kinds], errors of the served batch's tokens with and
    without an adapter as the formula has them (largest relative difference))."""
    W = synth.weights_small(rows, cols, seed=seed, device=device, dtype=torch.bfloat16)
    g = torch.Generator(device=device).manual_seed(seed + 1)
    # every kind's activations live mostly in a few directions of its own: what a low rank can repair
    base = torch.randn(kinds, rank // 2, cols, generator=g, device=device)

    def draw(n):
        of = torch.randint(0, kinds, (n,), generator=g, device=device, dtype=torch.int32)
        inside = torch.randn(n, rank // 2, generator=g, device=device)
        X = 0.1 * torch.randn(n, cols, generator=g, device=device)
        for k in range(kinds):
            X += (inside * (of == k)[:, None]) @ base[k]
        return X.to(torch.bfloat16), of

    packed = pack(W, draw(1024)[0].float().abs().mean(0), chunk_w)
    trainer, full = Trainer(packed, kinds, rank, tokens, seed), W.float().t()
    first = last = None
    for k in range(steps + 1):
        X, of = draw(tokens)
        err = trainer.step(X, of, X.float() @ full, lr * (1.0 - k / (steps + 1)))
        last = torch.stack([err[of == i].mean() for i in range(kinds)])
        first = last if first is None else first
    # a decoding step, every fourth request without an adapter
    X, of = draw(SERVED)
    of[::4] = -1
    served = windq_project(packed, X, trainer.adapters, of, ws=trainer.ws).float()
    plain = windq_project(packed, X, ws=trainer.ws).float()
    a, b = (c.float() for c in trainer.copies)
    side = torch.stack([torch.zeros(rows, device=device) if k < 0 else b[k] @ (a[k] @ x) for k, x in zip(of.tolist(), X.float())])
    differs = ((served - plain - side).abs().max() / plain.abs().max()).item()
    return first.tolist(), last.tolist(), differs


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    for name, default in (("rows", 4096), ("cols", 4096), ("chunk", 128), ("steps", 60), ("tokens", 2048), ("rank", 16)):
        ap.add_argument("--" + name, type=int, default=default)
    p = ap.parse_args()
    first, last, differs = run(p.rows, p.cols, p.chunk, p.steps, p.tokens, p.rank)
    for k, (x, y) in enumerate(zip(first, last)):
        print(f"kind {k}: mean squared error {x:.3e} packed, {y:.3e} with its adapter after {p.steps} steps")
    print(f"served batch of {SERVED} requests: {differs:.1e} off the sum of its parts")


if __name__ == "__main__":
    main()
