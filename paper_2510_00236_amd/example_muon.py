"""Training a pre-norm MLP block: Muon on its weight matrices, MicroAdam on the scale and offset of its norm.

    python -m paper_2510_00236_amd.example_muon            # GPT-2-small widths, a teacher's outputs as targets

The block is y = x + f(norm(x) W1) W2 with f(a) = a sigmoid(a).  A step calls, in this order (everything on the GPU, nothing synchronises with the host):
  1. pex_layer_norm, which keeps mean and 1/std of every row; the two products of the forward pass are torch's;
  2. the products of the backward pass (torch), then pex_layer_norm_grad: the cotangents of the norm's input (a layer before the block would
     receive their sum with those of its output, the residual path's), and S_id and S_sq of scale and offset, whose per-example gradients
     are sums over the sequence;
  3. pex_stat(identity) of the two matrices: the sum of their gradients over the batch;
  4. pex_muon_step of the matrices, pex_adam_step (MicroAdam, clipped by the global norm of the two vectors) of scale and offset.
"""
from __future__ import annotations

import argparse
import time

import torch

import paper_2510_00236_amd as pex

BOTH = ("identity", "square")


class Block:
    """Parameters (fp32), their optimizer state and every buffer a step needs."""

    def __init__(self, B, T, d, hidden, dev, seed=0):
        g = torch.Generator(device=dev).manual_seed(seed)
        rnd = lambda *s: torch.randn(*s, device=dev, generator=g)
        self.shape = (B, T, d, hidden)
        self.W = [rnd(d, hidden) * d ** -0.5, rnd(hidden, d) * hidden ** -0.5]
        self.W_m = [torch.zeros_like(w) for w in self.W]
        self.S = [torch.empty_like(w) for w in self.W]
        self.vectors = {"scale": torch.ones(d, device=dev), "offset": torch.zeros(d, device=dev)}
        self.vec_m = {k: torch.zeros(d, device=dev) for k in self.vectors}
        self.vec_v = {k: torch.zeros(d, device=dev) for k in self.vectors}
        self.vec_S = {k: {n: torch.empty(d, device=dev) for n in BOTH} for k in self.vectors}
        self.norm = (torch.empty(B, T, d, dtype=torch.bfloat16, device=dev), torch.empty(B, T, device=dev), torch.empty(B, T, device=dev))
        self.dx = torch.empty(B, T, d, dtype=torch.bfloat16, device=dev)
        self.sum_sq = torch.zeros(1, dtype=torch.float64, device=dev)
        code = pex.PEX_BF16
        need = [pex.pex_layer_norm_grad_workspace_bytes(B, T, d, code, BOTH), pex.pex_stat_workspace_bytes(B, T, d, hidden, code, "identity"),
                pex.pex_stat_workspace_bytes(B, T, hidden, d, code, "identity"), pex.pex_muon_step_workspace_bytes([tuple(w.shape) for w in self.W]),
                pex.pex_adam_step_workspace_bytes([d, d])]
        self.ws = torch.empty(max(need), dtype=torch.uint8, device=dev)


def train_step(block, x, target, step, lr=0.02, vector_lr=1e-3):
    """One step towards y = target; returns the mean squared error before it (on the GPU)."""
    B, T, d, hidden = block.shape
    ws = block.ws
    W1, W2 = (w.bfloat16() for w in block.W)
    # 1. forward
    h, mean, rstd = pex.pex_layer_norm(x, block.vectors["scale"], block.vectors["offset"], out=block.norm)
    a = h.view(B * T, d) @ W1
    gate = torch.sigmoid(a)
    r = a * gate
    y = x + (r @ W2).view(B, T, d)
    error = y.float() - target.float()
    # 2. backward: cotangents of the mean over the batch's tokens of half the squared error
    G2 = (error / T).bfloat16()
    G1 = (G2.view(B * T, d) @ W2.t()) * (gate + r * (1 - gate))
    Gh = (G1 @ W1.t()).view(B, T, d)
    pex.pex_layer_norm_grad(Gh, x, mean, rstd, block.vectors["scale"], want=BOTH, dX=block.dx, out=block.vec_S, workspace=ws)
    # 3. sums over the batch of the matrices' gradients
    pex.pex_stat(h, G1.view(B, T, hidden), "identity", S=block.S[0], workspace=ws)
    pex.pex_stat(r.view(B, T, hidden), G2, "identity", S=block.S[1], workspace=ws)
    # 4. updates
    pex.pex_muon_step(list(zip(block.W, block.W_m, block.S)), pex.MuonParams(lr=lr, grad_scale=1.0 / B), workspace=ws)
    prm = pex.AdamParams(lr=vector_lr, beta1=0.9, beta2=0.95, eps=1e-8, eps_root=0.0, weight_decay=0.0, grad_scale=1.0 / B, sq_scale=1.0 / B, step=step, B=B)
    pex.pex_adam_step([(block.vectors[k], block.vec_m[k], block.vec_v[k], block.vec_S[k]["identity"], block.vec_S[k]["square"]) for k in block.vectors],
                      "microadam", prm, block.sum_sq, 1.0, workspace=ws)
    return (error * error).mean()


def teacher(block, x, seed=1):
    """Targets: what a block of other weights makes of x."""
    B, T, d, hidden = block.shape
    g = torch.Generator(device=x.device).manual_seed(seed)
    W1, W2 = (torch.randn(a, b, device=x.device, generator=g) * a ** -0.5 for a, b in ((d, hidden), (hidden, d)))
    h = pex.pex_layer_norm(x)[0].view(B * T, d)
    return x + (torch.nn.functional.silu(h @ W1.bfloat16()) @ W2.bfloat16()).view(B, T, d)


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--B", type=int, default=16)
    ap.add_argument("--T", type=int, default=1024)
    ap.add_argument("--d", type=int, default=768)
    ap.add_argument("--steps", type=int, default=40)
    a = ap.parse_args()
    dev = torch.device("cuda:0")
    block = Block(a.B, a.T, a.d, 4 * a.d, dev)
    x = torch.randn(a.B, a.T, a.d, device=dev, generator=torch.Generator(device=dev).manual_seed(2)).bfloat16()
    target = teacher(block, x)
    first = float(train_step(block, x, target, 1))
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    for s in range(2, a.steps + 1):
        last = train_step(block, x, target, s)
    torch.cuda.synchronize()
    ms = (time.perf_counter() - t0) / max(1, a.steps - 1) * 1e3
    print(f"pre-norm MLP block d={a.d} hidden={4 * a.d} B={a.B} T={a.T}: {ms:.3f} ms a step; mean squared error {first:.4f} -> {float(last):.4f} in {a.steps} steps")


if __name__ == "__main__":
    main()
