"""Tunes the factors of a ladder on tokens: an adapted projection in front of a frozen head over a large vocabulary.

Where distilling (``distill_ladder``) brings a ladder's prefixes close to the full adapter, this tunes all of them, under a
chunk table that mixes their ranks, on what the text says next.  Logits are never stored.

    step      cwl_apply under the table -> cwl_head_loss: loss, and the gradient of the head's input
              -> cwl_apply_grads: dA, dB -> cwl_factor_step: orthogonalised momentum on fp32 masters, bf16 factors

    python -m paper_2601_21109_b200.tune_ladder [--steps N] [--tokens T] [--width D] [--vocab V] [--prompt P]
"""
from __future__ import annotations

import argparse
from typing import Optional

import numpy as np
import torch

from . import binding as cwl


class LadderTuner:
    """Device-resident state of the tuning: frozen X, W and head, targets (negative: none), factors, masters and momenta."""

    def __init__(self, X: torch.Tensor, W: torch.Tensor, head: torch.Tensor, A: torch.Tensor, B: torch.Tensor, targets: torch.Tensor,
                 table: cwl.DeviceChunkTable, window: int, lr: float = 0.02, momentum: float = 0.95, weight_decay: float = 0.0,
                 weight: Optional[torch.Tensor] = None):
        T, d_in, width, V, R = X.shape[0], X.shape[1], W.shape[1], head.shape[1], A.shape[1]
        dev = X.device
        self.X, self.W, self.head, self.targets, self.table, self.window = X, W, head, targets, table, int(window)
        self.lr, self.momentum, self.weight_decay = float(lr), float(momentum), float(weight_decay)
        self.status = torch.zeros(1, dtype=torch.int32, device=dev)
        self.apply_ws = torch.empty(cwl.cwl_apply_workspace_bytes(T, d_in, width, R), dtype=torch.uint8, device=dev)
        self.head_ws = torch.empty(cwl.cwl_head_loss_workspace_bytes(T, width, V, True), dtype=torch.uint8, device=dev)
        self.grads_ws = torch.empty(cwl.cwl_apply_grads_workspace_bytes(T, d_in, width, R), dtype=torch.uint8, device=dev)
        self.A, self.B = A.clone(), B.clone()
        self.master = [A.float(), B.float()]
        self.moments = [torch.zeros_like(m) for m in self.master]
        self.dA, self.dB = torch.empty_like(self.master[0]), torch.empty_like(self.master[1])
        self.weight = weight if weight is not None else (targets >= 0).float() / (targets >= 0).sum().clamp(min=1)
        self.hidden = torch.empty(T, width, dtype=torch.bfloat16, device=dev)
        self.d_hidden = torch.empty_like(self.hidden)
        self.loss, self.lse = (torch.empty(T, dtype=torch.float32, device=dev) for _ in range(2))
        self.update = cwl.FactorStep(self.master, [self.A, self.B], [self.dA, self.dB], self.moments)

    def forward(self) -> torch.Tensor:
        """The head's input under the chunk table."""
        return cwl.cwl_apply(self.X, self.W, self.A, self.B, self.table, self.window, Y=self.hidden, workspace=self.apply_ws,
                             status_word=self.status)

    def evaluate(self) -> torch.Tensor:
        """Loss of every token (times its weight), without gradients."""
        cwl.cwl_head_loss(self.forward(), self.head, self.targets, weight=self.weight, loss=self.loss, lse=self.lse,
                          workspace=self.head_ws, status_word=self.status)
        return self.loss

    def gradients(self) -> None:
        """Loss of every token, and the gradients of its sum with respect to the factors."""
        cwl.cwl_head_loss(self.forward(), self.head, self.targets, weight=self.weight, loss=self.loss, lse=self.lse, dX=self.d_hidden,
                          workspace=self.head_ws, status_word=self.status)
        cwl.cwl_apply_grads(self.X, self.d_hidden, self.A, self.B, self.table, self.window, dA=self.dA, dB=self.dB,
                            workspace=self.grads_ws, status_word=self.status)

    def step(self) -> None:
        """One training step on the current stream; no host synchronisation."""
        self.gradients()
        self.update = self.update.of(self.master, [self.A, self.B], [self.dA, self.dB], self.moments)
        self.update(self.lr, self.momentum, self.weight_decay)

    def capture(self) -> "torch.cuda.CUDAGraph":
        """Records one step into a CUDA graph, after an ordinary one that sets kernels up."""
        self.step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            self.step()
        return graph


def synthetic(T: int, d: int, V: int, R: int = 64, prompt: float = 0.25, seed: int = 0, **kw) -> LadderTuner:
    """A projection and a head of synthetic weights, tokens that a hidden adapter of the same rank finds likely, a ladder that
    starts near zero, and a chunk table that runs the tokens at 1/8, 1/4, 1/2 and all of its rank.  The first `prompt` share
    of the tokens has no targets."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(r, c, std):
        return (torch.randn(r, c, device="cuda", generator=gen) * std).bfloat16()
    X, W, head = normal(T, d, 1.0), normal(d, d, d ** -0.5), normal(d, V, 3.0 * d ** -0.5)
    hidden = cwl.cwl_apply(X, W, normal(d, R, d ** -0.5), normal(R, d, R ** -0.5),
                           cwl.DeviceChunkTable.from_host([0, T], [R], [1.0], [1]), 0)
    targets = cwl.cwl_token_logprobs(cwl.cwl_apply(hidden, head, None, None, None, 0), top_k=1).top_ids[:, 0].contiguous()
    targets[:int(prompt * T)] = -1
    rng = np.random.default_rng(seed)
    cuts = list(range(0, T, 64))
    ranks = np.array([max(1, R // 8), max(1, R // 4), R // 2, R], np.int32)[rng.integers(0, 4, len(cuts))]
    table = cwl.DeviceChunkTable.from_host(cuts + [T], ranks, np.ones(len(cuts), np.float32), [1] + [0] * (len(cuts) - 1))
    return LadderTuner(X, W, head, normal(d, R, d ** -0.5), normal(R, d, 1e-3), targets, table, window=8, **kw)


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=100)
    ap.add_argument("--tokens", type=int, default=2048)
    ap.add_argument("--width", type=int, default=4096)
    ap.add_argument("--vocab", type=int, default=32000)
    ap.add_argument("--prompt", type=float, default=0.25, help="share of the tokens that have no targets")
    a = ap.parse_args()
    t = synthetic(a.tokens, a.width, a.vocab, prompt=a.prompt)
    print(f"before: loss {float(t.evaluate().sum()):.4f}")
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    t.step()
    start.record()
    for _ in range(a.steps - 1):
        t.step()
    end.record()
    torch.cuda.synchronize()
    assert int(t.status.item()) == 0, "device status word set"
    if a.steps > 1:
        print(f"{a.steps} steps of {a.tokens} tokens, {start.elapsed_time(end) / (a.steps - 1):.3f} ms each")
    print(f"after:  loss {float(t.evaluate().sum()):.4f}")


if __name__ == "__main__":
    main()
