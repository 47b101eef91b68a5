"""Distils the full adapter of a ladder into its prefixes: the training step that the library's calls make up.

A ladder is only useful if its prefixes are (Sec. III-C picks them per chunk), and a singular value decomposition makes
them good in the norm of the weights, not in what the model answers.  Here the projection in front of the vocabulary is
the student: the full adapter's answers (the teacher) are recorded once, as the top log-probabilities of every token, and
the factors are then trained under a chunk table that mixes the ladder's ranks.

    teacher   cwl_apply at full rank -> cwl_token_logprobs: top K of the tempered teacher
    step      cwl_apply under the table -> cwl_distill_topk: loss, and its gradient in the place of the logits
              -> cwl_apply_grads: dA, dB -> Adam on fp32 copies of the factors (a few torch calls)

    python -m paper_2601_21109_b200.distill_ladder [--steps N] [--tokens T] [--width D] [--vocab V]
"""
from __future__ import annotations

import argparse
from typing import Optional

import numpy as np
import torch

from . import binding as cwl


class LadderDistiller:
    """Device-resident state of the training: frozen X and W, the teacher's record, factors and their Adam moments."""

    def __init__(self, X: torch.Tensor, W: torch.Tensor, A: torch.Tensor, B: torch.Tensor, teacher_table: cwl.DeviceChunkTable,
                 table: cwl.DeviceChunkTable, window: int, top_k: int = 64, temperature: float = 1.0, lr: float = 1e-3,
                 weight: Optional[torch.Tensor] = None):
        T, d_in, d_out, R = X.shape[0], X.shape[1], W.shape[1], A.shape[1]
        self.X, self.W, self.table, self.window, self.temperature, self.lr = X, W, table, int(window), float(temperature), float(lr)
        self.status = torch.zeros(1, dtype=torch.int32, device=X.device)
        self.apply_ws = torch.empty(cwl.cwl_apply_workspace_bytes(T, d_in, d_out, R), dtype=torch.uint8, device=X.device)
        self.grads_ws = torch.empty(cwl.cwl_apply_grads_workspace_bytes(T, d_in, d_out, R), dtype=torch.uint8, device=X.device)
        self.logits = torch.empty(T, d_out, dtype=torch.bfloat16, device=X.device)
        cwl.cwl_apply(X, W, A, B, teacher_table, 0, Y=self.logits, workspace=self.apply_ws, status_word=self.status)
        self.teacher = cwl.cwl_token_logprobs(self.logits, top_k=top_k, temperature=self.temperature, status_word=self.status)
        self.A, self.B = A.clone(), B.clone()
        self.master = [A.float(), B.float()]
        self.moments = [(torch.zeros_like(m), torch.zeros_like(m)) for m in self.master]
        self.weight = weight if weight is not None else torch.full((T,), 1.0 / T, device=X.device)
        self.loss = torch.empty(T, dtype=torch.float32, device=X.device)
        self.dA, self.dB = torch.empty_like(self.master[0]), torch.empty_like(self.master[1])
        self.steps = 0

    def forward(self) -> torch.Tensor:
        """The student's logits under the chunk table."""
        return cwl.cwl_apply(self.X, self.W, self.A, self.B, self.table, self.window, Y=self.logits, workspace=self.apply_ws,
                             status_word=self.status)

    def gradients(self) -> None:
        """Loss of every token, and the gradients of its sum with respect to the factors."""
        self.forward()
        cwl.cwl_distill_topk(self.logits, self.teacher.top_ids, self.teacher.top_logprobs, teacher="logprobs",
                             temperature=self.temperature, weight=self.weight, loss=self.loss, dlogits=self.logits,
                             status_word=self.status)
        cwl.cwl_apply_grads(self.X, self.logits, self.A, self.B, self.table, self.window, dA=self.dA, dB=self.dB,
                            workspace=self.grads_ws, status_word=self.status)

    def step(self) -> None:
        """One training step on the current stream; no host synchronisation."""
        self.gradients()
        self.steps += 1
        b1, b2 = 0.9, 0.999
        scale = self.lr * (1 - b2 ** self.steps) ** 0.5 / (1 - b1 ** self.steps)
        for p, (m, v), g, low in zip(self.master, self.moments, (self.dA, self.dB), (self.A, self.B)):
            m.lerp_(g, 1 - b1)
            v.mul_(b2).addcmul_(g, g, value=1 - b2)
            p.addcdiv_(m, v.sqrt().add_(1e-8), value=-scale)
            low.copy_(p)

    def agreement(self) -> float:
        """Share of the tokens whose most likely continuation is the teacher's."""
        top = cwl.cwl_token_logprobs(self.forward(), top_k=1).top_ids
        return float((top[:, 0] == self.teacher.top_ids[:, 0]).float().mean())


def synthetic(T: int, d: int, V: int, R: int = 64, seed: int = 0, **kw) -> LadderDistiller:
    """A projection of synthetic weights whose trained adapter matters (and whose 64 likeliest tokens carry most of the
    mass), its ladder by singular values, and a chunk table that runs the tokens at 1/8, 1/4, 1/2 and all of its rank."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(r, c, std):
        return (torch.randn(r, c, device="cuda", generator=gen) * std).bfloat16()
    X, W = normal(T, d, 1.0), normal(d, V, 3.0 * d ** -0.5)
    ladder = cwl.cwl_ladder_build(normal(d, R, 3.0 * d ** -0.5), normal(R, V, R ** -0.5), want_f32=False)
    rng = np.random.default_rng(seed)
    cuts = list(range(0, T, 64))
    ranks = np.array([max(1, R // 8), max(1, R // 4), R // 2, R], np.int32)[rng.integers(0, 4, len(cuts))]
    table = cwl.DeviceChunkTable.from_host(cuts + [T], ranks, np.ones(len(cuts), np.float32), [1] + [0] * (len(cuts) - 1))
    full = cwl.DeviceChunkTable.from_host([0, T], [R], [1.0], [1])
    return LadderDistiller(X, W, ladder["A"], ladder["B"], full, table, window=8, **kw)


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=100)
    ap.add_argument("--tokens", type=int, default=2048)
    ap.add_argument("--width", type=int, default=4096)
    ap.add_argument("--vocab", type=int, default=32000)
    a = ap.parse_args()
    d = synthetic(a.tokens, a.width, a.vocab)
    d.gradients()
    print(f"before: loss {float(d.loss.sum()):.4f}, top-1 agreement {d.agreement():.3f}")
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    d.step()
    start.record()
    for _ in range(a.steps - 1):
        d.step()
    end.record()
    torch.cuda.synchronize()
    assert int(d.status.item()) == 0, "device status word set"
    if a.steps > 1:
        print(f"{a.steps} steps of {a.tokens} tokens, {start.elapsed_time(end) / (a.steps - 1):.3f} ms each")
    d.gradients()
    print(f"after:  loss {float(d.loss.sum()):.4f}, top-1 agreement {d.agreement():.3f}")


if __name__ == "__main__":
    main()
