"""Algorithm 1 with the threshold of Algorithm 2: a small language model trained with dropped micro-batches.

    python -m paper_2306_10598_b200.drop_train --noise lognormal_0.05 --workers 8 --steps 40

A calibration sweep (api.sweep on simulated latencies of one of App. C.3's noise laws) gives tau*.  Then, step by step, every
worker's micro-batches run until the first one whose finish time is not below tau*; the gradients of those that ran are
accumulated in fp32 and divided by the number of labelled tokens that were really computed (the correction for a
stochastic batch size that divides by the computed batch).  The workers are taken one after the other on one GPU, so their
compute times are the simulated ones; the micro-batches are real.  The model predicts the next token from the current one:

    x = sqrt(D) table[ids]        api.embed            y = gelu(x), x kept in 8 bits      api.gelu_save8
    loss = cross entropy of y head^T over the vocabulary, where there is a label          api.vocab_loss

and the backward passes of the three."""
from __future__ import annotations

import argparse
import json
import math
from typing import Dict, List

import torch

from . import api
from . import workloads as W

PAD, NO_LABEL = 0, -100


def run_until(latencies: torch.Tensor, tau: float) -> torch.Tensor:
    """[N] number of micro-batches of each worker that finish before tau: latencies [N, M], strictly left to right in fp32."""
    p = torch.zeros_like(latencies[:, 0])
    ran = torch.zeros(latencies.shape[0], dtype=torch.int64, device=latencies.device)
    for m in range(latencies.shape[1]):
        p = p + latencies[:, m]
        ran += p < tau
    return ran


def micro_batch(table: torch.Tensor, head: torch.Tensor, ids: torch.Tensor, targets: torch.Tensor, dtable: torch.Tensor,
                dhead: torch.Tensor) -> torch.Tensor:
    """One micro-batch: its gradients (of the sum of its tokens' losses) are added to dtable and dhead, fp32.  Returns the
    tokens' losses."""
    scale = math.sqrt(table.shape[1])
    y, q, scales = api.gelu_save8(api.embed(table, ids, scale, PAD))
    loss, lse = api.vocab_loss(y, head, targets, NO_LABEL)
    dy, _ = api.vocab_loss_backward(y, head, targets, lse, torch.ones_like(loss), NO_LABEL, dweight=dhead, accumulate=True)
    dx = api.gelu_save8_backward(dy, q, scales)
    api.embed_backward(dx, ids, table.shape[0], scale, PAD, dtable=dtable, accumulate=True)
    return loss


class Text:
    """Sequences in which a fixed token follows each token most of the time; their ends are padding, and some places carry no
    label."""

    def __init__(self, vocab: int, seed: int, device):
        self.g = torch.Generator(device=device).manual_seed(seed)
        self.vocab, self.device = vocab, device
        self.follows = torch.randperm(vocab - 1, generator=self.g, device=device) + 1

    def batch(self, sequences: int, length: int):
        rand = lambda *s: torch.rand(*s, generator=self.g, device=self.device)   # noqa: E731
        ids = (rand(sequences, length + 1) * (self.vocab - 1)).long() + 1
        sure = rand(sequences, length) < 0.9
        for i in range(length):
            ids[:, i + 1] = torch.where(sure[:, i], self.follows[ids[:, i] - 1], ids[:, i + 1])
        ends = (length * (0.5 + 0.5 * rand(sequences, 1))).long()
        beyond = torch.arange(length, device=self.device) >= ends
        targets = torch.where(beyond | (rand(sequences, length) < 0.3), NO_LABEL, ids[:, 1:])
        return torch.where(beyond, PAD, ids[:, :-1]).contiguous(), targets.contiguous()


def train(noise: str = "lognormal_0.05", workers: int = 8, steps: int = 40, vocab: int = 1009, width: int = 128, sequences: int = 4,
          length: int = 32, lr: float = 0.02, t_comm: float = 0.5, calibration: int = 512, seed: int = 0, device="cuda") -> List[Dict]:
    w = W.c3_workload(noise, N=workers, T=calibration, t_comm=t_comm, seed=seed)
    r = api.sweep(W.fill_latencies(w, device), torch.from_numpy(W.make_taus(w)).to(device), t_comm)
    tau = float(r.tau_star)
    run = W.c3_workload(noise, N=workers, T=steps, t_comm=t_comm, seed=seed + 1)
    latencies = W.fill_latencies(run, device)

    g = torch.Generator(device=device).manual_seed(seed)
    masters = [torch.randn(vocab, width, generator=g, device=device) / math.sqrt(width) for _ in range(2)]
    grads = [torch.zeros_like(p) for p in masters]
    moments = [(torch.zeros_like(p), torch.zeros_like(p)) for p in masters]
    text = Text(vocab, seed, device)
    log = []
    for step in range(steps):
        table, head = (p.bfloat16() for p in masters)
        for d in grads:
            d.zero_()
        ran = run_until(latencies[step], tau).tolist()
        losses, labelled = torch.zeros((), device=device), torch.zeros((), dtype=torch.int64, device=device)
        for n in range(workers):
            for _ in range(ran[n]):
                ids, targets = text.batch(sequences, length)
                losses += micro_batch(table, head, ids, targets, *grads).sum()
                labelled += (targets != NO_LABEL).sum()
        for p, d, (m, v) in zip(masters, grads, moments):
            d /= labelled.clamp(min=1)                                # by what was computed, not by what was planned
            m.lerp_(d, 0.1)
            v.lerp_(d * d, 0.01)
            p -= lr * (m / (1 - 0.9 ** (step + 1))) / ((v / (1 - 0.99 ** (step + 1))).sqrt() + 1e-8)
        slowest = float(latencies[step].double().sum(-1).max())
        log.append({"step": step, "loss": float(losses) / max(1, int(labelled)), "micro_batches": sum(ran), "planned": workers * run.M,
                    "step_time": min(tau, slowest) + t_comm, "without_drop": slowest + t_comm, "tau": tau})
    api.dc_train_status()
    return log


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--noise", default="lognormal_0.05", choices=sorted(W.C3_NOISE))
    ap.add_argument("--workers", type=int, default=8)
    ap.add_argument("--steps", type=int, default=40)
    ap.add_argument("--vocab", type=int, default=1009)
    ap.add_argument("--width", type=int, default=128)
    args = ap.parse_args()
    log = train(args.noise, args.workers, args.steps, args.vocab, args.width)
    for row in log[:: max(1, len(log) // 10)]:
        print(json.dumps({k: round(v, 4) if isinstance(v, float) else v for k, v in row.items()}))
    took, sync = sum(r["step_time"] for r in log), sum(r["without_drop"] for r in log)
    share = sum(r["micro_batches"] for r in log) / sum(r["planned"] for r in log)
    print(json.dumps({"tau": log[0]["tau"], "first_loss": log[0]["loss"], "last_loss": log[-1]["loss"], "share_run": share,
                      "time": took, "time_without_drop": sync, "micro_batches_per_second_gain": share * sync / took}))


if __name__ == "__main__":
    main()
