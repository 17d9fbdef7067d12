"""Preference tuning by local steps and synchronisation rounds, on one GPU.

Each of K workers holds a two-layer scorer of token features (hidden features, then
logits over the vocabulary) and its own pairs of chosen and rejected sequences.  A local
step runs in the library from end to end: both linear layers with 4-bit operands, the
preference loss and its gradient by the logits, the layers' gradients with 4-bit
operands, clipping and packing over the gradient tensors of all workers, AdamW.  After
every interval the corrected outer step averages the workers and resets them.

    python -m workloads.preference_step [--workers 4 --rounds 4 --steps 5 ...]
"""
from __future__ import annotations

import argparse
from dataclasses import dataclass
from typing import List

import torch

import paper_2609_36662_amd as al


@dataclass(frozen=True)
class Shape:
    features: int = 256
    hidden: int = 320
    vocab: int = 1009
    pairs: int = 6
    longest: int = 40


class Worker:
    """One worker's data, its layers' 4-bit forms and the buffers of a step.  theta is its flat fp32 parameters."""

    def __init__(self, ctx, shape: Shape, theta: torch.Tensor, seed: int):
        self.ctx, self.shape = ctx, shape
        s, bf, dev = shape, torch.bfloat16, "cuda"
        g = torch.Generator().manual_seed(seed)
        lens = torch.randint(s.longest // 3, s.longest + 1, (2 * s.pairs,), generator=g)
        rows = int(lens.sum())
        self.offsets = torch.cat([torch.zeros(1, dtype=torch.int64), lens.cumsum(0)]).to(dev)
        self.x = torch.randn((rows, s.features), generator=g).to(dev, bf)
        labels = torch.randint(0, s.vocab, (rows,), generator=g)
        labels[torch.rand(rows, generator=g) < 0.25] = -100        # the prompts
        self.labels = labels.to(dev)
        sizes = [s.hidden * s.features, s.vocab * s.hidden]
        self.w = [t.view(o, -1) for t, o in zip(theta.split(sizes), (s.hidden, s.vocab))]
        empty = al.Mxfp4.empty
        self.wq = [empty(*w.shape) for w in self.w]
        self.wt = empty(s.hidden, s.vocab)                          # the head's transpose, for the gradient by its input
        self.xq, self.hq = empty(rows, s.features), empty(rows, s.hidden)
        self.xt, self.ht, self.dht = empty(s.features, rows), empty(s.hidden, rows), empty(s.hidden, rows)
        self.dq, self.dt = empty(rows, s.vocab), empty(s.vocab, rows)
        self.h, self.dh = (torch.empty((rows, s.hidden), dtype=bf, device=dev) for _ in range(2))
        self.logits = torch.empty((rows, s.vocab), dtype=bf, device=dev)
        self.logps, self.ref = torch.empty(2 * s.pairs, device=dev), torch.empty(2 * s.pairs, device=dev)
        self.losses, self.work = torch.empty(s.pairs, device=dev), torch.empty(2 * rows + 2 * s.pairs, device=dev)
        self.grads = [torch.empty_like(w) for w in self.w]
        al.autoloco_mxfp4_quantize(ctx, self.x, None, self.xt)      # the data's transpose does not change
        self.forward()
        al.autoloco_sequence_logps(ctx, self.logits, self.labels, self.offsets, self.ref, self.work)   # the frozen reference

    def forward(self) -> None:
        al.autoloco_mxfp4_quantize(self.ctx, self.w[0], self.wq[0])
        al.autoloco_mxfp4_quantize(self.ctx, self.w[1], self.wq[1], self.wt)
        al.autoloco_mxfp4_linear(self.ctx, self.x, self.wq[0], self.h, self.xq)
        self.h.relu_()
        al.autoloco_mxfp4_linear(self.ctx, self.h, self.wq[1], self.logits, self.hq)

    def gradients(self, beta: float) -> None:
        """The losses, and the mean loss's gradient by both layers."""
        self.forward()
        al.autoloco_preference_loss(self.ctx, self.logits, self.labels, self.offsets, self.ref, self.losses, self.logps,
                                    self.work, grads=self.logits, beta=beta, grad_scale=1.0 / self.shape.pairs)
        al.autoloco_mxfp4_quantize(self.ctx, self.logits, self.dq, self.dt)     # now the gradient by the logits
        al.autoloco_mxfp4_quantize(self.ctx, self.h, None, self.ht)
        al.autoloco_mxfp4_matmul(self.ctx, self.dt, self.ht, self.grads[1])
        al.autoloco_mxfp4_matmul(self.ctx, self.dq, self.wt, self.dh)
        self.dh.mul_(self.h > 0)
        al.autoloco_mxfp4_quantize(self.ctx, self.dh, None, self.dht)
        al.autoloco_mxfp4_matmul(self.ctx, self.dht, self.xt, self.grads[0])


def run(workers: int = 4, rounds: int = 4, steps: int = 5, shape: Shape = Shape(), lr: float = 2e-3, beta: float = 0.1,
        max_norm: float = 1.0, seed: int = 0) -> List[dict]:
    """Rounds of local steps; per round the mean losses of its first and last step, the largest gradient norm and the
    round's statistics."""
    n = shape.hidden * shape.features + shape.vocab * shape.hidden
    g = torch.Generator().manual_seed(seed)
    theta = torch.cat([torch.randn(shape.hidden * shape.features, generator=g) / shape.features ** 0.5,
                       torch.randn(shape.vocab * shape.hidden, generator=g) / shape.hidden ** 0.5]).cuda()
    momentum = torch.zeros_like(theta)
    params = [theta.clone() for _ in range(workers)]
    first, second, packed = ([torch.zeros_like(theta) for _ in range(workers)] for _ in range(3))
    sched = al.make_schedule(peak=lr, warmup=0, total=4 * rounds * steps)
    history, step = [], 0
    with al.autoloco_create(0) as ctx:
        team = [Worker(ctx, shape, p, seed + 1 + k) for k, p in enumerate(params)]
        grads = al.autoloco_grads_create(ctx, [w.grads for w in team], packed)
        for _ in range(rounds):
            start, losses, norm = step, [], 0.0
            for _ in range(steps):
                for w in team:
                    w.gradients(beta)
                clip = al.autoloco_clip_grad_norm(ctx, grads, max_norm)
                norm = max(norm, *clip.grad_norm[:workers])
                losses.append(torch.stack([w.losses.mean() for w in team]).mean())
                coeffs = al.make_adamw_coeffs(al.autoloco_inner_lr(sched, step), step + 1, weight_decay=0.0, max_grad_norm=0.0)
                al.autoloco_inner_adamw(ctx, params, first, second, packed, coeffs, stats=False)
                step += 1
            mass = al.autoloco_lr_mass(sched, start, steps)
            stats = al.autoloco_outer_step(ctx, theta, momentum, params, al.autoloco_outer_correction(al.make_outer_cfg(), mass, mass))
            history.append({"first_loss": float(losses[0]), "last_loss": float(losses[-1]), "grad_norm": norm, "D": stats.D,
                            "C": stats.C, "finite": bool(stats.finite)})
        torch.cuda.synchronize()
        grads.close()
    assert theta.numel() == n
    return history


def main() -> None:
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("workers", 4), ("rounds", 4), ("steps", 5), ("seed", 0)):
        p.add_argument(f"--{name}", type=int, default=value)
    for i, r in enumerate(run(**vars(p.parse_args()))):
        print(f"round {i}: loss {r['first_loss']:.4f} -> {r['last_loss']:.4f}, gradient norm up to {r['grad_norm']:.3f}, "
              f"D {r['D']:.4g}, C {r['C']:.4g}")


if __name__ == "__main__":
    main()
