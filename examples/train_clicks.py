"""A click model trained on what extraction leaves in device memory, batch after batch: records -> signs (`Plan.extract`) ->
rows of a table, pooled per slot (`train.embed`) -> a gated block (`train.gated`) -> one logit -> logistic loss, and back;
the table and the weights take an AdamW step (`train.AdamW`), the table's states in 8 bits.

    python examples/train_clicks.py [--records 8192] [--steps 60] [--dim 16] [--hidden 512] [--rows 1000003]

Records are synthetic (the repository's smallest workload: 16 fields and 8 crosses); a record's click is drawn from a rule
on two of its fields, which the model has to find.
"""
import argparse
import math
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2210_07768_amd import binding, train, workloads  # noqa: E402


class Model:
    """Weights in 32 bits, which the optimizer steps, and the 16-bit copies that the kernels read."""

    def __init__(self, slots, rows, dim, hidden, lr, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        width = slots * dim
        r = lambda *s, scale: torch.randn(*s, device="cuda", generator=g) * scale  # noqa: E731
        self.master = [r(rows, dim, scale=0.05), r(hidden, width, scale=1 / math.sqrt(width)), r(hidden, width, scale=1 / math.sqrt(width))]
        self.table, self.w_gate, self.w_up = [w.to(torch.bfloat16).requires_grad_() for w in self.master]
        self.out = r(hidden, scale=1 / math.sqrt(hidden)).requires_grad_()
        rest = dict(lr=lr, weight_decay=0.01)
        self.optimizers = [(train.AdamW(self.master[:1], bits=8, copies=[self.table], seed=seed, **rest), [self.table]),
                           (train.AdamW(self.master[1:], copies=[self.w_gate, self.w_up], **rest), [self.w_gate, self.w_up]),
                           (train.AdamW([self.out], **rest), [self.out])]

    def logits(self, result):
        pooled = train.embed(result, self.table)                       # records x slots x dim
        return train.gated(pooled.flatten(1), self.w_gate, self.w_up).float() @ self.out

    def step(self, result, clicks):
        loss = torch.nn.functional.binary_cross_entropy_with_logits(self.logits(result), clicks)
        loss.backward()
        for optimizer, weights in self.optimizers:
            optimizer.step([w.grad for w in weights])
            for w in weights:
                w.grad = None
        return loss.detach()


def clicks_of(result, seed):
    """Drawn with a probability that a bit of the first field's sign and one of the second's decide."""
    a, b = (result.slots[s].values for s in result.slot_ids[:2])
    agree = ((a >> 17) ^ (b >> 23)) & 1
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.rand(a.shape[0], device="cuda", generator=g) < torch.where(agree == 1, 0.8, 0.1)).float()


def run(records=8192, steps=60, dim=16, hidden=512, rows=1_000_003, lr=2e-3, tell=print):
    """Trains on `steps` batches and returns the losses."""
    workload = workloads.config1(records)
    plan = binding.Plan(workload.spec)
    batches = []
    for k in range(8):
        raw, off = workload.generate(k * records, records)
        batches.append((torch.from_numpy(raw.copy()).cuda(), torch.from_numpy(off.astype(np.int64)).cuda()))
    model, losses, keep = None, [], None
    for step in range(steps):
        raw, off = batches[step % len(batches)]
        if keep is None:
            result, keep = binding.extract_with_retry(plan, raw, off)  # (the workspace, in which results lie)
        else:
            result = plan.extract(raw, off)
        if model is None:
            model = Model(len(result.slot_ids), rows, dim, hidden, lr)
        losses.append(model.step(result, clicks_of(result, step % len(batches))))
        if step % 10 == 0 or step == steps - 1:
            tell(f"step {step}: loss {float(losses[-1]):.4f}")
    plan.close()
    return [float(x) for x in losses]


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("records", 8192), ("steps", 60), ("dim", 16), ("hidden", 512), ("rows", 1_000_003)):
        ap.add_argument("--" + name, type=int, default=value)
    run(**vars(ap.parse_args()))
