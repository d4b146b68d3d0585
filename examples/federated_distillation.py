"""One federated round of an output head with distillation.

    python examples/federated_distillation.py

Two federation groups train the head (V words, D wide) of a small model.  Each
local step, the R ranks of a group take a private batch with labels and a
public batch of which a teacher's top logits are known (fl_top_logits), and
contribute two bf16 gradients each: of the cross entropy (fl_head_loss,
fl_head_loss_grad) and of the divergence from the teacher (fl_head_distill,
fl_head_distill_grad).  The contributions are summed and AdamW is applied
(fl_local_step); after A steps the groups' heads are averaged (fl_fedavg).
Ranks, groups and the hidden states under the head are stand-ins: buffers on
one GPU and random features.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2609_20359_amd as P  # noqa: E402

V, D, T, K, TAU = 4000, 256, 512, 16, 2.0
G, R, A = 2, 2, 30
ALPHA = 0.5                       # share of the distillation in the loss
HP = dict(lr=3e-3, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.0)


class Batch:
    """Hidden states, labels drawn by the teacher, and its top logits."""

    def __init__(self, teacher, gen, prompt):
        self.hidden = torch.randn(T, D, generator=gen, device="cuda").bfloat16()
        logits = self.hidden.float() @ teacher.t()
        u = torch.rand(logits.shape, generator=gen, device="cuda").clamp_(1e-9, 1 - 1e-6)
        self.labels = (logits - torch.log(-torch.log(u))).argmax(1)
        self.labels[:prompt] = -100                       # tokens without a loss
        self.values = torch.empty(T, K, device="cuda")
        self.ids = torch.empty(T, K, dtype=torch.int32, device="cuda")
        self.lse = torch.empty(T, device="cuda")
        P.fl_top_logits(logits, K, TAU, self.values, self.ids, self.lse)


class Student:
    """A group's head: fp32 master with AdamW's moments, bf16 working copy."""

    def __init__(self, layout, weight):
        self.layout = layout
        self.master = weight.reshape(-1).float().clone()
        self.m, self.v = torch.zeros_like(self.master), torch.zeros_like(self.master)
        self.working = self.master.bfloat16()
        self.grads = [torch.empty(V * D, dtype=torch.bfloat16, device="cuda") for _ in range(2 * R)]
        self.loss, self.lse = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
        self.target, self.targets = torch.empty(T, device="cuda"), torch.empty(T, K, device="cuda")
        self.dhidden = torch.empty(T, D, dtype=torch.bfloat16, device="cuda")
        self.work = torch.empty(max(P.head_workspace_bytes(T, V, D, k, grad=g)
                                    for k in (0, K) for g in (False, True)),
                                dtype=torch.uint8, device="cuda")

    def contribute(self, b, r):
        """Rank r's two gradients on batch b; its loss and divergence, on the GPU."""
        w = self.working.view(V, D)
        live = (b.labels >= 0).sum()
        P.fl_head_loss(b.hidden, w, b.labels, self.loss, self.lse, self.target, workspace=self.work)
        ce = self.loss.sum() / live
        dloss = ((1 - ALPHA) / live).float().expand(T).contiguous()
        P.fl_head_loss_grad(b.hidden, w, b.labels, self.lse, self.target, dloss, self.dhidden,
                            self.grads[2 * r].view(V, D), workspace=self.work)
        P.fl_head_distill(b.hidden, w, b.ids, b.values, b.lse, TAU, self.loss, self.lse,
                          self.targets, workspace=self.work)
        kd = self.loss.mean()
        dloss = torch.full((T,), ALPHA / T, device="cuda")
        P.fl_head_distill_grad(b.hidden, w, b.ids, b.values, b.lse, TAU, self.lse, self.targets,
                               dloss, self.dhidden, self.grads[2 * r + 1].view(V, D),
                               workspace=self.work)
        return ce, kd

    def step(self, batches, number):
        said = [self.contribute(b, r) for r, b in enumerate(batches)]
        P.fl_local_step(self.layout, HP, number, self.grads, 1.0 / R, self.master, self.m, self.v,
                        self.working)
        return torch.stack([torch.stack(x) for x in said]).mean(0)


def run():
    """The round; per group the loss and the divergence of its first and last
    step, and the heads after averaging."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    teacher = torch.randn(V, D, generator=gen, device="cuda") * (3.0 / D ** 0.5)
    start = torch.randn(V, D, generator=gen, device="cuda") * (0.1 / D ** 0.5)
    layout = P.Layout([0, V * D])
    groups = [Student(layout, start) for _ in range(G)]
    data = [[Batch(teacher, gen, prompt=64 * r) for r in range(R)] for _ in range(G)]
    said = []
    for number in range(1, A + 1):
        said.append(torch.stack([s.step(b, number) for s, b in zip(groups, data)]))
    replicas = [s.working.clone() for s in groups]
    for s in groups:
        P.fl_fedavg(layout, replicas, [1.0] * G, s.master, s.working)
    torch.cuda.synchronize()
    out = dict(first=said[0].tolist(), last=said[-1].tolist(),
               heads=[s.working.clone() for s in groups])
    layout.close()
    return out


if __name__ == "__main__":
    r = run()
    for g in range(G):
        print("group %d: cross entropy %.3f -> %.3f, divergence from the teacher %.3f -> %.3f"
              % (g, r["first"][g][0], r["last"][g][0], r["first"][g][1], r["last"][g][1]))
    print("groups equal after averaging: %s" % torch.equal(r["heads"][0], r["heads"][1]))
