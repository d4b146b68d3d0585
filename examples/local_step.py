"""Local steps of a small language model that one GPU holds whole, and a federated
average.

    python examples/local_step.py

The model is an embedding, a root mean square norm and an output head: what the library
computes of any language model, without the layers between.  Two federation groups train
it on data of their own.  A local step is fl_embed, fl_layer_norm and fl_head_loss, their
gradients in the opposite order, and fl_adamw_tensors over the three parameters with
moments in 8 bits; after A steps the groups' working copies are averaged (fl_fedavg).  The
parameters are slices of one flat buffer, so the average is one call.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2609_20359_amd as P  # noqa: E402

V, D, T = 2000, 256, 1024
G, A = 2, 20
EPS, SCALE = 1e-5, D ** 0.5
HP = dict(lr=3e-3, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1)
SIZES = dict(embed=V * D, norm=D, head=V * D)


class Model:
    """A group's parameters: fp32 masters and bf16 working copies, moments in 8 bits."""

    def __init__(self, seed, groups_seed):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        n = sum(SIZES.values())
        self.layout = P.Layout([0, V * D, V * D + D, n], [1, 0, 1])
        self.master = torch.empty(n, device="cuda")
        masters = self.split(self.master)
        masters["embed"].copy_(torch.randn(V * D, generator=gen, device="cuda") * 0.02)
        masters["norm"].fill_(1.0)
        masters["head"].copy_(torch.randn(V * D, generator=gen, device="cuda") * 0.02)
        self.working = self.master.bfloat16()
        self.w = self.split(self.working)
        self.grad = torch.empty(n, dtype=torch.bfloat16, device="cuda")
        self.g = self.split(self.grad)
        self.tensors = P.Tensors(masters.values(), self.w.values(), [1, 0, 1])
        self.state = self.tensors.state(8)
        self.seed = groups_seed
        bf16 = dict(dtype=torch.bfloat16, device="cuda")
        self.x, self.y, self.dy, self.dx = (torch.empty(T, D, **bf16) for _ in range(4))
        self.rstd, self.loss, self.lse, self.target = (torch.empty(T, device="cuda") for _ in range(4))
        self.dloss = torch.full((T,), 1.0 / T, device="cuda")
        self.work = torch.empty(max(P.embed_workspace_bytes(T, V, D),
                                    P.layer_norm_workspace_bytes(T, D),
                                    P.head_workspace_bytes(T, V, D, grad=False),
                                    P.head_workspace_bytes(T, V, D, grad=True)),
                                dtype=torch.uint8, device="cuda")

    @staticmethod
    def split(flat):
        parts = flat.split(list(SIZES.values()))
        return dict(zip(SIZES, parts))

    def gradients(self, ids, labels):
        """The tokens' losses, and the gradients of their mean in self.grad."""
        w, g = self.w, self.g
        table, head = w["embed"].view(V, D), w["head"].view(V, D)
        P.fl_embed(ids, table, self.x, scale=SCALE)
        P.fl_layer_norm(self.x, w["norm"], None, EPS, self.y, None, self.rstd, rms=True)
        P.fl_head_loss(self.y, head, labels, self.loss, self.lse, self.target, workspace=self.work)
        P.fl_head_loss_grad(self.y, head, labels, self.lse, self.target, self.dloss, self.dy,
                            g["head"].view(V, D), workspace=self.work)
        P.fl_layer_norm_grad(self.x, w["norm"], None, self.rstd, self.dy, self.dx, g["norm"], None,
                             rms=True, workspace=self.work)
        P.fl_embed_grad(ids, self.dx, g["embed"].view(V, D), scale=SCALE, workspace=self.work)
        return self.loss

    def step(self, ids, labels, number):
        """One local step; the mean loss before it, on the GPU."""
        loss = self.gradients(ids, labels).mean()
        P.fl_adamw_tensors(self.tensors, HP, number, self.g.values(), self.state, seed=self.seed)
        return loss


class Data:
    """Tokens of a group, and the ones that follow: a fixed word after each word, or with
    a tenth of them any."""

    def __init__(self, seed):
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(seed)
        order = torch.Generator(device="cuda")
        order.manual_seed(1)
        self.after = torch.randperm(V, generator=order, device="cuda")

    def batch(self):
        u = torch.rand(T, generator=self.gen, device="cuda")
        ids = (V ** u).long().clamp_(max=V - 1)
        any_ = torch.randint(0, V, (T,), generator=self.gen, device="cuda")
        labels = torch.where(torch.rand(T, generator=self.gen, device="cuda") < 0.1, any_,
                             self.after[ids])
        return ids, labels


def run():
    """The round; each group's loss at its first and last step, and the models after the
    average."""
    groups = [Model(3, 10 + k) for k in range(G)]
    data = [Data(20 + k) for k in range(G)]
    said = []
    for number in range(1, A + 1):
        said.append(torch.stack([m.step(*d.batch(), number) for m, d in zip(groups, data)]))
    replicas = [m.working.clone() for m in groups]
    for m in groups:
        P.fl_fedavg(m.layout, replicas, [1.0] * G, m.master, m.working)
    torch.cuda.synchronize()
    out = dict(first=said[0].tolist(), last=said[-1].tolist(),
               models=[m.working.clone() for m in groups], masters=[m.master for m in groups],
               states=[m.state for m in groups])
    for m in groups:
        m.layout.close()
    return out


if __name__ == "__main__":
    r = run()
    for g in range(G):
        print("group %d: loss %.3f -> %.3f" % (g, r["first"][g], r["last"][g]))
    print("groups equal after averaging: %s" % torch.equal(r["models"][0], r["models"][1]))
