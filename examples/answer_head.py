"""An answer head over embeddings that the engine keeps current: trained on a graph's nodes, asked after every batch of updates.

    python examples/answer_head.py [--config 1] [--div 1] [--steps 60] [--batches 3] [--type f32|bf16|f16]

The graph, the GNN and the update batches are those of synth.get_config.  A head of layer norm, one hidden layer with a
residual and a classifier learns labels (here: made from the nodes' features) from the embeddings of all nodes.  Then
edges come and go: the engine returns the rows that changed and the head answers for those rows only: the label's
log probability, how uncertain the answer is, and the three best classes.
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import synth  # noqa: E402
from paper_2309_11071_amd import Ink, head  # noqa: E402
from paper_2309_11071_amd.binding import make_updates  # noqa: E402


class DeviceRows:
    """Rows in the engine's memory (an update's result) as something torch.as_tensor can view until the engine's next call."""

    def __init__(self, ptr, shape, typestr):
        self.__cuda_array_interface__ = dict(data=(ptr, False), shape=shape, typestr=typestr, version=3)


class Head:
    """norm -> x + gelu(x W1 + b1) -> W2 + b2, with 32-bit logits.  Weights are held in 32 bits and cast for the products."""

    def __init__(self, dim, classes, dtype, seed=0):
        g = torch.Generator().manual_seed(seed)

        def xavier(k, m):
            return (torch.rand(k, m, generator=g) * 2 - 1) * (6.0 / (k + m)) ** 0.5
        self.dtype = dtype
        self.p = dict(gamma=torch.ones(dim), beta=torch.zeros(dim), w1=xavier(dim, dim), b1=torch.zeros(dim), w2=xavier(dim, classes), b2=torch.zeros(classes))
        self.p = {k: v.cuda() for k, v in self.p.items()}

    def forward(self, rows):
        p, t = {k: v.to(self.dtype) for k, v in self.p.items()}, self.dtype
        x = rows.to(t)
        y, mean, rstd = head.layer_norm(x, self.p["gamma"], self.p["beta"])
        h, z = head.linear(y, p["w1"], p["b1"], act="gelu", residual=y, keep_pre=True)
        logits = head.linear(h, p["w2"], p["b2"], out_dtype=torch.float32 if t is not torch.float16 else None)
        return logits, (p, x, mean, rstd, y, z, h)

    def answer(self, rows, labels=None, top=3):
        return head.log_probs(self.forward(rows)[0], labels, top=top)

    def step(self, rows, labels, rate):
        """One step of gradient descent on the mean of -log p(label); returns that mean before the step (a GPU scalar)."""
        logits, (p, x, mean, rstd, y, z, h) = self.forward(rows)
        out = head.log_probs(logits, labels)
        n = (labels >= 0).sum().clamp(min=1)
        scale = 1024.0 if self.dtype is torch.float16 else 1.0     # the range of half precision; the update takes it out again
        g = (-scale / n).expand(len(labels)).contiguous()
        d_logits = head.log_probs_backward(logits, labels, out["lse"], g_logp=g)
        dh, dw2, db2 = head.linear_backward(d_logits, h, p["w2"])
        dy, dw1, db1 = head.linear_backward(dh, y, p["w1"], pre=z, act="gelu")
        _, dgamma, dbeta = head.layer_norm_backward(dy + dh, x, mean, rstd, self.p["gamma"], need_dx=False)
        for k, d in dict(gamma=dgamma, beta=dbeta, w1=dw1, b1=db1, w2=dw2, b2=db2).items():
            self.p[k] -= rate / scale * d.float()
        return -out["logp"].sum() / n


def main(argv=None):
    a = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    a.add_argument("--config", type=int, default=1)
    a.add_argument("--div", type=int, default=1)
    a.add_argument("--steps", type=int, default=60)
    a.add_argument("--batches", type=int, default=3)
    a.add_argument("--classes", type=int, default=7)
    a.add_argument("--type", default="f32", choices=("f32", "bf16", "f16"))
    a = a.parse_args(argv)
    dtype = dict(f32=torch.float32, bf16=torch.bfloat16, f16=torch.float16)[a.type]
    cfg = synth.get_config(a.config, a.div)
    src, dst = synth.make_graph(cfg)
    rowptr, col = synth.in_csr_from_edges(cfg.n_nodes, src, dst)
    features = synth.make_features(cfg)
    ink = Ink(rowptr, col, features, synth.make_model(cfg))
    ink.full_infer()
    table = torch.from_numpy(ink.get_layer(ink.n_layers, 0)).cuda()
    # labels that embeddings can tell: the largest of a few random projections of the embedding; one node in ten has none
    g = torch.Generator().manual_seed(1)
    labels = (table.cpu() @ torch.randn(table.shape[1], a.classes, generator=g)).argmax(1)
    labels[torch.rand(len(labels), generator=g) < 0.1] = -1
    labels = labels.cuda()
    model = Head(table.shape[1], a.classes, dtype)
    losses = [float(model.step(table, labels, 0.5)) for _ in range(a.steps)]
    before = model.answer(table, labels)
    known = labels >= 0
    print("loss %.4f -> %.4f; right %.1f %%" % (losses[0], losses[-1], 100 * float((before["top_ids"][:, 0] == labels)[known].float().mean())))
    sampler = synth.BatchSampler(cfg, src, dst)
    answers = before["top_ids"].clone()
    for _ in range(a.batches):
        res = ink.apply_updates(make_updates(*sampler.next_batch()), fetch=False)
        n = res["n_changed"]
        if n == 0:
            continue
        ids = torch.as_tensor(DeviceRows(res["changed_ids_ptr"], (n,), "<i4"), device="cuda").long()
        rows = torch.as_tensor(DeviceRows(res["embeddings_ptr"], (n, ink.out_dim), "<f4"), device="cuda")
        table[ids] = rows
        out = model.answer(rows, labels[ids])
        moved = int((out["top_ids"][:, 0] != answers[ids, 0]).sum())
        answers[ids] = out["top_ids"]
        print("%d nodes changed, %d answers; mean entropy %.3f, mean log p %.3f" % (n, moved, float(out["entropy"].mean()), float(out["logp"].mean())))
    whole = model.answer(table, labels)          # the answers kept up to date are those of all rows at once
    ink.close()
    return losses, answers, whole["top_ids"]


if __name__ == "__main__":
    losses, kept, whole = main()
    same = float((kept == whole).all(1).float().mean())
    print("answers kept up to date agree with a pass over all nodes: %.2f %%" % (100 * same))
    sys.exit(0 if np.isfinite(losses).all() and same > 0.999 else 1)
