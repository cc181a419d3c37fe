"""A head of gated residual blocks over embeddings that the engine keeps current: trained with AdamW, asked in 8 bits.

    python examples/residual_head.py [--config 1] [--div 1] [--steps 60] [--batches 3] [--blocks 2] [--type f32|bf16|f16] [--bits 8|32]

The graph, the GNN and the update batches are those of synth.get_config.  A block normalises the residual stream, widens it by a gated pair of
projections and narrows it by a linear layer, whose result joins the stream in the next block's norm.  Parameters are held in 32 bits; the
step writes the 16-bit copies that the products read.  Then edges come and go, and the head answers for the rows that changed, its gated
pairs in 8 bits.
"""
import argparse
import os
import sys

import numpy as np
import torch

HERE = os.path.dirname(os.path.abspath(__file__))
for p in (os.path.dirname(HERE), HERE):
    if p not in sys.path:
        sys.path.insert(0, p)
import synth  # noqa: E402
from answer_head import DeviceRows  # noqa: E402
from paper_2309_11071_amd import Ink, head  # noqa: E402
from paper_2309_11071_amd.binding import make_updates  # noqa: E402


class ResidualHead:
    """Blocks of norm, gated pair and linear layer, then a norm and a classifier."""

    def __init__(self, dim, hidden, blocks, classes, dtype, bits=32, seed=0):
        g = torch.Generator().manual_seed(seed)

        def xavier(k, m):
            return (torch.rand(k, m, generator=g) * 2 - 1) * (6.0 / (k + m)) ** 0.5
        made = []
        for _ in range(blocks):
            made += [torch.ones(dim), xavier(dim, hidden), xavier(dim, hidden), xavier(hidden, dim)]
        made += [torch.ones(dim), xavier(dim, classes), torch.zeros(classes)]
        self.blocks, self.dtype, self.steps = blocks, dtype, 0
        self.params = [p.cuda() for p in made]
        self.copies = None if dtype is torch.float32 else [p.to(dtype) for p in self.params]
        self.moments = head.adamw_moments(self.params, bits)

    @property
    def weights(self):
        return self.params if self.copies is None else self.copies

    def forward(self, rows):
        w, kept, stream, out = self.weights, [], rows.to(self.dtype), None
        for b in range(self.blocks):
            gamma, gate, up, down = w[4 * b:4 * b + 4]
            y, stream, rstd = head.rms_norm(stream if out is None else out, gamma, residual=None if out is None else stream)
            h = head.gated(y, gate, up)
            out = head.linear(h, down)
            kept.append((y, stream, rstd, h))
        y, stream, rstd = head.rms_norm(out, w[-3], residual=stream)
        return head.linear(y, w[-2], w[-1]), kept + [(y, stream, rstd)]

    def backward(self, d_logits, kept):
        """Gradients of the parameters, in their order, and that of the rows."""
        w, grads = self.weights, []
        y, stream, rstd = kept[-1]
        dy, d_last, d_bias = head.linear_backward(d_logits, y, w[-2])
        ds, d_gamma = head.rms_norm_backward(dy, stream, rstd, w[-3])
        grads = [d_gamma, d_last, d_bias]
        for b in reversed(range(self.blocks)):
            gamma, gate, up, down = w[4 * b:4 * b + 4]
            y, stream, rstd, h = kept[b]
            dh, d_down, _ = head.linear_backward(ds, h, down, need_dbias=False)
            dy, d_gate, d_up = head.gated_backward(dh, y, gate, up)
            ds, d_gamma = head.rms_norm_backward(dy, stream, rstd, gamma, d_total=ds)
            grads = [d_gamma, d_gate, d_up, d_down] + grads
        return grads, ds

    def step(self, rows, labels, rate):
        """One step of AdamW on the mean of -log p(label); returns that mean before the step (a GPU scalar)."""
        logits, kept = self.forward(rows)
        out = head.log_probs(logits, labels)
        n = (labels >= 0).sum().clamp(min=1)
        scale = 1024.0 if self.dtype is torch.float16 else 1.0     # the range of half precision; the step takes it out again
        g = (-scale / n).expand(len(labels)).contiguous()
        grads, _ = self.backward(head.log_probs_backward(logits, labels, out["lse"], g_logp=g), kept)
        self.steps += 1
        head.adamw(self.params, grads, self.moments, self.steps, lr=rate, grad_scale=1.0 / scale, copies=self.copies, seed=1)
        return -out["logp"].sum() / n

    def to_8_bits(self):
        """The gated pairs' weights as e4m3 numbers with a scale for each column, a column's numbers side by side: laid out once after training."""
        def eight(w):
            scale = w.float().abs().amax(0) / 448
            return (w.float() / scale.clamp(min=1e-30)).t().contiguous().to(head.E4M3).t(), scale
        self.eights = [eight(self.params[4 * b + 1]) + eight(self.params[4 * b + 2]) for b in range(self.blocks)]

    def answer(self, rows, labels=None, top=3):
        """Log probabilities and best classes, with the gated pairs in 8 bits."""
        w, stream, out = self.weights, rows.to(self.dtype), None
        for b in range(self.blocks):
            gate, gate_scale, up, up_scale = self.eights[b]
            y, scale, stream, _ = head.rms_norm(stream if out is None else out, w[4 * b], residual=None if out is None else stream, out_dtype=head.E4M3)
            h = head.gated(y, gate, up, x_scale=scale, gate_scale=gate_scale, up_scale=up_scale, out_dtype=self.dtype)
            out = head.linear(h, w[4 * b + 3])
        y, _, _ = head.rms_norm(out, w[-3], residual=stream)
        return head.log_probs(head.linear(y, w[-2], w[-1]), labels, top=top)


def main(argv=None):
    a = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    a.add_argument("--config", type=int, default=1)
    a.add_argument("--div", type=int, default=1)
    a.add_argument("--steps", type=int, default=60)
    a.add_argument("--batches", type=int, default=3)
    a.add_argument("--blocks", type=int, default=2)
    a.add_argument("--classes", type=int, default=7)
    a.add_argument("--type", default="bf16", choices=("f32", "bf16", "f16"))
    a.add_argument("--bits", type=int, default=8, choices=(8, 32))
    a = a.parse_args(argv)
    cfg = synth.get_config(a.config, a.div)
    src, dst = synth.make_graph(cfg)
    rowptr, col = synth.in_csr_from_edges(cfg.n_nodes, src, dst)
    ink = Ink(rowptr, col, synth.make_features(cfg), synth.make_model(cfg))
    ink.full_infer()
    table = torch.from_numpy(ink.get_layer(ink.n_layers, 0)).cuda()
    # labels that embeddings can tell: the largest of a few random projections of the embedding; one node in ten has none
    g = torch.Generator().manual_seed(1)
    labels = (table.cpu() @ torch.randn(table.shape[1], a.classes, generator=g)).argmax(1)
    labels[torch.rand(len(labels), generator=g) < 0.1] = -1
    labels = labels.cuda()
    dim = table.shape[1]
    model = ResidualHead(dim, dim * 8 // 3, a.blocks, a.classes, dict(f32=torch.float32, bf16=torch.bfloat16, f16=torch.float16)[a.type], a.bits)
    losses = [float(model.step(table, labels, 3e-3)) for _ in range(a.steps)]
    model.to_8_bits()
    before = model.answer(table, labels)
    known = labels >= 0
    print("loss %.4f -> %.4f; right in 8 bits %.1f %%" % (losses[0], losses[-1], 100 * float((before["top_ids"][:, 0] == labels)[known].float().mean())))
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
    sys.exit(0 if np.isfinite(losses).all() and same > 0.99 else 1)
