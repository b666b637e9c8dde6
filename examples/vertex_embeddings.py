"""Learned vertex embeddings from sampled edges: a row for every vertex, trained so that a vertex tells its neighbours from all others.

Each step samples neighbours of a batch of vertices (coop_sample), looks up the row of every edge's destination (coop_embed), norms it
(coop_layer_norm), predicts the edge's source among all vertices (coop_softmax_xent: no logits are stored), takes the gradients back the
same way, of the table for the touched rows only (coop_embed_grad_rows), and steps all parameters (AdamW; by default with moments of 8 bits,
and with the output weights held in bf16 beside their fp32 originals).  Nothing waits for the GPU but the sampler's edge count and the
losses that are printed.

    python examples/vertex_embeddings.py [--scale 16 --edges 1000000 --dim 128 --batch 1024 --steps 200]
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2310_12403_amd as P  # noqa: E402
import synth  # noqa: E402


class VertexEmbeddings:
    def __init__(self, n_vertices, dim, bits=8, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.table = torch.randn((n_vertices, dim), generator=g, device="cuda")
        self.out = torch.zeros((n_vertices, dim), device="cuda")
        self.out16 = self.out.to(torch.bfloat16)
        self.gamma, self.beta = torch.ones(dim, device="cuda"), torch.zeros(dim, device="cuda")
        self.opt = P.AdamW([self.table, self.out, self.gamma, self.beta], bits=bits, by_rows=[True, False, False, False],
                           copies=[None, self.out16, None, None])
        self.alpha = 1 / math.sqrt(dim)
        self.steps = 0

    def step(self, vertices, neighbours, lr):
        """vertices, neighbours: int32 [edges] on the device.  The step's losses, fp32 [edges]."""
        n = vertices.numel()
        x = P.coop_embed(self.table, vertices, dtype=torch.bfloat16)
        y, mean, rstd = P.coop_layer_norm(x, self.gamma, self.beta)
        loss, lse = P.coop_softmax_xent(y, self.out16, neighbours, alpha=self.alpha)
        dloss = torch.full((n,), 1 / max(n, 1), device="cuda")
        dy, dout = P.coop_softmax_xent_grad(y, self.out16, neighbours, lse, dloss, alpha=self.alpha)
        dx, dgamma, dbeta = P.coop_layer_norm_grad(dy, x, mean, rstd, self.gamma)
        rows = P.coop_embed_grad_rows(dx, vertices, self.table.shape[0], wait=False)
        self.steps += 1
        self.opt.set_grads([None, dout, dgamma, dbeta])
        self.opt.step(self.steps, lr, weight_decay=0.0, rows={0: rows}, seed=0)
        return loss


def edges_of(block):
    """(destination, source) of a block's edges, int32 on the device"""
    degrees = block.indptr.diff()
    return torch.repeat_interleave(block.dst_ids, degrees, output_size=block.n_edges), block.col_global


def train(indptr, indices, dim=128, batch=1024, fanout=10, steps=200, lr=1e-2, bits=8, seed=0, log=print):
    """Trains on a graph in the CSR format of coop_graph_load; returns the model and the mean loss of each step."""
    n_vertices = indptr.numel() - 1
    graph = P.coop_graph_load(indptr.cuda(), indices.cuda())
    batches = synth.seed_batches(n_vertices, min(batch, n_vertices), seed=seed)
    model = VertexEmbeddings(n_vertices, dim, bits, seed)
    losses = []
    for i in range(steps):
        block = P.coop_sample(graph, batches(i).cuda(), (fanout,), P.COOP_NS, it=i, seed=seed)[0]
        vertices, neighbours = edges_of(block)
        losses.append(model.step(vertices, neighbours, lr).mean())
        if log and (i % max(1, steps // 10) == 0 or i + 1 == steps):
            log("step %4d: %6d edges, loss %.4f (uniform: %.4f)" % (i, vertices.numel(), float(losses[-1]), math.log(n_vertices)))
    P.coop_gather_status()  # raises if an id or a target was out of range
    return model, [float(x) for x in losses]


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--scale", type=int, default=14, help="2^scale vertices of a synthetic R-MAT graph")
    ap.add_argument("--edges", type=int, default=262144)
    ap.add_argument("--dim", type=int, default=128)
    ap.add_argument("--batch", type=int, default=1024)
    ap.add_argument("--fanout", type=int, default=10)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--lr", type=float, default=1e-2)
    ap.add_argument("--bits", type=int, default=8, choices=(8, 32), help="of the optimizer's moments")
    a = ap.parse_args()
    train(*synth.rmat_csr(scale=a.scale, n_edges=a.edges), dim=a.dim, batch=a.batch, fanout=a.fanout, steps=a.steps, lr=a.lr, bits=a.bits)


if __name__ == "__main__":
    main()
