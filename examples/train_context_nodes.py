"""Trains node vectors on sampled blocks: learned embeddings, one attention layer per hop, softmax over all nodes.

Every step samples a mini-batch with the neighbour cache (``gs_sample_batch``), looks the input nodes' vectors up, lets every
hop's destinations attend over their sampled neighbours, and predicts a neighbour of each seed among all nodes of the graph.
Random-init weights, a seeded synthetic graph.

    python examples/train_context_nodes.py [--config tiny] [--steps 50] [--norm layer|rms] [--max-norm X]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2406_17918_b200 as gs  # noqa: E402
from paper_2406_17918_b200.autograd import block_attention, embedding, rms_norm, table_cross_entropy  # noqa: E402
from workloads import batch_seeds, build_graph, get_config, seed_permutation  # noqa: E402


class Model(torch.nn.Module):
    def __init__(self, num_nodes: int, hops: int, heads: int = 4, dim: int = 16, norm: str = "layer"):
        super().__init__()
        self.heads, self.dim, width = heads, dim, heads * dim
        new = lambda *shape: torch.nn.Parameter(torch.randn(*shape) * shape[-1] ** -0.5)  # noqa: E731
        self.vectors = new(num_nodes, width)                 # input vectors of the nodes
        self.context = new(num_nodes, width)                 # their vectors as prediction targets
        self.project = torch.nn.ParameterList([new(width, 3 * width) for _ in range(hops)])
        self.mix = torch.nn.ParameterList([new(width, width) for _ in range(hops)])
        self.norm = torch.nn.ParameterList([torch.nn.Parameter(torch.ones(width)) for _ in range(hops)]) if norm == "rms" else None

    def forward(self, input_nodes, blocks, sizes, fanouts):
        """blocks, input side first, as (indptr, indices); sizes: (destinations, sources) of each."""
        x = embedding(self.vectors, input_nodes, scale=self.vectors.shape[1] ** 0.5)
        for l, ((indptr, indices), (n, _), weight, mix, f) in enumerate(zip(blocks, sizes, self.project, self.mix, fanouts)):
            qkv = (x @ weight).view(x.shape[0], 3, self.heads, self.dim)      # strided operands: no copies
            h = block_attention(qkv[:n, 0], qkv[:, 1], qkv[:, 2], indptr, indices, max_row=f)
            h = h.reshape(n, -1) @ mix
            x = torch.nn.functional.layer_norm(x[:n] + h, x.shape[1:]) if self.norm is None else rms_norm(h, self.norm[l], residual=x[:n])[0]
        return x

    def loss(self, hidden, targets):
        return table_cross_entropy(hidden.bfloat16(), self.context.bfloat16(), targets)


def neighbour_targets(graph, seeds, generator):
    """A random neighbour of every seed, -1 for seeds without one."""
    begin, end = graph.indptr[seeds.long()], graph.indptr[seeds.long() + 1]
    pick = begin + (torch.rand(seeds.shape, generator=generator, device=seeds.device, dtype=torch.float64) * (end - begin)).long()
    return torch.where(end > begin, graph.indices[pick.clamp(max=graph.indices.numel() - 1)], -1)


def train(config: str = "tiny", steps: int = 50, lr: float = 0.02, log=print, norm: str = "layer", max_norm: float = 0.0):
    cfg = get_config(config)
    dev = torch.device("cuda")
    torch.manual_seed(1)
    rng = torch.Generator(device=dev)
    rng.manual_seed(2)
    graph = build_graph(cfg).to(dev)
    G = gs.gs_graph_create(graph.indptr, graph.indices, None)
    cache = gs.gs_cache_init(G, cfg["fanouts"], cfg["cache_width"], 3, cfg["shared"])
    workspace = torch.empty(gs.gs_workspace_bytes(G, cfg["fanouts"], cfg["batch"]), dtype=torch.uint8, device=dev)
    perm = seed_permutation(cfg)
    model = Model(cfg["num_nodes"], len(cfg["fanouts"]), norm=norm).to(dev)
    parameters = list(model.parameters())
    clip_workspace = torch.empty(gs.gs_grad_workspace_bytes(len(parameters)), dtype=torch.uint8, device=dev)
    optimizer = torch.optim.Adam(parameters, lr=lr)
    history = []
    for step in range(steps):
        seeds = batch_seeds(perm, step, cfg["batch"]).to(dev)
        blocks, nodes, _ = gs.gs_sample_batch(cache, seeds, gs.GS_MODE_OTF, cfg["runs"][0][1], step + 1, workspace)
        n, m = gs.gs_batch_counts(cache)                     # frontier sizes by sampling step, edges by layer
        hops = cache.num_hops
        sizes = [(n[hops - 1 - l], n[hops - l]) for l in range(hops)]
        csr = [(b.indptr(sizes[l][0]), b.indices(m[l])) for l, b in enumerate(blocks)]
        hidden = model(nodes[:n[hops]], csr, sizes, cfg["fanouts"])
        loss = model.loss(hidden, neighbour_targets(graph, seeds, rng)).mean()
        optimizer.zero_grad(set_to_none=True)
        loss.backward()
        gs.gs_train_status()                                 # synchronises; no step on gradients that a kernel did not finish
        if max_norm:
            gs.gs_grad_clip([p.grad for p in parameters if p.grad is not None], max_norm, clip_workspace)
        optimizer.step()
        history.append(float(loss.detach()))
        if step % 10 == 0 or step + 1 == steps:
            log("step %4d  input nodes %6d  loss %.4f" % (step, n[hops], history[-1]))
    return history


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--config", default="tiny")
    ap.add_argument("--steps", type=int, default=50)
    ap.add_argument("--norm", default="layer", choices=["layer", "rms"], help="norm behind every hop")
    ap.add_argument("--max-norm", type=float, default=0.0, help="gradients are scaled to this norm at most (0: left as they are)")
    a = ap.parse_args()
    train(a.config, a.steps, norm=a.norm, max_norm=a.max_norm)
