"""A training step of a sampled GCN with a learned vector per node, gated residuals and clipped gradients.

Graphs without features learn a row per node.  The rows of a layer are drawn anew for every layer (Section 5.1), so
that what a residual carries on cannot be the previous layer's output of the same node; it is the node's own row, looked up
once more:

    x_l = s T[S_l]                              the rows of the nodes of layer l              csgs_embed
    u_L = N(x_L)                                                                              csgs_norm_residual
    h_l = (P~_l relu(u_{l+1})) W_l              the sampled layer (Section 3, Eq. 1)          csgs_aggregate, csgs_layer_gemm
    u_l = N(beta x_l + a(gate_l) .* N(h_l))     gate, residual and the norms around them      csgs_norm_residual
    logits = u_0 W_out

The gradients go the same way back; a node that is in several layers' sets receives the sum of its rows' gradients
(csgs_embed_grad_rows), and what all gradients together measure is clipped (csgs_grad_clip) before the step.  No call waits for the device:
the numbers of sampled nodes stay there.

  python -m paper_2101_07706_amd.residual_gcn [--config tiny] [--steps 20]

trains on made-up labels: which part of the local id range a node is in.
"""
from __future__ import annotations

import argparse
import math
import time

import numpy as np
import torch

from . import csgs, pipeline, synth


class ResidualGCN:
    """Parameters, buffers and one training step.  The gradients of a step are left in .grads, the table's in .table_rows, .table_ids and
    .table_count; .norm and .status tell of the last clipping, .skipped how many steps were left out because their gradients were not finite (all on
    the device)."""

    def __init__(self, dg, width, n_classes, n_layers, batch, samples, skew, adj_cap, seed=0, max_norm=1.0, lr=0.1, beta=0.5, gate_act=csgs.GATE_SIGMOID):
        dev = self.device = dg.device
        self.dg, self.width, self.L, self.batch, self.B, self.skew, self.seed = dg, width, n_layers, batch, samples, skew, seed
        self.max_norm, self.lr, self.beta, self.gate_act, self.scale = max_norm, lr, beta, gate_act, math.sqrt(width)
        D, L, f32 = width, n_layers, torch.float32
        g = torch.Generator().manual_seed(seed)
        randn = lambda *shape, std: (torch.randn(*shape, generator=g) * std).to(dev)
        self.table = randn(dg.n_nodes, D, std=1.0 / math.sqrt(D))
        self.params = {"w_out": randn(D, n_classes, std=1.0 / math.sqrt(D)), "bottom.pre_w": torch.ones(D, device=dev), "bottom.pre_b": torch.zeros(D, device=dev)}
        for l in range(L):
            self.params[f"{l}.w"] = randn(D, D, std=1.0 / math.sqrt(D))
            self.params[f"{l}.gate"] = torch.zeros(D, device=dev)
            for k in ("post", "pre"):
                self.params[f"{l}.{k}_w"], self.params[f"{l}.{k}_b"] = torch.ones(D, device=dev), torch.zeros(D, device=dev)
        self.grads = {k: torch.zeros_like(v) for k, v in self.params.items()}
        # sampling
        n_max = max(batch, samples)
        self.ws = pipeline.Workspace(dg.n_nodes, n_max, samples, dg.colidx.numel(), dev)
        self.lbs = [pipeline.LayerBuffers(n_max, samples, dg.n_nodes, adj_cap, dg.n_parts, dev) for _ in range(L)]
        # rows of layer 0 are the batch, of layer l the nodes drawn for layer l - 1; all layers' ids and rows lie after each other
        self.caps = [batch] + [samples] * L
        self.at = [0] + list(np.cumsum(self.caps))
        total = self.at[-1]
        part = lambda t: [t[self.at[l]:self.at[l + 1]] for l in range(L + 1)]
        new = lambda: torch.zeros(total, D, dtype=f32, device=dev)
        self.ids = torch.full((total,), -1, dtype=torch.int32, device=dev)
        self.place = torch.arange(samples, dtype=torch.int32, device=dev)
        self.X, self.U, self.dX, self.dU = part(new()), part(new()), new(), part(new())
        self.dX_parts = part(self.dX)
        self.H, self.Z, self.dH, self.dZ = (part(new())[:L] for _ in range(4))
        self.logits = torch.zeros(batch, n_classes, dtype=f32, device=dev)
        self.table_rows, self.table_ids = torch.zeros(total, D, dtype=f32, device=dev), torch.zeros(total, dtype=torch.int32, device=dev)
        self.table_count, self.row_place = torch.zeros(1, dtype=torch.int32, device=dev), torch.arange(total, dtype=torch.int32, device=dev)
        self.norm, self.status, self.skipped = torch.zeros(1, dtype=f32, device=dev), *(torch.zeros(1, dtype=torch.int32, device=dev) for _ in range(2))
        # scratch of the gradient calls; they follow each other on one stream
        nbytes = max([csgs.csgs_embed_grad_scratch_bytes(total, dg.n_nodes, D), csgs.csgs_aggregate_grad_scratch_bytes(samples, self.lbs[0].adj_col.numel()),
                      csgs.csgs_layer_gemm_grad_w_scratch_bytes(n_max, D, max(D, n_classes)), csgs.csgs_layer_gemm_grad_w_scratch_bytes(n_max, D, n_classes)]
                     + [csgs.csgs_norm_residual_grad_scratch_bytes(c, D) for c in self.caps])
        self.scratch = torch.empty(nbytes // 8 + 32, dtype=torch.int64, device=dev)
        names = list(self.grads)
        self.list = csgs.make_grad_list([self.grads[k] for k in names] + [self.table_rows], rows_dev=[None] * len(names) + [self.table_count])

    def rows_dev(self, l):
        """Device count of the rows of layer l (None: all of the batch)."""
        return None if l == 0 else self.lbs[l - 1].n_next

    def norms(self, l):
        """Arguments of csgs_norm_residual and its gradient for layer l (the last one: the bottom's norm alone)."""
        p = self.params
        if l == self.L:
            return dict(pre=csgs.NORM_LAYER, pre_w=p["bottom.pre_w"], pre_b=p["bottom.pre_b"], M_dev=self.rows_dev(l))
        return dict(gate=p[f"{l}.gate"], gate_act=self.gate_act, post=csgs.NORM_RMS, post_w=p[f"{l}.post_w"], post_b=p[f"{l}.post_b"], pre=csgs.NORM_LAYER,
                    pre_w=p[f"{l}.pre_w"], pre_b=p[f"{l}.pre_b"], beta=self.beta, M_dev=self.rows_dev(l))

    def forward(self, S0, it):
        """Samples the layers of the batch S0 (device int32, distinct ids) and computes its logits."""
        assert S0.numel() == self.batch
        L, lbs = self.L, self.lbs
        self.ids[:self.batch] = S0
        for l in range(L):
            pipeline.sample_step(self.dg, self.ws, S0 if l == 0 else None, self.skew, self.B, self.seed, it, l, lbs[l], want_q=False)
            # places past the count hold no node
            self.ids[self.at[l + 1]:self.at[l + 2]] = torch.where(self.place < lbs[l].n_next, lbs[l].S_next, -1)
        for l in range(L + 1):
            csgs.csgs_embed(self.table, self.ids[self.at[l]:self.at[l + 1]], self.X[l], scale=self.scale, n_dev=self.rows_dev(l))
        csgs.csgs_norm_residual(self.X[L], None, None, self.U[L], **self.norms(L))
        for l in range(L - 1, -1, -1):
            pipeline.compute_step(lbs[l], self.caps[l], self.U[l + 1], None, False, True, self.params[f"{l}.w"], self.Z[l], self.H[l], nS_dev=self.rows_dev(l))
            csgs.csgs_norm_residual(self.X[l], self.H[l], None, self.U[l], **self.norms(l))
        csgs.csgs_layer_gemm(self.U[0], self.params["w_out"], self.logits)
        return self.logits

    def backward(self, G):
        """Gradients of everything from G = dL/dlogits, before clipping."""
        L, g, lbs = self.L, self.grads, self.lbs
        csgs.csgs_layer_gemm_grad_w(self.U[0], G, g["w_out"], self.scratch)
        csgs.csgs_layer_gemm_grad_z(G, self.params["w_out"], self.dU[0])
        for l in range(L):
            n = self.rows_dev(l)
            csgs.csgs_norm_residual_grad(self.X[l], self.H[l], None, self.dU[l], self.dX_parts[l], self.dH[l], g[f"{l}.gate"], g[f"{l}.post_w"], g[f"{l}.post_b"],
                                         g[f"{l}.pre_w"], g[f"{l}.pre_b"], self.scratch, **self.norms(l))
            csgs.csgs_layer_gemm_grad_w(self.Z[l], self.dH[l], g[f"{l}.w"], self.scratch, M_dev=n)
            csgs.csgs_layer_gemm_grad_z(self.dH[l], self.params[f"{l}.w"], self.dZ[l], M_dev=n)
            csgs.csgs_aggregate_grad(lbs[l].adj_rowptr[:self.caps[l] + 1], lbs[l].adj_col, lbs[l].adj_val, lbs[l].n_next, self.dZ[l], self.U[l + 1], self.dU[l + 1],
                                     self.scratch, nS_dev=n)
        csgs.csgs_norm_residual_grad(self.X[L], None, None, self.dU[L], self.dX_parts[L], None, None, None, None, g["bottom.pre_w"], g["bottom.pre_b"], self.scratch,
                                     **self.norms(L))
        csgs.csgs_embed_grad_rows(self.ids, self.dX, self.dg.n_nodes, self.table_ids, self.table_count, self.table_rows, self.scratch, scale=self.scale)

    def clip(self):
        self.status.zero_()      # (calls only set bits)
        csgs.csgs_grad_clip(self.list, csgs.GRAD_L2, self.max_norm, self.norm, self.status)

    def descend(self):
        """A step of gradient descent on all parameters.  Clipping makes NaN of gradients whose norm is not finite: such a step changes nothing.  Decided on the
        device, from the status and not from the norm, which as a float may be infinite where the total is not."""
        finite = (self.status & csgs.ST_NONFINITE_GRAD) == 0
        self.skipped += ~finite
        for k, p in self.params.items():
            p.sub_(torch.where(finite, self.grads[k], 0.0), alpha=self.lr)
        live = (self.row_place < self.table_count) & finite
        step = torch.where(live.unsqueeze(1), self.table_rows, torch.zeros(1, device=self.device))
        self.table.index_add_(0, torch.where(live, self.table_ids, 0).long(), step, alpha=-self.lr)

    def step(self, S0, labels, it):
        """One training step: the mean cross entropy of the batch (device), before the step."""
        logp = torch.log_softmax(self.forward(S0, it), 1)
        G = torch.exp(logp)
        pick = labels.unsqueeze(1)
        loss = -logp.gather(1, pick).mean()
        G.scatter_add_(1, pick, torch.full_like(pick, -1, dtype=G.dtype))
        self.backward(G.div_(self.batch))
        self.clip()
        self.descend()
        return loss


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--config", default="tiny", choices=list(synth.CONFIGS))
    ap.add_argument("--steps", type=int, default=20)
    a = ap.parse_args()
    cfg = synth.CONFIGS[a.config]
    g = synth.make_graph(cfg)
    dg = pipeline.DeviceGraph(g)
    n_classes = cfg.n_classes or 4
    net = ResidualGCN(dg, cfg.hidden, n_classes, cfg.n_layers, cfg.batch, cfg.samples, cfg.skew, min(g.nnz, 16_000_000))
    for it in range(a.steps):
        S0 = torch.from_numpy(synth.make_batch(g, cfg.batch, cfg.seed, it)).to(dg.device)
        labels = (S0.long() - g.local_lo) * n_classes // (g.local_hi - g.local_lo)
        torch.cuda.synchronize()
        t = time.perf_counter()
        loss = float(net.step(S0, labels, it))
        ms = 1e3 * (time.perf_counter() - t)
        print(f"step {it}: loss {loss:.4f}, gradient norm {float(net.norm):.4f}, rows of the table {int(net.table_count)}, {ms:.2f} ms"
              + (", not taken" if int(net.status) else ""), flush=True)
    assert int(net.skipped) == 0 and all(int(lb.status) == 0 for lb in net.lbs), "a call reported an error"


if __name__ == "__main__":
    main()
