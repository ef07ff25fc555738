"""A sparse expert layer over the nodes of a batch of graphs, from the library's operators.

    h   = act(group norm of x)            over the nodes of each graph
    w   = router(h Wr)                    k of E experts a node, balance and z loss
    y   = sum_j w_j (h We[expert j])      nodes sorted by expert, typed products, weighted sum
    out = x + dropout(y)

Dispatch and combine are message passing: the (node, expert) pairs are a COO graph whose CSR by expert
sorts the nodes, and the weighted sum over a node's k results is an aggregation.  ``forward`` and
``backward`` are a training step (bf16 weights and activations), ``serve`` the same layer with the
experts' weights in 4 bits and no host synchronisation.  Run as a program it takes a few steps and times
both.
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2507_16991_amd as mp  # noqa: E402

BF16 = torch.bfloat16


class ExpertLayer:
    """Weights of the layer: F channels, E experts (a multiple of 8, at most 16), k of them a node."""

    def __init__(self, F, E, k, groups, *, act="silu", p=0.1, seed=0, device="cuda:0"):
        g = torch.Generator(device=device).manual_seed(seed)

        def randn(*shape):
            return torch.randn(*shape, generator=g, device=device)

        self.F, self.E, self.k, self.groups, self.act, self.p, self.seed = F, E, k, groups, act, p, seed
        self.gamma = 1 + 0.1 * randn(F)
        self.beta = 0.1 * randn(F)
        self.Wr = (randn(1, F, E) / F ** 0.5).to(BF16)
        self.We = (randn(E, F, F) / F ** 0.5).to(BF16)
        self.quantized = None

    def _dispatch(self, idx):
        """Nodes sorted by expert: (rowptr [E + 1], node of every place, the places of a node's choices,
        pair of every place)."""
        N = int(idx.shape[0])
        pairs = torch.arange(N * self.k, device=idx.device, dtype=torch.int32)
        rowptr, node, pair, _ = mp.coo_to_csr(pairs // self.k, idx.view(-1), self.E, want_perm=True,
                                              check=False)
        place = torch.empty_like(pairs)
        place[pair.long()] = pairs
        return rowptr, node, place, pair

    def _starts(self, N, device):
        return torch.arange(0, (N + 1) * self.k, self.k, device=device, dtype=torch.int32)

    def forward(self, ptr, x, step):
        """x [N, F] bf16 -> (out [N, F] bf16, losses [2]: balance and z, what backward needs)."""
        N = int(x.shape[0])
        h, mean, rstd = mp.group_norm(ptr, x, self.groups, weight=self.gamma, bias=self.beta, act=self.act)
        logits = mp.segment_matmul([0, N], h, self.Wr)
        idx, weight, counts, losses = mp.route(logits, self.k)
        rowptr, node, place, pair = self._dispatch(idx)
        seg = rowptr.tolist()  # (the bf16 products take the segments from the host)
        hs = mp.message_gather(node, h, msg_dtype=BF16)
        ys = mp.segment_matmul(seg, hs, self.We)
        starts = self._starts(N, x.device)
        y, _, _ = mp.spmm(starts, place, ys, mp.MP_SUM, w=weight.view(-1), out_dtype=BF16)
        out = mp.dropout(y, self.p, self.seed, offset=step, residual=x)
        saved = dict(ptr=ptr, x=x, step=step, h=h, mean=mean, rstd=rstd, logits=logits, idx=idx,
                     weight=weight, counts=counts, node=node, place=place, pair=pair, seg=seg, hs=hs, ys=ys,
                     starts=starts)
        return out, losses, saved

    def backward(self, s, dout, dloss):
        """Gradients given dout [N, F] bf16 and dloss [2] (the losses' weights): a dict of x and the
        weights."""
        N = int(dout.shape[0])
        dy = mp.dropout_backward(dout, self.p, self.seed, offset=s["step"])
        # y = sum_j w_j ys[place of (node, j)]
        w = s["weight"].view(-1)
        dys = mp.message_gather(s["node"], dy, w=w[s["pair"].long()])
        dw = mp.edge_dot(s["ys"], dy, bidx=s["node"], oidx=s["pair"]).view(N, self.k)
        dhs, dWe = mp.segment_matmul_backward(s["seg"], s["hs"], self.We, dys.to(BF16))
        dh, _, _ = mp.spmm(s["starts"], s["place"], dhs, mp.MP_SUM)
        dlogits = mp.route_backward(s["logits"], s["idx"], s["weight"], s["counts"], dweight=dw, dloss=dloss)
        dhr, dWr = mp.segment_matmul_backward([0, N], s["h"], self.Wr, dlogits.to(BF16))
        dx, dgamma, dbeta = mp.group_norm_backward(
            s["ptr"], s["x"], (dh + dhr).to(BF16), self.groups, s["mean"], s["rstd"], weight=self.gamma,
            bias=self.beta, act=self.act)
        return dict(x=dx + dout, gamma=dgamma, beta=dbeta, Wr=dWr, We=dWe)

    def serve(self, ptr, x):
        """The layer without dropout, the experts' weights in 4 bits."""
        if self.quantized is None:  # laid out once
            self.quantized = mp.mx_quantize(self.We.transpose(1, 2))
        N = int(x.shape[0])
        h, _, _ = mp.group_norm(ptr, x, self.groups, weight=self.gamma, bias=self.beta, act=self.act)
        idx, weight, _, _ = mp.route(mp.segment_matmul([0, N], h, self.Wr), self.k)
        rowptr, node, place, _ = self._dispatch(idx)
        ys = mp.mx_segment_matmul(rowptr, mp.message_gather(node, h, msg_dtype=BF16), *self.quantized)
        y, _, _ = mp.spmm(self._starts(N, x.device), place, ys, mp.MP_SUM, w=weight.view(-1), out_dtype=BF16)
        return x + y


def batch(N, graphs, F, seed=0, device="cuda:0"):
    """Features of N nodes in `graphs` graphs of random sizes."""
    g = torch.Generator().manual_seed(seed)
    cut = torch.randint(0, N + 1, (graphs - 1,), generator=g).sort().values
    ptr = torch.cat([torch.zeros(1, dtype=torch.long), cut, torch.full((1,), N)]).int().to(device)
    return ptr, torch.randn(N, F, generator=g).to(BF16).to(device)


def main():
    layer = ExpertLayer(F=128, E=8, k=2, groups=32)
    ptr, x = batch(169343, 4096, 128)
    target = torch.randn_like(x, dtype=torch.float32)
    dloss = torch.tensor([0.01, 0.001], device=x.device)
    t0, t1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    for step in range(5):
        t0.record()
        out, losses, saved = layer.forward(ptr, x, step)
        diff = out.float() - target
        grads = layer.backward(saved, (diff * (2.0 / diff.numel())).to(BF16), dloss)
        layer.We = (layer.We.float() - 50.0 * grads["We"]).to(BF16)
        layer.Wr = (layer.Wr.float() - 0.5 * grads["Wr"]).to(BF16)
        t1.record()
        torch.cuda.synchronize()
        print(f"step {step}: mean square {float(diff.square().mean()):.4f}, balance {float(losses[0]):.4f}, "
              f"z {float(losses[1]):.4f}, {t0.elapsed_time(t1):.2f} ms", flush=True)
    layer.quantized = None
    for rows in (16, 169343):
        p = torch.tensor([0, rows], dtype=torch.int32, device=x.device)
        layer.serve(p, x[:rows])
        t0.record()
        layer.serve(p, x[:rows])
        t1.record()
        torch.cuda.synchronize()
        print(f"serve {rows} rows: {t0.elapsed_time(t1):.3f} ms", flush=True)


if __name__ == "__main__":
    main()
