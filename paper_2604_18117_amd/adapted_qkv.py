"""Example: the QKV projection of an image transformer as a server and a fine-tuning run use it, all of it on this library's kernels.

Serving (``AdaptedQKV.__call__``): one quantised projection for every request of the batch, the low-rank adapters of the requests that have one added in
place on its output, queries and keys normalised and rotated by the positions of their patches in place in the same rows:

    activation step -> forward -> adapters -> norm and rotation of queries and keys

Training (``AdaptedQKV.backward``): the gradients of the adapters (and of the norm's weights) from those of the finished queries, keys and values, through
the frozen projection.

    python -m paper_2604_18117_amd.adapted_qkv            # serves a batch, prints the time of its four calls
    python -m paper_2604_18117_amd.adapted_qkv --train    # fits two adapters to a shifted layer, prints the loss
"""
from __future__ import annotations

import argparse
import math

import torch

from paper_2604_18117_amd import binding as lq


def grid_positions(height: int, width: int) -> torch.Tensor:
    """(row, column) of every patch of an image, row by row."""
    y, x = torch.meshgrid(torch.arange(height), torch.arange(width), indexing="ij")
    return torch.stack([y.flatten(), x.flatten()], 1).float().cuda()


class AdaptedQKV:
    """A quantised QKV projection with a pool of adapters, two-axis positions and buffers for batches of M rows.

    W: 3 dim x dim fp32, with a low-rank branch L, R (as for lq_pack_weights); heads of dim / heads values."""

    def __init__(self, W, L, R, M: int, heads: int, slots: int, rank: int, theta: float = 1e4):
        n, dim = W.shape
        self.dim, self.heads, self.head_dim, self.M = dim, heads, dim // heads, M
        self.cfg = lq.make_config(n, dim, L.shape[1], "int", 64, 8, 8)
        self.packed = lq.lq_pack_weights(self.cfg, W, L, R)
        self.adapters = lq.make_adapter_config(n, dim, rank, slots)
        pairs = [self.head_dim // 4, self.head_dim // 4]  # half of a head's pairs to each axis
        self.qk = lq.make_qk_config(heads, heads, self.head_dim, pairs, "half")
        self.inv_freq = torch.cat([theta ** (-torch.arange(p, dtype=torch.float64) / p) for p in pairs]).float().cuda()
        self.wq, self.wk = torch.ones(self.head_dim, device="cuda"), torch.ones(self.head_dim, device="cuda")
        # the pool: A starts random, B at zero, so that a new adapter changes nothing
        self.A = (torch.randn(slots, rank, dim, device="cuda") / math.sqrt(dim)).bfloat16()
        self.B = torch.zeros(slots, n, rank, dtype=torch.bfloat16, device="cuda")
        self.ranks = torch.full((slots,), rank, dtype=torch.int32, device="cuda")
        self.scales = torch.ones(slots, device="cuda")
        self.act = torch.empty(lq.lq_act_sizes(self.cfg, M), dtype=torch.uint8, device="cuda")
        inter, work = lq.lq_adapter_sizes(self.adapters, M)
        self.inter, self.work = torch.empty(inter, dtype=torch.uint8, device="cuda"), torch.empty(work, dtype=torch.uint8, device="cuda")
        self.plan = torch.empty(lq.lq_adapter_plan_sizes(M, slots), dtype=torch.uint8, device="cuda")
        self.rows = None  # of the batch that the plan is for

    def group(self, ids: torch.Tensor) -> None:
        """The batch's composition: the adapter of each row (-1: none).  Once per batch; every layer of a model could share it."""
        self.rows = None
        lq.lq_adapter_plan(self.adapters.slots, ids, plan=self.plan)
        self.rows = ids.shape[0]

    def _grouped(self, X) -> None:
        if X.shape[0] != self.rows:
            raise ValueError(f"a batch of {X.shape[0]} rows, the last one grouped has {self.rows}")

    def heads_of(self, rows: torch.Tensor):
        """Views of the queries and keys in the projection's rows."""
        return [rows[:, k * self.dim:(k + 1) * self.dim].view(-1, self.heads, self.head_dim) for k in range(2)]

    def project(self, X, Y=None):
        """The adapted projection, before the norm: what the backward needs beside X."""
        self._grouped(X)
        lq.lq_quantize_act(self.cfg, self.packed, X, act=self.act)
        Y = lq.lq_linear_lowrank_fwd(self.cfg, self.packed, self.act, X.shape[0], Y=Y)
        return lq.lq_adapter_fwd(self.adapters, self.plan, X, self.A, self.B, self.ranks, self.scales, Y, Y=Y, inter=self.inter)

    def __call__(self, X, pos, Y=None):
        """Rows of finished queries, keys and values; all four steps in the same rows."""
        Y = self.project(X, Y)
        q, k = self.heads_of(Y)
        lq.lq_qk_norm_rope_fwd(self.qk, q, k, self.wq, self.wk, pos, self.inv_freq, qo=q, ko=k)
        return Y

    def backward(self, X, rows, pos, grad):
        """Gradients of A, B, wq and wk.  rows: project(X); grad: the derivative with respect to the finished rows, overwritten."""
        self._grouped(X)
        q, k = self.heads_of(rows)
        gq, gk = self.heads_of(grad)
        _, _, dwq, dwk = lq.lq_qk_norm_rope_bwd(self.qk, q, k, self.wq, self.wk, pos, self.inv_freq, gq, gk, dq=gq, dk=gk)
        _, dA, dB = lq.lq_adapter_bwd(self.adapters, self.plan, X, self.A, self.B, self.ranks, self.scales, self.inter, grad, work=self.work)
        return dA, dB, dwq, dwk


def layer(dim: int, rank: int, seed: int = 0):
    """A synthetic QKV layer with its branch's factors."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return [torch.randn(s, generator=g, device="cuda") * f for s, f in (((3 * dim, dim), 0.02), ((3 * dim, rank), 1e-3), ((rank, dim), 1e-3))]


def serve(images: int = 2, side: int = 64, dim: int = 1152, heads: int = 16, adapters: int = 3, steps: int = 50) -> float:
    """A batch of images, each with its own adapter or none.  Returns us per call."""
    M = images * side * side
    m = AdaptedQKV(*layer(dim, 32), M, heads, adapters, 32)
    m.B.normal_(std=0.02)
    X = torch.randn(M, dim, device="cuda").bfloat16()
    m.group(torch.arange(images, dtype=torch.int32, device="cuda").repeat_interleave(side * side) - 1)  # the first image has none
    pos, Y = grid_positions(side, side), torch.empty(M, 3 * dim, dtype=torch.bfloat16, device="cuda")
    ev = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
    for i in range(2 * steps):
        if i == steps:
            ev[0].record()
        m(X, pos, Y)
    ev[1].record()
    torch.cuda.synchronize()
    return ev[0].elapsed_time(ev[1]) / steps * 1e3


def train(steps: int = 60, side: int = 16, dim: int = 256, heads: int = 4, rank: int = 8):
    """Two adapters learn two layers that differ from the quantised one by a product of small rank each.  Returns the losses."""
    W, L, R = layer(dim, 32)
    M = 2 * side * side
    m = AdaptedQKV(W, L, R, M, heads, 2, rank)
    ids = torch.arange(2, dtype=torch.int32, device="cuda").repeat_interleave(side * side)
    m.group(ids)
    pos = grid_positions(side, side)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    shift = [torch.randn(3 * dim, rank, generator=g, device="cuda") @ torch.randn(rank, dim, generator=g, device="cuda") * 0.01 for _ in range(2)]
    masters = [m.A.float().requires_grad_(), m.B.float().requires_grad_()]
    opt = torch.optim.Adam(masters, lr=3e-3)
    losses = []
    for _ in range(steps):
        X = torch.randn(M, dim, generator=g, device="cuda").bfloat16()
        target = torch.cat([X[ids == s].float() @ (W + shift[s]).t() for s in range(2)]).bfloat16()
        tq, tk = m.heads_of(target)
        lq.lq_qk_norm_rope_fwd(m.qk, tq, tk, m.wq, m.wk, pos, m.inv_freq, qo=tq, ko=tk)
        rows = m.project(X)
        out = rows.clone()
        q, k = m.heads_of(out)
        lq.lq_qk_norm_rope_fwd(m.qk, q, k, m.wq, m.wk, pos, m.inv_freq, qo=q, ko=k)
        diff = out.float() - target.float()
        losses.append(float((diff * diff).mean()))
        dA, dB, _, _ = m.backward(X, rows, pos, (diff * (2.0 / M)).bfloat16())
        masters[0].grad, masters[1].grad = dA, dB
        opt.step()
        with torch.no_grad():
            m.A.copy_(masters[0])
            m.B.copy_(masters[1])
    return losses


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--train", action="store_true")
    a = ap.parse_args()
    if a.train:
        losses = train()
        print("loss", " ".join(f"{v:.4f}" for v in losses[::10] + losses[-1:]))
    else:
        print(f"2 images of 64 x 64 patches, 1152 wide, 16 heads, adapters of rank 32: {serve():.1f} us")


if __name__ == "__main__":
    main()
