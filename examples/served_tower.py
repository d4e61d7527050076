"""A residual tower behind decompressed lookups: trained with norms and clipped gradients, then served with 4-bit weights.

    python examples/served_tower.py [--steps 20] [--dtype f32|f16|bf16]

    h = x w0' + b0                                dlc_linear_forward
    n1 = norm(h) g1                               dlc_norm_forward
    a = silu(n1 w1' + b1)                         dlc_linear_forward
    r = a w2' + b2                                dlc_linear_forward
    n2 = norm(r + h) g2                           dlc_norm_forward, which adds the residual
    logit = n2 w3' + b3                           dlc_linear_forward

Training adds the layers' backward calls, dlc_gradient_norm and dlc_gradient_clip over all gradients, and the update.  Serving
takes the weights as E2M1 with a scale for 32 columns, made once (dlc_mx_quantize); rows go into the products as E4M3, from
dlc_mx_quantize or straight from dlc_norm_forward (dlc_mx_linear_forward).  Buffers and workspaces are made once.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import dlc_workloads as W  # noqa: E402
from paper_2407_04272_amd import binding as b  # noqa: E402

TYPES = {"f32": (b.F32, torch.float32), "f16": (b.F16, torch.float16), "bf16": (b.BF16, torch.bfloat16)}


class Tower:
    """Weights, gradients, buffers and calls for a fixed number of samples."""

    def __init__(self, rows, features, hidden=512, wide=1024, dtype="f32", seed=1):
        self.code, self.type = TYPES[dtype]
        self.rows = rows
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        self.sizes = [(hidden, features), (wide, hidden), (hidden, wide), (1, hidden)]
        self.w = [(torch.randn(s, generator=gen, device="cuda") * s[1] ** -0.5).to(self.type) for s in self.sizes]
        self.bias = [self.empty(s[0]).zero_() for s in self.sizes]
        self.g = [self.empty(hidden).fill_(1) for _ in range(2)]
        self.dw, self.dbias, self.dg = ([torch.empty_like(v) for v in p] for p in (self.w, self.bias, self.g))
        self.gradients = b.GradientList(self.dw + self.dbias + self.dg)
        acts = [b.ACT_NONE, b.ACT_SILU, b.ACT_NONE, b.ACT_NONE]
        self.layers = [b.make_dense_config(self.code, rows, k, n, act=a) for (n, k), a in zip(self.sizes, acts)]
        self.norm = b.make_norm_config(self.code, rows, hidden, eps=1e-5)
        # what forward leaves for backward, and the gradients on their way
        self.h, self.n1, self.r, self.s, self.n2 = (self.empty(rows, hidden) for _ in range(5))
        self.z, self.a, self.da = (self.empty(rows, wide) for _ in range(3))
        self.logit, self.d_logit = self.empty(rows, 1), self.empty(rows, 1)
        self.dn, self.ds, self.dx = self.empty(rows, hidden), self.empty(rows, hidden), self.empty(rows, features)
        need = [f(c) for c in self.layers for f in (b.dlc_linear_workspace_bytes, lambda c: b.dlc_linear_workspace_bytes(c, True))]
        need += [b.dlc_norm_workspace_bytes(self.norm), b.dlc_gradient_workspace_bytes(self.gradients)]
        self.work = torch.empty(max(need), dtype=torch.uint8, device="cuda")
        self.sum, self.length = self.empty(1, dtype=torch.float64), self.empty(1, dtype=torch.float32)

    def empty(self, *shape, dtype=None):
        return torch.empty(shape, dtype=dtype or self.type, device="cuda")

    def forward(self, x):
        c, w, bias = self.layers, self.w, self.bias
        b.dlc_linear_forward(c[0], x, w[0], bias[0], None, self.h, None, self.work)
        b.dlc_norm_forward(self.norm, self.h, None, self.g[0], None, self.n1)
        b.dlc_linear_forward(c[1], self.n1, w[1], bias[1], None, self.a, self.z, self.work)
        b.dlc_linear_forward(c[2], self.a, w[2], bias[2], None, self.r, None, self.work)
        b.dlc_norm_forward(self.norm, self.r, self.h, self.g[1], self.s, self.n2)
        b.dlc_linear_forward(c[3], self.n2, w[3], bias[3], None, self.logit, None, self.work)
        return self.logit

    def backward(self, x, d_logit):
        """-> the gradient of x; the parameters' are in dw, dbias and dg"""
        c, w = self.layers, self.w
        b.dlc_linear_backward(c[3], self.n2, w[3], None, d_logit, self.dn, self.dw[3], self.dbias[3], self.work)
        b.dlc_norm_backward(self.norm, self.s, self.g[1], self.dn, None, self.ds, self.dg[1], self.work)
        b.dlc_linear_backward(c[2], self.a, w[2], None, self.ds, self.da, self.dw[2], self.dbias[2], self.work)
        b.dlc_linear_backward(c[1], self.n1, w[1], self.z, self.da, self.dn, self.dw[1], self.dbias[1], self.work)
        # h went into the first norm and around it: the gradient along the residual is added in the norm's own pass
        b.dlc_norm_backward(self.norm, self.h, self.g[0], self.dn, self.ds, self.dn, self.dg[0], self.work)
        b.dlc_linear_backward(c[0], x, w[0], None, self.dn, self.dx, self.dw[0], self.dbias[0], self.work)
        return self.dx

    def update(self, rate, max_norm):
        b.dlc_gradient_norm(self.gradients, self.sum, self.work)
        b.dlc_gradient_clip(self.gradients, self.sum, max_norm, self.length)
        for p, d in zip(self.w + self.bias + self.g, self.gradients.tensors):
            p -= rate * d


class Served:
    """The same tower with 4-bit weights and 8-bit rows in the products."""

    def __init__(self, tower, rows):
        self.t, code, empty = tower, tower.code, tower.empty
        self.w = []
        for w in tower.w:
            cfg = b.make_mx_config(code, b.MX_E2M1, *w.shape)
            q, s = self.buffers(cfg)
            b.dlc_mx_quantize(cfg, w, q, s)
            self.w.append((q, s))
        acts = [b.ACT_NONE, b.ACT_SILU, b.ACT_NONE, b.ACT_NONE]
        self.layers = [b.make_mx_linear_config(code, b.MX_E4M3, rows, k, n, act=a) for (n, k), a in zip(tower.sizes, acts)]
        self.rows_in = [b.make_mx_config(code, b.MX_E4M3, rows, k) for _, k in tower.sizes]
        self.x = [self.buffers(c) for c in self.rows_in]
        hidden, wide = tower.sizes[0][0], tower.sizes[1][0]
        self.norm = b.make_norm_config(code, rows, hidden, eps=1e-5)
        self.h, self.a, self.r, self.logit = empty(rows, hidden), empty(rows, wide), empty(rows, hidden), empty(rows, 1)
        self.work = torch.empty(max(b.dlc_mx_linear_workspace_bytes(c) for c in self.layers), dtype=torch.uint8, device="cuda")

    @staticmethod
    def buffers(cfg):
        return tuple(torch.empty(s, dtype=torch.uint8, device="cuda") for s in (b.dlc_mx_data_shape(cfg), b.dlc_mx_scale_shape(cfg)))

    def layer(self, i, y):
        b.dlc_mx_linear_forward(self.layers[i], *self.x[i], *self.w[i], self.t.bias[i], None, y, self.work)

    def forward(self, x):
        b.dlc_mx_quantize(self.rows_in[0], x, *self.x[0])
        self.layer(0, self.h)
        b.dlc_norm_forward(self.norm, self.h, None, self.t.g[0], None, None, *self.x[1])
        self.layer(1, self.a)
        b.dlc_mx_quantize(self.rows_in[2], self.a, *self.x[2])
        self.layer(2, self.r)
        b.dlc_norm_forward(self.norm, self.r, self.h, self.t.g[1], None, None, *self.x[3])
        self.layer(3, self.logit)
        return self.logit


def run(steps=20, dtype="f32", tables=26, batch=4096, dim=64, rate=0.5, max_norm=1.0, report=print):
    """-> the losses, and the share of samples that the served tower decides as the trained one does"""
    ty = TYPES[dtype][1]
    lookups = torch.from_numpy(W.workload2(T=tables, B=batch, D=dim).payload).cuda() * 20.0
    x = lookups.transpose(0, 1).reshape(batch, tables * dim).to(ty)     # the tables' rows side by side
    gen = torch.Generator(device="cuda")
    gen.manual_seed(7)
    truth = torch.randn((tables * dim,), generator=gen, device="cuda")
    label = (x.float() @ truth > 0).float()[:, None]
    tower = Tower(batch, tables * dim, dtype=dtype)
    losses = []
    for step in range(steps):
        logit = tower.forward(x).float()
        losses.append(float(torch.nn.functional.binary_cross_entropy_with_logits(logit, label)))
        tower.d_logit.copy_((torch.sigmoid(logit) - label) / batch)
        tower.backward(x, tower.d_logit)
        tower.update(rate, max_norm)
        report(f"step {step}: loss {losses[-1]:.4f}, the gradients' norm {float(tower.length):.3f}")
    trained = tower.forward(x)
    served = Served(tower, batch).forward(x)
    same = float(((trained > 0) == (served > 0)).float().mean())
    report(f"served with 4-bit weights: {100 * same:.1f} % decided alike")
    return losses, same


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--dtype", choices=sorted(TYPES), default="f32")
    a = ap.parse_args()
    run(a.steps, a.dtype)
