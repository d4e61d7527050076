"""A training step around the exchange: lookups are decompressed, go through a dense tower, and the gradient that comes back
is compressed for the way home.

    python examples/dense_tower.py [--steps 20] [--dtype f32|f16|bf16]

Tower, over the lookups of all tables side by side:

    h1 = relu(x w1' + b1)                      dlc_linear_forward
    h2 = silu(g) * u,  [g | u] = h1 w2'        dlc_gated_forward
    h3 = drop(relu(h2 w3' + b3)) + h1          dlc_linear_forward, dropout and residual in its epilogue
    h4 = drop(h3)                              dlc_dropout
    logit = h4 w4' + b4                        dlc_linear_forward

and the same layers' backward calls.  Masks are made from (seed, step) on the way forward and again on the way back; none is
stored.  Buffers and the workspace are made once.
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
    """The tower's weights, buffers and calls, for a fixed number of samples."""

    def __init__(self, rows, features, hidden=512, dtype="f32", drop=0.1, seed=1):
        code, ty = TYPES[dtype]
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)

        def weight(n, k):
            return (torch.randn((n, k), generator=gen, device="cuda") * k ** -0.5).to(ty)

        def empty(*shape):
            return torch.empty(shape, dtype=ty, device="cuda")

        wide = 2 * hidden
        self.w = [weight(hidden, features), weight(2 * wide, hidden), weight(hidden, wide), weight(1, hidden)]
        self.bias = [torch.zeros(n, dtype=ty, device="cuda") for n in (hidden, 0, hidden, 1)]
        self.dw = [torch.empty_like(w) for w in self.w]
        self.dbias = [torch.empty_like(v) for v in self.bias]
        # what forward leaves for backward, and the gradients on their way
        self.h1, self.z1 = empty(rows, hidden), empty(rows, hidden)
        self.h2, self.gu = empty(rows, wide), empty(rows, 2 * wide)
        self.h3, self.z3, self.h4 = empty(rows, hidden), empty(rows, hidden), empty(rows, hidden)
        self.logit = empty(rows, 1)
        self.d_logit, self.d3, self.d2 = empty(rows, 1), empty(rows, hidden), empty(rows, wide)
        self.d1, self.dx = empty(rows, hidden), empty(rows, features)
        self.layers = [b.make_dense_config(code, rows, features, hidden, act=b.ACT_RELU),
                       b.make_dense_config(code, rows, hidden, wide, act=b.ACT_SILU),
                       b.make_dense_config(code, rows, wide, hidden, act=b.ACT_RELU, dropout_p=drop, seed=seed),
                       b.make_dense_config(code, rows, hidden, 1)]
        self.head = b.make_dropout_config(code, rows, hidden, drop, seed=seed + 1)
        need = max(max(f(c), f(c, True)) for f, c in
                   zip((b.dlc_linear_workspace_bytes, b.dlc_gated_workspace_bytes) + 2 * (b.dlc_linear_workspace_bytes,), self.layers))
        self.work = torch.empty(need, dtype=torch.uint8, device="cuda")

    def forward(self, x, step):
        c1, c2, c3, c4 = self.layers
        c3.offset = self.head.offset = step   # other masks in every step
        b.dlc_linear_forward(c1, x, self.w[0], self.bias[0], None, self.h1, self.z1, self.work)
        b.dlc_gated_forward(c2, self.h1, self.w[1], None, self.h2, self.gu, self.work)
        b.dlc_linear_forward(c3, self.h2, self.w[2], self.bias[2], self.h1, self.h3, self.z3, self.work)
        b.dlc_dropout(self.head, self.h3, None, self.h4)
        b.dlc_linear_forward(c4, self.h4, self.w[3], self.bias[3], None, self.logit, None, self.work)
        return self.logit

    def backward(self, x, d_logit):
        """-> the gradient of x; the weights' gradients are in dw and dbias"""
        c1, c2, c3, c4 = self.layers
        b.dlc_linear_backward(c4, self.h4, self.w[3], None, d_logit, self.d3, self.dw[3], self.dbias[3], self.work)
        b.dlc_dropout(self.head, self.d3, None, self.d3)                      # dropout's gradient is the same call
        b.dlc_linear_backward(c3, self.h2, self.w[2], self.z3, self.d3, self.d2, self.dw[2], self.dbias[2], self.work)
        b.dlc_gated_backward(c2, self.h1, self.w[1], self.gu, self.d2, self.d1, self.dw[1], None, self.work)
        self.d1 += self.d3                                                    # h1 also went around as the residual
        b.dlc_linear_backward(c1, x, self.w[0], self.z1, self.d1, self.dx, self.dw[0], self.dbias[0], self.work)
        return self.dx

    def update(self, rate):
        for p, g in zip(self.w + self.bias, self.dw + self.dbias):
            p -= rate * g


def exchange(ctx, payload, container, sizes, received):
    """What a payload goes through on its way to the other side; -> compression ratio"""
    assert ctx.compress(payload, container, sizes) == b.OK and ctx.sync_status() == b.OK
    total = int(sizes[0].item())
    assert ctx.decompress(container, total, received) == b.OK and ctx.sync_status() == b.OK
    return payload.numel() * payload.element_size() / total


def run(steps=20, dtype="f32", tables=26, batch=4096, dim=64, rate=0.05, report=print):
    """-> the losses"""
    ty = TYPES[dtype][1]
    lookups = torch.from_numpy(W.workload2(T=tables, B=batch, D=dim).payload).cuda() * 20.0
    ctx = b.Context(b.make_config(b.F32, tables, batch, dim))
    back = b.Context(b.make_config(b.F32, tables, batch, dim))
    container = torch.empty(b.dlc_compress_bound(ctx.cfg), dtype=torch.uint8, device="cuda")
    sizes = torch.zeros(1 + tables, dtype=torch.int64, device="cuda")
    received, returned = torch.empty_like(lookups), torch.empty_like(lookups)
    tower = Tower(batch, tables * dim, dtype=dtype)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(7)
    truth = torch.randn((tables * dim,), generator=gen, device="cuda")
    label = (lookups.transpose(0, 1).reshape(batch, -1) @ truth > 0).float()[:, None]
    losses = []
    for step in range(steps):
        ctx.set_error_bounds(eb=0.01)
        there = exchange(ctx, lookups, container, sizes, received)
        x = received.transpose(0, 1).reshape(batch, tables * dim).to(ty)   # the tables' rows side by side
        logit = tower.forward(x, step).float()
        losses.append(float(torch.nn.functional.binary_cross_entropy_with_logits(logit, label)))
        tower.d_logit.copy_((torch.sigmoid(logit) - label) / batch)
        dx = tower.backward(x, tower.d_logit)
        grad = dx.float().reshape(batch, tables, dim).transpose(0, 1).contiguous()
        back.set_error_bounds(eb=float(grad.abs().max()) * 0.01)
        home = exchange(back, grad, container, sizes, returned)
        tower.update(rate)
        report(f"step {step}: loss {losses[-1]:.4f}, lookups compressed {there:.1f} times, their gradient {home:.1f} times")
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--dtype", choices=sorted(TYPES), default="f32")
    a = ap.parse_args()
    run(a.steps, a.dtype)
