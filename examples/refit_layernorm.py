"""Re-learn a slim layer whose output is normalised over its channels: conv -> layer norm -> ReLU, fitted to a feature map.

The layer-wise regression of ``dr_regress_step`` fits f~(W, b; X) = ReLU(conv(X; W) + b) by SGD.  Here the layer carries a
layer norm between the convolution and the ReLU, and the filters take the orthogonalised update instead of the plain one:

    z = conv(x; W) + b                     dr_conv_slim
    u = layer norm over the channels of z  dr_layernorm            (keeps mean and 1/sqrt(var + eps) of every pixel)
    y = ReLU(u),  L = |y - y_target|^2 / (2 B)
    du = dL/du where y > 0                 dr_relu, dr_regress_grad
    dz, dgamma, dbeta                      dr_layernorm_bwd
    dW                                     dr_conv_wgrad
    W                                      dr_muon_update          (float32 master weights, bfloat16 copy for the next pass)
    gamma, beta                            dr_sgd_update

The convolution's own bias stays at zero: the layer norm's beta takes its place.  Run on a GPU:

    python examples/refit_layernorm.py [--steps 40] [--batch 32] [--size 28] [--cin 64] [--cout 192] [--update muon|sgd]
"""
from __future__ import annotations

import argparse
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import torch  # noqa: E402

import paper_1708_04728_b200 as dr  # noqa: E402

EPS_LN, EPS_NS = 1e-5, 1e-7


def scratch(nbytes):
    """Zero-filled device memory at a 256-byte boundary."""
    t = torch.zeros(nbytes + 256, dtype=torch.uint8, device="cuda")
    return t[(-t.data_ptr()) % 256:][:max(nbytes, 1)]


class Refit:
    """One slim layer with its layer norm, its optimiser state and every buffer of a step: a step allocates nothing."""

    def __init__(self, batch, size, cin, cout, k=3, update="muon", lr=0.02, lr_sgd=0.05, momentum=0.9, decay=0.0, seed=0):
        self.B, self.H, self.cin, self.cout, self.k, self.update = batch, size, cin, cout, k, update
        self.lr, self.lr_sgd, self.momentum, self.decay = lr, lr_sgd, momentum, decay
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        f32 = dict(dtype=torch.float32, device="cuda")
        self.w = torch.randn((cout, k, k, cin), generator=g, device="cuda") * (2.0 / (k * k * cin)) ** 0.5
        self.shadow = self.w.to(torch.bfloat16)
        self.vw, self.dw = torch.zeros_like(self.w), torch.empty_like(self.w)
        self.bias = torch.zeros(cout, **f32)
        self.gamma, self.beta = torch.ones(cout, **f32), torch.zeros(cout, **f32)
        self.v_gamma, self.v_beta = torch.zeros(cout, **f32), torch.zeros(cout, **f32)
        self.dgamma, self.dbeta, self.dsum = (torch.empty(cout, **f32) for _ in range(3))
        self.loss = torch.zeros(1, **f32)
        npix = batch * size * size
        act = lambda: torch.empty((batch, size, size, cout), dtype=torch.bfloat16, device="cuda")
        self.z, self.y, self.du, self.dz = act(), act(), act(), act()
        self.mean, self.rstd = torch.empty(npix, **f32), torch.empty(npix, **f32)
        self.npix = npix
        self.desc = dr.dr_conv_desc(k=k, stride=1, pad=k // 2, Cin=cin, Cout=cout, flags=dr.DR_BIAS)
        self.ws_conv = scratch(dr.dr_conv_workspace_bytes(self.desc, batch, size, size))
        self.ws_wgrad = scratch(dr.dr_conv_wgrad_workspace_bytes(self.desc, batch, size, size))
        self.ws_regress = scratch(dr.dr_regress_workspace_bytes(cout))
        self.ws_ln = scratch(dr.dr_layernorm_bwd_workspace_bytes(npix, cout))
        self.ws_muon = scratch(dr.dr_orthogonalise_workspace_bytes(1, cout, k * k * cin))

    def forward(self, x, stream=None):
        B, H = self.B, self.H
        dr.dr_conv_slim_ws(self.desc, B, H, H, x, self.shadow, self.bias, None, self.z, None, self.ws_conv, self.ws_conv.numel(), stream)
        dr.dr_layernorm(self.npix, self.cout, self.z, 0, self.gamma, self.beta, EPS_LN, self.y, 0, self.mean, self.rstd, 0, stream)
        dr.dr_relu(self.y.numel(), self.y, self.y, stream)
        return self.y

    def gradients(self, x, target, stream=None):
        B, H, C = self.B, self.H, self.cout
        self.forward(x, stream)
        dr.dr_regress_grad(B, H, H, C, self.y, target, True, self.du, self.dsum, self.loss, self.ws_regress, self.ws_regress.numel(), stream)
        dr.dr_layernorm_bwd(self.npix, C, self.du, 0, self.z, 0, self.gamma, self.mean, self.rstd, self.dz, 0, self.dgamma, self.dbeta,
                            self.ws_ln, self.ws_ln.numel(), 0, stream)
        dr.dr_conv_wgrad(self.desc, B, H, H, x, self.dz, self.dw, self.ws_wgrad, self.ws_wgrad.numel(), stream)

    def step(self, x, target, stream=None):
        """One step; self.loss holds the loss before it."""
        self.gradients(x, target, stream)
        if self.update == "muon":
            dr.dr_muon_update(1, self.cout, self.k * self.k * self.cin, self.w, self.vw, self.dw, self.lr, self.momentum, self.decay, True, 5, None,
                              EPS_NS, self.shadow, self.ws_muon, self.ws_muon.numel(), stream)
        else:
            dr.dr_sgd_update(self.w.numel(), self.w, self.vw, self.dw, self.lr, self.momentum, self.decay, self.shadow, stream)
        n = self.B * self.H * self.H / self.B           # the gradients of gamma and beta sum over the pixels of an image
        dr.dr_sgd_update(self.cout, self.gamma, self.v_gamma, self.dgamma, self.lr_sgd / n, self.momentum, 0.0, None, stream)
        dr.dr_sgd_update(self.cout, self.beta, self.v_beta, self.dbeta, self.lr_sgd / n, self.momentum, 0.0, None, stream)


def teacher(batch, size, cin, cout, k=3, seed=1):
    """Inputs, and the feature map of a layer of the same form with filters, gamma and beta of its own."""
    t = Refit(batch, size, cin, cout, k, seed=seed)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + 1)
    t.gamma.copy_(1 + 0.2 * torch.randn(cout, generator=g, device="cuda"))
    t.beta.copy_(0.3 * torch.randn(cout, generator=g, device="cuda"))
    x = torch.randn((batch, size, size, cin), generator=g, device="cuda").to(torch.bfloat16)
    return x, t.forward(x).clone()


def filter_rate(lr, update):
    """The filters' learning rate: the one that was asked for, zero included, or the update's default."""
    return lr if lr is not None else 0.4 if update == "muon" else 0.0005


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=40)
    ap.add_argument("--batch", type=int, default=32)
    ap.add_argument("--size", type=int, default=28)
    ap.add_argument("--cin", type=int, default=64)
    ap.add_argument("--cout", type=int, default=192)
    ap.add_argument("--update", choices=["muon", "sgd"], default="muon")
    ap.add_argument("--lr", type=float, default=None, help="of the filters; default 0.4 (muon), 0.0005 (sgd)")
    a = ap.parse_args()
    x, target = teacher(a.batch, a.size, a.cin, a.cout)
    layer = Refit(a.batch, a.size, a.cin, a.cout, update=a.update, lr=filter_rate(a.lr, a.update))
    for i in range(a.steps):
        layer.step(x, target)
        if i % 5 == 0 or i == a.steps - 1:
            print(f"step {i:3d}  loss {float(layer.loss):.4f}")
    status, info = dr.dr_device_status()
    if status:
        raise SystemExit(f"device status {status} {info}")


if __name__ == "__main__":
    main()
