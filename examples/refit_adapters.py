"""Re-learn one 1 x 1 slim layer for several tasks at once: shared filters, and a low-rank adapter for each task.

A network that has been slimmed once serves many tasks whose features differ a little.  Instead of a copy of the layer for every task, the
filters W stay as they are and each task a gets a pair of thin matrices; images of all tasks run, and are learned, in the same batch:

    x' = dropout(x)                                        dr_dropout           (of the layer's input; p = 0 leaves it out)
    y  = ReLU(x' W^T + bias + scale_a D(x') A_a^T B_a^T)   dr_adapter           (D: dropout in front of the adapter; keeps t = D(x') A_a^T)
    L  = |y - y_target|^2 / (2 B),  dz = dL/d(..) where y > 0   dr_regress_grad
    dx', dA, dB                                            dr_adapter_bwd
    dx = dropout(dx')                                      dr_dropout           (the same mask again, from the same counter)
    A, B                                                   dr_sgd_update, or dr_muon_update for each task's matrices

A counter in device memory moves the masks on with every step, so the whole step can be captured into a CUDA graph.  Run on a GPU:

    python examples/refit_adapters.py [--steps 60] [--images 32] [--size 14] [--cin 256] [--cout 192] [--rank 8] [--tasks 4] [--update sgd|muon]
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

EPS_NS = 1e-7


def scratch(nbytes):
    """Zero-filled device memory at a 256-byte boundary."""
    t = torch.zeros(nbytes + 256, dtype=torch.uint8, device="cuda")
    return t[(-t.data_ptr()) % 256:][:max(nbytes, 1)]


class Tasks:
    """The layer, its tasks' adapters, their optimiser state and every buffer of a step: a step allocates nothing."""

    def __init__(self, images, size, cin, cout, rank=8, tasks=4, p=0.1, p_input=0.0, update="sgd", lr=0.02, momentum=0.9, decay=0.0, seed=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        bf, f32 = dict(dtype=torch.bfloat16, device="cuda"), dict(dtype=torch.float32, device="cuda")
        self.B, self.H, self.M, self.cin, self.cout, self.rank, self.tasks = images, size, images * size * size, cin, cout, rank, tasks
        self.p_input, self.update, self.lr, self.momentum, self.decay, self.seed = p_input, update, lr, momentum, decay, 1000 + seed
        self.w = (torch.randn((cout, cin), generator=g, device="cuda") * (2.0 / cin) ** 0.5).to(torch.bfloat16)
        self.bias = torch.zeros(cout, **f32)
        # an adapter begins as the zero map: B = 0
        self.a = torch.randn((tasks, rank, cin), generator=g, device="cuda") * cin ** -0.5
        self.b = torch.zeros((tasks, cout, rank), **f32)
        self.a16, self.b16 = self.a.to(torch.bfloat16), self.b.to(torch.bfloat16)
        self.va, self.vb, self.da, self.db = (torch.zeros_like(t) for t in (self.a, self.b, self.a, self.b))
        self.scale = torch.full((tasks,), 2.0, **f32)
        # every image is a request of its own: its rows, and its task
        self.row_start = torch.arange(images + 1, dtype=torch.int32, device="cuda") * (size * size)
        self.task = (torch.arange(images, device="cuda") % tasks).to(torch.int32)
        self.step_count = torch.zeros(1, dtype=torch.int64, device="cuda")
        self.xd = torch.empty((self.M, cin), **bf)
        self.y, self.dz = (torch.empty((images, size, size, cout), **bf) for _ in range(2))
        self.dx = torch.empty((self.M, cin), **bf)
        self.t, self.dbias, self.loss = torch.zeros((self.M, rank), **f32), torch.empty(cout, **f32), torch.zeros(1, **f32)
        self.desc = dr.dr_adapter_desc(Cin=cin, Cout=cout, rank=rank, adapters=tasks, flags=dr.DR_BIAS | dr.DR_RELU, drop_p=p, drop_seed=self.seed, drop_offset=0)
        self.ws = scratch(max(dr.dr_adapter_workspace_bytes(self.desc, self.M), dr.dr_adapter_bwd_workspace_bytes(self.desc, self.M)))
        self.ws_regress = scratch(dr.dr_regress_workspace_bytes(cout))
        if update == "muon":
            self.ws_muon = scratch(max(dr.dr_orthogonalise_workspace_bytes(tasks, rank, cin), dr.dr_orthogonalise_workspace_bytes(tasks, cout, rank)))

    def forward(self, x, stream=None):
        """x: [images, size, size, cin] bfloat16; returns y."""
        if self.p_input:
            dr.dr_dropout(self.M, self.cin, x, 0, None, 0, self.xd, 0, self.p_input, self.seed + 1, 0, self.step_count, 0, stream)
            x = self.xd
        dr.dr_adapter(self.desc, self.M, x, 0, self.w, self.bias, self.a16, self.b16, self.scale, self.B, self.row_start, self.task, self.y, 0, self.t,
                      self.step_count, self.ws, self.ws.numel(), stream)
        return self.y

    def gradients(self, x, target, stream=None):
        B, H = self.B, self.H
        self.forward(x, stream)
        dr.dr_regress_grad(B, H, H, self.cout, self.y, target, True, self.dz, self.dbias, self.loss, self.ws_regress, self.ws_regress.numel(), stream)
        dr.dr_adapter_bwd(self.desc, self.M, self.dz, 0, self.xd if self.p_input else x, 0, self.w, self.a16, self.b16, self.scale, B, self.row_start, self.task,
                          self.t, self.dx, 0, self.da, self.db, self.step_count, self.ws, self.ws.numel(), stream)
        if self.p_input:
            dr.dr_dropout(self.M, self.cin, self.dx, 0, None, 0, self.dx, 0, self.p_input, self.seed + 1, 0, self.step_count, 0, stream)

    def step(self, x, target, stream=None):
        """One step; self.loss holds the loss before it."""
        self.gradients(x, target, stream)
        for w, v, g, w16, rows, cols in ((self.a, self.va, self.da, self.a16, self.rank, self.cin), (self.b, self.vb, self.db, self.b16, self.cout, self.rank)):
            if self.update == "muon":
                dr.dr_muon_update(self.tasks, rows, cols, w, v, g, self.lr, self.momentum, self.decay, True, 5, None, EPS_NS, w16, self.ws_muon,
                                  self.ws_muon.numel(), stream)
            else:
                dr.dr_sgd_update(w.numel(), w, v, g, self.lr / (self.H * self.H), self.momentum, self.decay, w16, stream)
        with torch.cuda.stream(stream) if stream is not None else torch.cuda.stream(torch.cuda.current_stream()):
            self.step_count += 1


def teacher(images, size, cin, cout, rank=8, tasks=4, seed=1):
    """Inputs, and the feature maps of a layer of the same form: the same filters, tasks' adapters of their own, nothing dropped."""
    t = Tasks(images, size, cin, cout, rank, tasks, p=0.0, seed=0)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    t.a16 = (torch.randn((tasks, rank, cin), generator=g, device="cuda") * cin ** -0.5).to(torch.bfloat16)
    t.b16 = (0.3 * torch.randn((tasks, cout, rank), generator=g, device="cuda") * rank ** -0.5).to(torch.bfloat16)
    x = torch.randn((images, size, size, cin), generator=g, device="cuda").relu().to(torch.bfloat16)
    return x, t.forward(x).clone()


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--images", type=int, default=32)
    ap.add_argument("--size", type=int, default=14)
    ap.add_argument("--cin", type=int, default=256)
    ap.add_argument("--cout", type=int, default=192)
    ap.add_argument("--rank", type=int, default=8)
    ap.add_argument("--tasks", type=int, default=4)
    ap.add_argument("--drop", type=float, default=0.1, help="in front of the adapters")
    ap.add_argument("--drop-input", type=float, default=0.0, help="of the layer's input")
    ap.add_argument("--update", choices=["sgd", "muon"], default="sgd")
    ap.add_argument("--lr", type=float, default=0.02)
    a = ap.parse_args()
    x, target = teacher(a.images, a.size, a.cin, a.cout, a.rank, a.tasks)
    layer = Tasks(a.images, a.size, a.cin, a.cout, a.rank, a.tasks, a.drop, a.drop_input, a.update, a.lr)
    for i in range(a.steps):
        layer.step(x, target)
        if i % 10 == 0 or i == a.steps - 1:
            print(f"step {i:3d}  loss {float(layer.loss):.4f}")
    status, info = dr.dr_device_status()
    if status:
        raise SystemExit(f"device status {status} {info}")


if __name__ == "__main__":
    main()
