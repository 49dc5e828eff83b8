"""A model of one interaction layer trained by gradient descent with the library's operators, as a user's program would call them:

    element embedding -> radial network (dense layers on the edges) -> channelwise tensor product -> symmetric contraction
    -> readout (dense layers on the invariant channels) -> energies; their gradients in reverse; clipping by the global norm; update.

With `self_connection` the embedded features reach the readout past the interaction too, through a matrix of their element.  With `orthogonalised` the
matrices between features (those of the radial network, of the self connection, of the readout's first layer) take the orthogonalised update; the table, the
contraction's weights, biases and the last layer take gradient descent, as all parameters do without it.

Synthetic structures, random targets.  `python -m paper_2504_10700_amd.training_step` trains for some steps and prints the loss, the gradient's norm and
the time of a step.  Buffers and workspaces are allocated once; a step enqueues its calls on the current stream and never synchronises.
"""
from __future__ import annotations

import argparse
import time

import numpy as np
import torch

from . import binding as sc
from . import dl_binding as dl
from . import ee_binding as ee
from . import gc_binding as gc
from . import gp_binding as gp
from . import ou_binding as ou
from . import tp_binding as tp
from .workloads import TPWorkload, graph_indices, make_tp_graph

BASIS, HIDDEN, READOUT = 8, 64, 16      # radial basis functions, width of the radial network, of the readout


class Dense:
    """A dense layer with the buffers of its two passes.  Parameters W, b; gradients dW, db."""

    def __init__(self, rows: int, k_in: int, k_out: int, activation: int, row_type, bias: bool, make, kind: int):
        self.rows, self.activation = rows, activation
        self.cfg = dl.make_config(k_in, k_out, activation, kind)
        self.W = make(k_in, k_out, scale=k_in ** -0.5)
        self.b = make(k_out, scale=0.1) if bias else None
        self.dW = torch.empty_like(self.W)
        self.db = torch.empty_like(self.b) if bias else None
        self.Y = torch.empty(rows, k_out, dtype=row_type, device="cuda")
        self.Z = torch.empty_like(self.Y) if activation != dl.DL_NONE else None
        self.dX = torch.empty(rows, k_in, dtype=row_type, device="cuda")
        self.workspace_bytes = dl.dl_workspace_bytes(self.cfg, rows)

    def forward(self, X, residual=None):
        self.X = X
        dl.dl_forward(self.cfg, self.rows, X, self.W, self.b, residual, self.Y, self.Z)
        return self.Y

    def backward(self, dY, workspace, want_dx=True):
        dX = self.dX if want_dx else None
        dl.dl_backward(self.cfg, self.rows, self.X, self.W, self.Z, dY, dX, self.dW, self.db, workspace, workspace.numel())
        return dX


class Model:
    def __init__(self, num_atoms: int, mean_degree: int = 20, channels: int = 128, elements: int = 89, l_Y: int = 3, dtype: int = sc.SC_F32,
                 max_norm: float = 10.0, learning_rate: float = 1e-2, seed: int = 7, self_connection: bool = False, orthogonalised: bool = False,
                 matrix_rate: float = 1e-3):
        wl = TPWorkload("training_step", num_atoms, mean_degree, channels, l_Y, 0, l_Y, "f64" if dtype == sc.SC_F64 else "f32", seed)
        rng = np.random.default_rng(seed)
        sender, receiver = make_tp_graph(wl, rng)
        row_ptr, send_ptr, send_edge = graph_indices(sender, receiver, num_atoms)
        device = lambda a: torch.tensor(a, device="cuda")  # noqa: E731
        self.sender, self.row_ptr, self.send_ptr, self.send_edge = (device(a) for a in (sender, row_ptr, send_ptr, send_edge))
        self.z = device(rng.integers(0, min(elements, 6), num_atoms).astype(np.int32))
        self.n, self.edges, self.learning_rate = num_atoms, int(sender.size), learning_rate
        real = torch.float64 if dtype == sc.SC_F64 else torch.float32
        g = torch.Generator().manual_seed(seed)
        new = lambda *shape, scale=1.0: (torch.randn(*shape, generator=g, dtype=torch.float64) * scale).to(real).cuda()  # noqa: E731
        empty = lambda *shape: torch.empty(*shape, dtype=real, device="cuda")  # noqa: E731

        # inputs of a batch: radial basis and spherical harmonics of the edges, targets of the structures (ten atoms each)
        self.basis, self.Y = new(self.edges, BASIS), new(self.edges, wl.n_Y)
        self.structure = torch.arange(num_atoms, device="cuda") // 10
        self.target = new(int(self.structure[-1]) + 1)

        self.tp = tp.tp_plan_create(channels, l_Y, 0, l_Y, dtype)
        self.sc = sc.sc_plan_create(channels, l_Y, 3, elements, [(0, 1)], dtype)
        tp_paths, sc_paths = tp.tp_plan_info(self.tp).num_paths, sc.sc_plan_info(self.sc).num_paths
        self.embedding = ee.make_config(elements, channels, 1.0, dtype)
        self.T, self.W_sc = new(elements, channels), new(elements, sc_paths, channels, scale=0.3)
        dense = lambda rows, k_in, k_out, act, bias=True: Dense(rows, k_in, k_out, act, real, bias, new, dtype)  # noqa: E731
        self.radial = [dense(self.edges, BASIS, HIDDEN, dl.DL_SILU), dense(self.edges, HIDDEN, HIDDEN, dl.DL_SILU),
                       dense(self.edges, HIDDEN, HIDDEN, dl.DL_SILU), dense(self.edges, HIDDEN, tp_paths * channels, dl.DL_NONE, False)]
        self.radial[-1].W.mul_(mean_degree ** -0.5)
        self.readout = [dense(num_atoms, channels, READOUT, dl.DL_SILU), dense(num_atoms, READOUT, 1, dl.DL_NONE)]

        self.h, self.dh = empty(num_atoms, channels), empty(num_atoms, channels)
        self.A, self.dA = empty(num_atoms, channels, wl.n_out), empty(num_atoms, channels, wl.n_out)
        self.B = empty(num_atoms, channels)
        self.dR, self.dY = empty(self.edges, tp_paths * channels), empty(self.edges, wl.n_Y)
        self.dT, self.dW_sc = torch.empty_like(self.T), torch.empty_like(self.W_sc)
        layers = self.radial + self.readout
        self.parameters = [self.T, self.W_sc] + [p for x in layers for p in (x.W, x.b) if p is not None]
        self.gradients = [self.dT, self.dW_sc] + [p for x in layers for p in (x.dW, x.db) if p is not None]
        needed = 0
        self.connected = self_connection
        if self_connection:
            self.connection = gp.make_config(elements, channels, channels, 1, dtype)
            self.W_own = new(elements, channels, channels, scale=channels ** -0.5)
            self.dW_own, self.B_own, self.dh_own = torch.empty_like(self.W_own), torch.empty_like(self.B), torch.empty_like(self.h)
            self.parameters.append(self.W_own)
            self.gradients.append(self.dW_own)
            # the order of the atoms by element depends on z alone: made once for the batch
            self.grouping = torch.empty(max(gp.gp_grouping_bytes(self.connection, num_atoms), 256), dtype=torch.uint8, device="cuda")
            gp.gp_group(self.connection, num_atoms, self.z, self.grouping, self.grouping.numel())
            needed = gp.gp_workspace_bytes(self.connection, num_atoms)
        self.orthogonalised = orthogonalised
        self.descended = (self.parameters, self.gradients)
        if orthogonalised:
            pairs = [(x.W, x.dW) for x in self.radial + self.readout[:-1]] + ([(self.W_own, self.dW_own)] if self_connection else [])
            matrices, of_matrices = [list(x) for x in zip(*pairs)]
            self.momentum = [torch.zeros_like(w) for w in matrices]
            self.update = ou.make_config(matrix_rate)
            self.updated = ou.make_tensors(of_matrices, self.momentum, matrices, scale=[max(1.0, w.shape[-1] / w.shape[-2]) ** 0.5 for w in matrices])
            needed = max(needed, ou.ou_workspace_bytes(self.update, self.updated))
            others = [(p, d) for p, d in zip(self.parameters, self.gradients) if all(p is not w for w in matrices)]
            self.descended = tuple(list(x) for x in zip(*others))
        self.clip = gc.make_config(max_norm, 1e-6, dtype)
        self.clipped = gc.make_tensors(self.gradients, self.gradients)      # in place
        self.norm = empty(2)                                                # and the coefficient
        # the contraction's workspace carries the grouping from its forward to its backward; the others share one
        self.sc_workspace = torch.empty(sc.sc_workspace_bytes(self.sc, num_atoms), dtype=torch.uint8, device="cuda")
        self.workspace = torch.empty(max([needed] + [x.workspace_bytes for x in layers] + [
            ee.ee_workspace_bytes(self.embedding, num_atoms), tp.tp_workspace_bytes(self.tp, self.edges), gc.gc_workspace_bytes(self.clip, self.clipped)]),
            dtype=torch.uint8, device="cuda")

    def energies(self):
        """Forward: an energy per atom."""
        ee.ee_forward(self.embedding, self.n, self.z, self.T, self.h)
        x = self.radial[0].forward(self.basis)
        x = self.radial[1].forward(x, residual=x)
        x = self.radial[2].forward(x, residual=x)
        self.R = self.radial[3].forward(x)
        tp.tp_forward(self.tp, self.n, self.n, self.edges, self.Y, self.h, self.R, self.sender, self.row_ptr, self.A)
        sc.sc_forward(self.sc, self.n, self.A, self.z, self.W_sc, self.B, self.sc_workspace, self.sc_workspace.numel())
        features = self.B
        if self.connected:
            features = self.B_own
            gp.gp_forward(self.connection, self.n, self.z, self.grouping, self.h, self.W_own, self.B, features, self.workspace, self.workspace.numel())
        return self.readout[1].forward(self.readout[0].forward(features))

    def loss(self):
        energy = torch.zeros_like(self.target).index_add_(0, self.structure, self.energies()[:, 0])
        self.difference = energy - self.target
        return 0.5 * (self.difference ** 2).mean()

    def backward(self):
        """Gradients of the loss for all parameters."""
        ws = self.workspace
        dE = (self.difference / self.target.numel())[self.structure][:, None].contiguous()
        dB = self.readout[0].backward(self.readout[1].backward(dE, ws), ws)
        sc.sc_backward(self.sc, self.n, self.A, self.z, self.W_sc, dB, self.dA, self.dW_sc, self.sc_workspace, self.sc_workspace.numel(),
                       sc.SC_REUSE_GROUPING | sc.SC_REUSE_WEIGHTS)
        tp.tp_backward(self.tp, self.n, self.n, self.edges, self.Y, self.h, self.R, self.sender, self.row_ptr, self.send_ptr, self.send_edge, self.dA,
                       self.dY, self.dh, self.dR, ws, ws.numel())
        if self.connected:
            gp.gp_backward(self.connection, self.n, self.z, self.grouping, self.h, self.W_own, dB, self.dh_own, self.dW_own, ws, ws.numel())
            self.dh.add_(self.dh_own)
        ee.ee_backward(self.embedding, self.n, self.z, self.dh, self.dT, ws, ws.numel())
        dx = self.radial[3].backward(self.dR, ws)
        dx = self.radial[2].backward(dx, ws).add_(dx)        # the residual's gradient is the upstream one
        dx = self.radial[1].backward(dx, ws).add_(dx)
        self.radial[0].backward(dx, ws, want_dx=False)

    def step(self):
        """One step of the optimizer; the loss before it, on the device."""
        loss = self.loss()
        self.backward()
        gc.gc_clip(self.clip, self.clipped, self.norm, self.workspace, self.workspace.numel())
        torch._foreach_add_(*self.descended, alpha=-self.learning_rate)
        if self.orthogonalised:
            ou.ou_step(self.update, self.updated, self.workspace, self.workspace.numel())
        return loss


def main() -> None:
    parser = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    parser.add_argument("--atoms", type=int, default=10_000)
    parser.add_argument("--degree", type=int, default=20)
    parser.add_argument("--channels", type=int, default=128)
    parser.add_argument("--steps", type=int, default=20)
    parser.add_argument("--self-connection", action="store_true", help="the embedded features reach the readout through a matrix of their element")
    parser.add_argument("--orthogonalised", action="store_true", help="matrices take the orthogonalised update")
    args = parser.parse_args()
    model = Model(args.atoms, args.degree, args.channels, self_connection=args.self_connection, orthogonalised=args.orthogonalised)
    print(f"{model.n} atoms, {model.edges} edges, {sum(p.numel() for p in model.parameters)} parameters", flush=True)
    for i in range(args.steps):
        torch.cuda.synchronize()
        start = time.perf_counter()
        loss = model.step()
        torch.cuda.synchronize()
        print(f"step {i}: loss {loss.item():.5f}, gradient norm {model.norm[0].item():.4f}, {1e3 * (time.perf_counter() - start):.2f} ms", flush=True)


if __name__ == "__main__":
    main()
