"""A preconditioned layer trained and answering with the library's operators:

    python -m paper_2509_07103_amd.preconditioned [--steps 60] [--batch 2048] [--n-in 64] [--n-out 64] [--grid 9]

    y = gamma lmKAN(x) + Linear(ReLU(x))                      (App. E, ReLU first)

Training: forward and backward of the layer, then ``lmkan_muon_step`` on the table, node by node as a batch of
(G+1)^2 matrices of pairs x outputs, and on the linear term's weights.  Answering: the linear term's weights to
8 bits once (``lmkan_quantize_rows``), then per batch ``lmkan_forward`` and ``lmkan_linear_i8``, which scales the
rows on the way and adds the term to gamma times the layer's output in place.  (With an odd grid the linear term
does not fold into the table exactly.)
"""
from __future__ import annotations

import argparse

import torch

from .binding import (LayerDesc, LinearDesc, MatrixDesc, MuonParams, lmkan_backward, lmkan_forward, lmkan_linear_i8,
                      lmkan_muon_step, lmkan_quantize_rows)


class PreconditionedLayer:
    """Table [G+1][G+1][pairs][n_out], weights [n_out][n_in], their momenta, and the weights' codes once they answer."""

    def __init__(self, n_in: int, n_out: int, grid: int, gamma: float, device, seed: int = 0):
        g = torch.Generator(device="cpu").manual_seed(seed)
        self.layer, self.gamma = LayerDesc(n_in, n_out, grid), gamma
        self.table = torch.zeros(self.layer.coef_shape(), device=device)
        self.weight = (torch.randn((n_out, n_in), generator=g) / n_in ** 0.5).to(device)
        self.nodes = MatrixDesc((grid + 1) ** 2, n_in // 2, n_out)
        self.dense = MatrixDesc(1, n_out, n_in)
        self.linear = LinearDesc(n_in, n_out, relu=True)
        self.momenta = torch.zeros_like(self.table), torch.zeros_like(self.weight)
        self.codes = self.scale = None

    def train_step(self, x: torch.Tensor, target: torch.Tensor, muon: MuonParams) -> torch.Tensor:
        """One step on the mean square error, which is returned."""
        rectified = torch.relu(x)
        off = lmkan_forward(self.layer, x, self.table).mul_(self.gamma).addmm_(rectified, self.weight.t()).sub_(target)
        grad_y = off * (2.0 / off.numel())
        grad_weight = grad_y.t().contiguous() @ rectified
        _, grad_table = lmkan_backward(self.layer, x, self.table, grad_y.mul_(self.gamma), need_grad_x=False)
        n, d = self.nodes.shape(), self.dense.shape()
        lmkan_muon_step(self.nodes, muon, grad_table.view(n), self.momenta[0].view(n), self.table.view(n))
        lmkan_muon_step(self.dense, muon, grad_weight.view(d), self.momenta[1].view(d), self.weight.view(d))
        return off.square().mean()

    def freeze(self) -> None:
        self.codes, self.scale = lmkan_quantize_rows(self.weight)

    def answer(self, x: torch.Tensor) -> torch.Tensor:
        y = lmkan_forward(self.layer, x, self.table)
        return lmkan_linear_i8(self.linear, x, self.codes, self.scale, beta=self.gamma, y=y)

    def answer_in_float(self, x: torch.Tensor) -> torch.Tensor:
        return self.gamma * lmkan_forward(self.layer, x, self.table) + torch.relu(x) @ self.weight.t()


def run(steps: int = 60, batch: int = 2048, n_in: int = 64, n_out: int = 64, grid: int = 9, device="cuda:0"):
    """Trains on a fixed random function; returns (losses, relative difference of the 8-bit answer)."""
    g = torch.Generator(device="cpu").manual_seed(1)
    mix = (torch.randn((n_in, n_out), generator=g) / n_in ** 0.5).to(device)
    model = PreconditionedLayer(n_in, n_out, grid, 0.3, device)
    losses = []
    for step in range(steps):
        x = torch.randn((batch, n_in), generator=g).to(device)
        muon = MuonParams(lr=0.02 * (1.0 - step / steps), momentum=0.9)
        losses.append(float(model.train_step(x, torch.tanh(x @ mix), muon)))
    model.freeze()
    x = torch.randn((batch, n_in), generator=g).to(device)
    want = model.answer_in_float(x)
    return losses, float((model.answer(x) - want).norm() / want.norm())


def main() -> None:
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("steps", 60), ("batch", 2048), ("n-in", 64), ("n-out", 64), ("grid", 9)):
        p.add_argument(f"--{name}", type=int, default=value)
    a = p.parse_args()
    losses, off = run(a.steps, a.batch, a.n_in, a.n_out, a.grid)
    for k in range(0, len(losses), max(1, len(losses) // 10)):
        print(f"step {k:4d}  loss {losses[k]:.5f}")
    print(f"last step  loss {losses[-1]:.5f}; answer with 8-bit weights and rows: {off:.2%} off")


if __name__ == "__main__":
    main()
