"""A preconditioned layer trained and answering with the library's operators:

    python -m paper_2509_07103_amd.preconditioned [--steps 60] [--batch 2048] [--n-in 64] [--n-out 64] [--grid 9] [--norm]

    y = gamma lmKAN(x) + Linear(ReLU(x))                      (App. E, ReLU first)

Training: forward and backward of the layer, then ``lmkan_muon_step`` on the table, node by node as a batch of
(G+1)^2 matrices of pairs x outputs, and on the linear term's weights.  Answering: the linear term's weights to
8 bits once (``lmkan_quantize_rows``), then per batch ``lmkan_forward`` and ``lmkan_linear_i8``, which scales the
rows on the way and adds the term to gamma times the layer's output in place.  (With an odd grid the linear term
does not fold into the table exactly.)

With ``--norm`` the layer is a normalised one, z = LayerNorm(x), y = gamma lmKAN(z) + Linear(ReLU(z)).  Between its passes
only the 8-bit checkpoint of z that ``lmkan_layer_norm`` makes on the way is kept; all gradients come from it.  It answers
requests that each have a low-rank adapter of the linear term (``lmkan_adapters_add``).
"""
from __future__ import annotations

import argparse

import torch

from .binding import (AdapterDesc, LayerDesc, LinearDesc, MatrixDesc, MuonParams, NormDesc, lmkan_adapters_add, lmkan_backward,
                      lmkan_forward, lmkan_layer_norm, lmkan_layer_norm_backward, lmkan_linear_grad, lmkan_linear_i8,
                      lmkan_muon_step, lmkan_quantize_rows, lmkan_restore_rows)


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


class NormalisedLayer(PreconditionedLayer):
    """The same behind a layer norm (without an affine map of its own: table and weights take any).  What is kept for the
    backward pass is a byte for every element of z and 8 for every row."""

    def __init__(self, n_in: int, n_out: int, grid: int, gamma: float, device, seed: int = 0):
        super().__init__(n_in, n_out, grid, gamma, device, seed)
        self.norm = NormDesc(n_in)

    def forward(self, x: torch.Tensor):
        """(y, what the backward pass needs)."""
        z, stats, kept = lmkan_layer_norm(self.norm, x, keep=True)
        y = lmkan_forward(self.layer, z, self.table).mul_(self.gamma).addmm_(torch.relu(z), self.weight.t())
        return y, (stats, kept)

    def gradients(self, saved, grad_y: torch.Tensor):
        """(grad_x, grad_table, grad_weight)."""
        stats, kept = saved
        z = lmkan_restore_rows(*kept)
        grad_weight, _ = lmkan_linear_grad(self.linear, *kept, grad_y, need_grad_bias=False)
        grad_z, grad_table = lmkan_backward(self.layer, z, self.table, self.gamma * grad_y)
        grad_z.add_((grad_y @ self.weight).mul_(z > 0))
        grad_x, _, _ = lmkan_layer_norm_backward(self.norm, grad_z, stats, kept=kept, need_grad_weight=False, need_grad_bias=False)
        return grad_x, grad_table, grad_weight

    def train_step(self, x: torch.Tensor, target: torch.Tensor, muon: MuonParams) -> torch.Tensor:
        y, saved = self.forward(x)
        off = y.sub_(target)
        _, grad_table, grad_weight = self.gradients(saved, off * (2.0 / off.numel()))
        n, d = self.nodes.shape(), self.dense.shape()
        lmkan_muon_step(self.nodes, muon, grad_table.view(n), self.momenta[0].view(n), self.table.view(n))
        lmkan_muon_step(self.dense, muon, grad_weight.view(d), self.momenta[1].view(d), self.weight.view(d))
        return off.square().mean()

    def answer(self, x: torch.Tensor, adapters=None, index: torch.Tensor | None = None) -> torch.Tensor:
        """``adapters``: (AdapterDesc, a, b, scale or None), one of them for every row by ``index``."""
        z, _, _ = lmkan_layer_norm(self.norm, x)
        y = super().answer(z)
        if adapters is not None:
            desc, a, b, scale = adapters
            lmkan_adapters_add(desc, z, index, a, b, y, scale=scale)
        return y

    def answer_in_float(self, x: torch.Tensor, adapters=None, index: torch.Tensor | None = None) -> torch.Tensor:
        y = self.forward(x)[0]
        if adapters is not None:
            desc, a, b, scale = adapters
            z = torch.relu(lmkan_layer_norm(self.norm, x)[0])
            for r in range(desc.count):
                rows = torch.nonzero(index == r)[:, 0]
                add = (z[rows] @ a[r].t()) @ b[r].t()
                y[rows] += add if scale is None else scale[r] * add
        return y


def random_adapters(count: int, rank: int, n_in: int, n_out: int, device, seed: int = 2):
    """Adapters of the linear term, as ``NormalisedLayer.answer`` takes them."""
    g = torch.Generator(device="cpu").manual_seed(seed)
    a = (torch.randn((count, rank, n_in), generator=g) / n_in ** 0.5).to(device)
    b = (0.1 * torch.randn((count, n_out, rank), generator=g)).to(device)
    return AdapterDesc(count, rank, n_in, n_out, relu=True), a, b, None


def run(steps: int = 60, batch: int = 2048, n_in: int = 64, n_out: int = 64, grid: int = 9, device="cuda:0",
        normalised: bool = False):
    """Trains on a fixed random function; returns (losses, relative difference of the 8-bit answer).  A normalised layer
    answers requests with adapters, of which every ninth row has none."""
    g = torch.Generator(device="cpu").manual_seed(1)
    mix = (torch.randn((n_in, n_out), generator=g) / n_in ** 0.5).to(device)
    model = (NormalisedLayer if normalised else PreconditionedLayer)(n_in, n_out, grid, 0.3, device)
    losses = []
    for step in range(steps):
        x = torch.randn((batch, n_in), generator=g).to(device)
        muon = MuonParams(lr=0.02 * (1.0 - step / steps), momentum=0.9)
        losses.append(float(model.train_step(x, torch.tanh(x @ mix), muon)))
    model.freeze()
    x = torch.randn((batch, n_in), generator=g).to(device)
    requests = ()
    if normalised:
        requests = random_adapters(8, 8, n_in, n_out, device), (torch.arange(batch, device=device) % 9 - 1).int()
    want = model.answer_in_float(x, *requests)
    return losses, float((model.answer(x, *requests) - want).norm() / want.norm())


def main() -> None:
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("steps", 60), ("batch", 2048), ("n-in", 64), ("n-out", 64), ("grid", 9)):
        p.add_argument(f"--{name}", type=int, default=value)
    p.add_argument("--norm", action="store_true")
    a = p.parse_args()
    losses, off = run(a.steps, a.batch, a.n_in, a.n_out, a.grid, normalised=a.norm)
    for k in range(0, len(losses), max(1, len(losses) // 10)):
        print(f"step {k:4d}  loss {losses[k]:.5f}")
    print(f"last step  loss {losses[-1]:.5f}; answer with 8-bit weights and rows: {off:.2%} off")


if __name__ == "__main__":
    main()
