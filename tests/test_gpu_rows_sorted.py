"""Adapters of many rows (sorted by adapter, three launches), and the bits that products keep, against float64.

Tolerances, u = 2^-24:
  adapters   a sum of n products in float32 is off by n u of the sum of magnitudes at most, 2 u where a matrix instruction cuts;
             roundings are of either sign, so that (sqrt(n_in) + sqrt(rank) + 16) u times the root of the sum of squares of
             what enters an element bounds them with room (the terms that are lost to a part of 8 bits less, 2^-16 of their
             size, would be 256 u)
  one term   where one product reaches an element: its parts are exact and so are their products; all but the largest add up
             to less than 2^-6 of it, so that 2 u for the last sum (which may cut) and a quarter for the others bound it
"""
import pytest
import torch

import paper_2509_07103_amd as pkg
from test_gpu_rows import CODE, DT, U, _adapters, _check_adapters, _checkpoint, _guarded, _out, _randn, _rows, _values, _within, dev  # noqa: F401

pytestmark = pytest.mark.gpu


def _sorted(desc, batch):
    """Three launches have a workspace, one has none."""
    assert pkg.lmkan_adapters_workspace_bytes(desc, batch) > 0, "not the path of many rows"


def _selecting(x_type, batch, n_in, rank, seed):
    """Rows x and A [2][rank][n_in] of zeros and ones whose A x is exact in float32 and has 24 bits."""
    g = torch.Generator().manual_seed(seed)
    if x_type == "f32":
        x, parts = 1.0 + torch.rand((batch, n_in), generator=g), 1
    else:
        # 1.0 .. 1.9 in the type's bits, and the rest of 24 bits in one element more (float16) or two (bfloat16)
        first = (1.0 + 0.9 * torch.rand((batch, n_in), generator=g)).to(DT[x_type]).float()
        if x_type == "f16":
            x, parts = torch.where(torch.arange(n_in) % 2 == 0, first, torch.randint(0, 2048, (batch, n_in), generator=g) * 2.0 ** -24 * 2), 2
        else:
            small = torch.randint(0, 256, (batch, n_in), generator=g).float()
            x, parts = torch.where(torch.arange(n_in) % 3 == 0, first, small * torch.where(torch.arange(n_in) % 3 == 1, 2.0 ** -15, 2.0 ** -23)), 3
    x = x * torch.where(torch.rand((batch, 1), generator=g) < 0.5, 1.0, -1.0)
    assert torch.equal(x.to(DT[x_type]).float(), x)
    a = torch.zeros(2, rank, n_in)
    for r in range(2):
        for k in range(rank):
            at = (5 * k + r) % (n_in // parts) * parts
            a[r, k, at:at + parts] = 1.0
    return x.to(DT[x_type]), a


@pytest.mark.parametrize("types", ["f16 f32", "bf16 f32", "f16 f16", "bf16 bf16", "f32 f32", "f32 bf16"])
@pytest.mark.parametrize("rank", [8, 16, 32, 40, 64, 128, 200])
def test_products_keep_the_bits_of_what_a_makes_of_x(dev, types, rank):
    w, x_type = types.split()
    batch, n_in, n_out = 2500, 384, 160
    x, a = _selecting(x_type, batch, n_in, rank, seed=300 + rank)
    low = torch.stack([x.double() @ a[r].double().T for r in range(2)])
    assert torch.equal(low.float().double(), low) and (low.abs() < 2).all()
    b = torch.zeros(2, n_out, rank)
    g = torch.Generator().manual_seed(301)
    at = torch.randint(0, rank, (2, n_out, 1), generator=g)
    b.scatter_(2, at, (1.0 + torch.rand((2, n_out, 1), generator=g)) * torch.where(torch.rand((2, n_out, 1), generator=g) < 0.5, 1.0, -1.0))
    a, b, index = a.to(DT[w]), b.to(DT[w]), torch.randint(0, 2, (batch,), generator=g).int()
    desc = pkg.AdapterDesc(2, rank, n_in, n_out, dtype=CODE[w], x_dtype=CODE[x_type])
    _sorted(desc, batch)
    got = pkg.lmkan_adapters_add(desc, x.to(dev), index.to(dev), a.to(dev), b.to(dev), torch.zeros((batch, n_out), device=dev))
    want = torch.stack([low[r] @ b[r].double().T for r in range(2)])[index.long(), torch.arange(batch)]
    assert (want != 0).all()
    _within(got, want, 2.25 * U * want.abs(), "y")
