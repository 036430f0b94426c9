"""Adapters of many rows (sorted by adapter, three launches), and the bits that products keep, against float64.

Tolerances, u = 2^-24:
  adapters   as for the linear term's gradient: roundings are of either sign and partial sums grow like the root of the number
             of terms, so that the root of the sum of squares times (n_in / 4 + rank / 4 + 64) u bounds them with room (a matrix
             instruction may cut instead of round, one-sided, on a quarter of the terms), two more for the sum with y
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


@pytest.mark.parametrize("size", [-100, -110, -115, -120, -126])
def test_bits_of_small_gradients(dev, size):
    """24 bits of a float32 gradient, those of them from 2^-133 on: one row, so that every element is one product."""
    codes, exps = _checkpoint(_rows(1, 200, seed=310) * 2.0 ** 40)
    gy = (1.0 + torch.rand((1, 90), generator=torch.Generator().manual_seed(311))) * 2.0 ** size
    value = _values(codes, exps)
    for relu in (False, True):
        gw, gb = pkg.lmkan_linear_grad(pkg.LinearDesc(200, 90, relu=relu), codes.to(dev), exps.to(dev), gy.to(dev))
        v = value.clamp(min=0.0) if relu else value
        want = gy.double().T @ v
        _within(gw, want, 2.25 * U * want.abs() + 2.0 ** -133 * v.abs(), "grad_weight")
        assert torch.equal(gb.cpu(), gy[0])


@pytest.mark.parametrize("w", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("size", [-100, -110, -115, -120, -126])
def test_bits_of_a_small_product_with_a(dev, w, size):
    """The same of what A makes of x, where adapters have 16 bits; all of it where they have 32."""
    batch, n, rank = 2000, 64, 8
    g = torch.Generator().manual_seed(315)
    x = (1.0 + torch.rand((batch, n), generator=g)) * 2.0 ** size
    a, b = torch.zeros(1, rank, n), torch.zeros(1, n, rank)
    a[0, torch.arange(rank), torch.arange(rank)] = 1.0
    b[0, torch.arange(n), torch.arange(n) % rank] = (1.0 + torch.rand((n,), generator=g)) * 2.0 ** (14 if w == "f16" else 40)
    a, b = a.to(DT[w]), b.to(DT[w])
    desc = pkg.AdapterDesc(1, rank, n, n, dtype=CODE[w])
    _sorted(desc, batch)
    got = pkg.lmkan_adapters_add(desc, x.to(dev), torch.zeros(batch, dtype=torch.int32, device=dev), a.to(dev), b.to(dev), torch.zeros((batch, n), device=dev))
    want = (x.double() @ a[0].double().T) @ b[0].double().T
    lost = 0.0 if w == "f32" else 2.0 ** -133
    # (and a result below the smallest normal number has its own unit)
    _within(got, want, 2.25 * U * want.abs() + lost * b[0].double().sum(dim=1) + 2.0 ** -149, "y")


@pytest.mark.parametrize("small", ["x", "a", "b"])
def test_float16_numbers_below_the_smallest_normal_one_count_in_many_rows(dev, small):
    """Multiples of 2^-24 are not taken as zeros.  Matrix instructions line products up by their factors' exponents, and a subnormal
    factor has that of 2^-14: sums are rounded as if it were that large, which is 2^-38 of the other factor for a product.  On the
    way up B is cut to parts that are normal numbers of bfloat16."""
    x, index, a, b, y, scale = _adapters(1500, 128, 64, 16, 3, w="f16", x="f16", y="f32", seed=345, index=torch.arange(1500) % 3)
    tiny = {"x": x, "a": a, "b": b}[small]
    tiny.copy_(tiny * 2.0 ** -18)
    desc = pkg.AdapterDesc(3, 16, 128, 64, dtype=CODE["f16"], x_dtype=CODE["f16"])
    _sorted(desc, 1500)
    got = pkg.lmkan_adapters_add(desc, x.to(dev), index.to(dev), a.to(dev), b.to(dev), torch.zeros_like(y).to(dev))
    for r in range(3):
        xd, ad, bd = x[r::3].double(), a[r].double(), b[r].double()
        want = (xd @ ad.T) @ bd.T
        size = ((xd.abs().clamp(min=2.0 ** -14).square() @ ad.abs().clamp(min=2.0 ** -14).square().T) @ bd.square().T).sqrt()
        _within(got[r::3], want, (128 / 4 + 16 / 4 + 64) * U * size + 2 * U * want.abs(), "y")
        # (a factor of ten leading zeros: u 2^10 of its product, twice that where a sum cuts)
        assert float((got[r::3].cpu().double() - want).norm() / want.norm()) < 2.0 ** -13
