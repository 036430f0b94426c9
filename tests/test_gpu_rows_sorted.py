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


def _check_sorted(dev, data, relu, scaled, w="f32", x_type="f32", y_type="f32", shift=None):
    """Against float64 within the root of the sum of squares; `shift`: every tensor starts that many elements into a buffer, of
    which nothing around the result may change."""
    x, index, a, b, y, scale = data
    count, rank, n_in = a.shape
    desc = pkg.AdapterDesc(count, rank, n_in, b.shape[1], dtype=CODE[w], x_dtype=CODE[x_type], y_dtype=CODE[y_type], relu=relu)
    _sorted(desc, x.shape[0])
    put = (lambda t: t.to(dev)) if shift is None else (lambda t: _guarded(t, dev, shift)[0])
    got, whole = (y.clone().to(dev), lambda: True) if shift is None else _guarded(y, dev, shift)
    pkg.lmkan_adapters_add(desc, put(x), put(index), put(a), put(b), got, scale=put(scale) if scaled else None)
    xd = x.double().clamp(min=0.0) if relu else x.double()
    want, size = y.double().clone(), torch.zeros(y.shape, dtype=torch.float64)
    has = (index >= 0) & (index < count)
    for r in index[has].unique().tolist():
        n = torch.nonzero(index == r)[:, 0]
        s = float(scale[r]) if scaled else 1.0
        ad, bd = a[r].double(), b[r].double()
        want[n] += s * ((xd[n] @ ad.T) @ bd.T)
        size[n] = s * ((xd[n].square() @ ad.square().T) @ bd.square().T).sqrt()
    assert torch.equal(got[~has].cpu(), y[~has])                       # bit for bit
    _within(got[has], want[has], ((n_in / 4 + rank / 4 + 64) * U * size + 2 * U * want.abs() + _out(want, y_type))[has], "y")
    assert whole()
    return desc, got.cpu()


@pytest.mark.parametrize("types", ["f32 f32 f32", "bf16 bf16 bf16", "f16 f16 f32", "bf16 f32 f32", "f32 f16 bf16"])
@pytest.mark.parametrize("rank", [1, 3, 6, 8, 16, 17, 20, 32, 33, 48, 64])
def test_small_ranks_of_many_rows(dev, rank, types):
    w, x, y = types.split()
    for n_in, n_out, relu in [(256, 160, True), (333, 77, False)]:
        _check_sorted(dev, _adapters(1500, n_in, n_out, rank, 3, w=w, x=x, y=y, seed=320), relu, True, w, x, y)


@pytest.mark.parametrize("kind", ["one", "none", "first", "last", "waves", "runs", "turns", "beyond"])
@pytest.mark.parametrize("batch", [3000, 40001])
def test_arrangements_of_many_requests(dev, kind, batch):
    """Rows of one adapter, of none, runs that fill waves of 64 and runs that do not, indices far out of range; 40001 rows are
    sorted in two parts."""
    at, none = torch.arange(batch), torch.full((batch,), -1)
    index = {"one": torch.full((batch,), 4), "none": none, "first": torch.where(at == 0, 0, none), "last": torch.where(at == batch - 1, 8, none),
             "waves": at // 256 % 11 - 1, "runs": at // 77 % 9, "turns": at % 9, "beyond": torch.tensor([-2 ** 31, 2 ** 31 - 1, 9, 8, 0])[at % 5]}[kind]
    _check_sorted(dev, _adapters(batch, 80, 50, 10, 9, index=index, seed=325), False, True)


@pytest.mark.parametrize("count", [1, 2, 1023, 1025, 8191, 8192])
def test_many_adapters_of_many_rows(dev, count):
    index = (torch.arange(2500) * 7919) % (count + 1) - int(count > 1)
    index[::5] = count - 1
    _check_sorted(dev, _adapters(2500, 24, 20, 4, count, index=index, seed=330), True, False)


@pytest.mark.parametrize("types", ["f32 f32 f32", "bf16 bf16 bf16", "f16 f16 f32", "bf16 f32 f16", "f32 f16 bf16"])
@pytest.mark.parametrize("shape", [(128, 96, 16), (131, 45, 5), (333, 77, 130)], ids=str)
@pytest.mark.parametrize("shift", [1, 3, 8])
def test_many_rows_anywhere_and_nothing_written_beyond(dev, shape, types, shift):
    w, x, y = types.split()
    n_in, n_out, rank = shape
    _check_sorted(dev, _adapters(1100, n_in, n_out, rank, 5, w=w, x=x, y=y, seed=335), True, True, w, x, y, shift=shift)


@pytest.mark.parametrize("types", ["f32 f32 f32", "bf16 bf16 bf16", "f16 f16 f32", "f32 f16 bf16"])
@pytest.mark.parametrize("shape", [(128, 64, 24), (131, 65, 23)], ids=str)
def test_values_that_are_not_finite_stay_in_their_rows_of_a_tile(dev, shape, types):
    w, x_type, y_type = types.split()
    n_in, n_out, rank = shape
    rows = 1500
    data = _adapters(rows, n_in, n_out, rank, 3, w=w, x=x_type, y=y_type, seed=340, index=torch.arange(rows) % 3)
    x, index, a, b, y, scale = data
    desc, clean = _check_sorted(dev, data, False, True, w, x_type, y_type)
    x, a, b, y = x.clone(), a.clone(), b.clone(), y.clone()
    x[7, 5] = float("nan")
    x[9, n_in - 1] = float("-inf")
    a[2, 0, 0] = float("inf")
    b[1, n_out - 1, rank - 1] = float("inf")
    y[12, 3] = float("nan")
    got = pkg.lmkan_adapters_add(desc, x.to(dev), index.to(dev), a.to(dev), b.to(dev), y.to(dev), scale=scale.to(dev)).cpu()
    want = torch.zeros(rows, n_out, dtype=torch.bool)
    want[7] = want[9] = want[2::3] = True
    want[1::3, n_out - 1] = want[12, 3] = True
    assert torch.equal(~torch.isfinite(got), want)
    assert torch.equal(got[~want], clean[~want])


def test_many_rows_twice_in_a_workspace_and_in_a_graph(dev):
    """The same workspace for two calls one after the other, eager and replayed, gives what workspaces of their own give."""
    first, second = _adapters(1500, 96, 64, 12, 4, seed=350), _adapters(2900, 96, 64, 12, 4, seed=360)
    desc = pkg.AdapterDesc(4, 12, 96, 64)
    ws = torch.empty(max(pkg.lmkan_adapters_workspace_bytes(desc, n) for n in (1500, 2900)), dtype=torch.uint8, device=dev)
    data = [[t.to(dev) for t in d] for d in (first, second)]
    want = [pkg.lmkan_adapters_add(desc, x, i, a, b, y.clone(), scale=s) for x, i, a, b, y, s in data]
    out = [torch.empty_like(t) for t in want]

    def both():
        for (x, i, a, b, y, s), to in zip(data, out):
            to.copy_(y)
            pkg.lmkan_adapters_add(desc, x, i, a, b, to, scale=s, workspace=ws)
    both()
    assert all(torch.equal(o, t) for o, t in zip(out, want))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for _ in range(4):
        ws.fill_(0x5a)
        for o in out:
            o.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, t) for o, t in zip(out, want))


def test_the_example_answers_with_adapters(dev, monkeypatch):
    """The command's run of a normalised layer goes through the operators that the package's description names, on many rows,
    and its answers in 8 bits are those in float32 but for the rounding of rows and weights."""
    from paper_2509_07103_amd import preconditioned
    names = ["lmkan_layer_norm", "lmkan_layer_norm_backward", "lmkan_restore_rows", "lmkan_linear_grad", "lmkan_linear_i8", "lmkan_adapters_add"]
    calls = []

    def spy(name, call):
        def recorded(*args, **kw):
            calls.append(name)
            return call(*args, **kw)
        return recorded
    for name in names:
        monkeypatch.setattr(preconditioned, name, spy(name, getattr(preconditioned, name)))
    losses, off = preconditioned.run(2, 1100, 32, 24, 7, normalised=True)
    assert len(losses) == 2 and set(calls) == set(names)
    # codes are off by half a step of 1/127 of the largest in a row, of which there are two factors
    assert off < 0.05
