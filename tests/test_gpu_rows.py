"""Operators on rows (layer norm and its gradients, 8-bit checkpoints, the linear term's gradient from them, low-rank
adapters) against plain implementations in float64.

Tolerances, u = 2^-24 (a float32 rounding is off by u of the value at most), elementwise:
  checkpoints   exact: both scalings are by powers of two, the rounding is that of the definition
  norm          hat is fl(fl(x - mean) rstd) of float32 statistics: off by u |mean| rstd + 3 u |hat|; the affine map adds
                one rounding, the output type its own
  gradients     a sum of n terms in chains of at most K additions is off by K u sum |terms|.  Over a row, chains are at
                most cols / 64 + 48 long (64 lanes a row, or up to 48 elements a lane for short rows, and the steps that
                join lanes); over the rows of a batch at most min(rows, 1300) + 8
  linear        a product of 24 bits of the gradient is off by u, a sum over n rows by n u of the sum of magnitudes;
                roundings are of either sign and partial sums grow like the root of the number of terms, so that the root
                of the sum of squares times (n / 4 + 64) u bounds them with room (a matrix instruction may cut instead of
                round, one-sided, on n / 16 sums of three parts each)
  adapters      n_in + rank + 16 roundings of the sum of magnitudes, two more for the sum with y
and a 16-bit result adds its own unit (half a step) of the value; below the smallest normal number half a step is absolute.
"""
import numpy as np
import pytest
import torch

import paper_2509_07103_amd as pkg

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
CODE = {"f32": pkg.LMKAN_F32, "f16": pkg.LMKAN_F16, "bf16": pkg.LMKAN_BF16}
UNIT = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 2.0 ** -150, "f16": 2.0 ** -25, "bf16": 2.0 ** -134}
U = 2.0 ** -24
TYPES = ["f32", "f16", "bf16"]


@pytest.fixture(scope="module")
def dev():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    pkg.lib()
    return torch.device("cuda:0")


def _randn(*shape, seed=0):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed))


def _rows(rows, cols, dtype="f32", seed=0, offset=0.5):
    """Rows with means and sizes of their own."""
    x = _randn(rows, cols, seed=seed) * (0.25 + 2.0 * torch.rand((rows, 1), generator=torch.Generator().manual_seed(seed + 1)))
    return (x + offset * _randn(rows, 1, seed=seed + 2)).to(DT[dtype])


def _within(got, want, tol, what=""):
    off = (got.detach().cpu().double() - want).abs()
    bad = ~(off <= tol)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float((off / tol).nan_to_num(nan=np.inf).max()):.3g} of the tolerance"


def _out(value, dtype):
    """Rounding to the output's type."""
    return UNIT[dtype] * value.abs() + TINY[dtype]


# ---- checkpoints -----------------------------------------------------------------------------------------------------

def _checkpoint(x, relu=False):
    """(codes, bytes) by the definition, in numpy."""
    x = x.float().numpy().astype(np.float64)
    if relu:
        x = np.where(x < 0, 0.0, x)
    rows, cols = x.shape
    blocks = -(-cols // 32)
    full = np.zeros((rows, blocks * 32))
    full[:, :cols] = x
    full = full.reshape(rows, blocks, 32)
    finite = np.isfinite(full).all(axis=2)
    top = np.abs(np.where(finite[..., None], full, 0.0)).max(axis=2)
    e = np.frexp(top)[1] - 7
    e = e + (np.rint(np.ldexp(top, -e)) > 127)
    e = np.clip(e, -133, 121)
    codes = np.clip(np.rint(np.ldexp(np.where(finite[..., None], full, 0.0), -e[..., None])), -127, 127)
    stored = np.where(finite, np.where(top > 0, e + 133, 0), 255)
    return (torch.from_numpy(codes.reshape(rows, -1)[:, :cols].astype(np.int8)), torch.from_numpy(stored.astype(np.uint8)))


def _values(codes, exps):
    """float64 of what a checkpoint stands for."""
    e = exps.to(torch.int64).repeat_interleave(32, dim=1)[:, :codes.shape[1]]
    v = torch.from_numpy(np.ldexp(codes.numpy().astype(np.float64), e.numpy() - 133))
    return torch.where(e == 255, torch.full_like(v, float("nan")), v)


SHAPES = [(1, 1), (1, 31), (3, 32), (2, 33), (5, 63), (7, 64), (4, 100), (3, 128), (64, 500), (9, 1000), (2, 1024), (3, 2050), (2, 4096),
          (1, 16384), (2, 20011), (1, 131070), (333, 8), (1000, 3), (70001, 2)]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("dtype", TYPES)
def test_checkpoint_and_restore_are_exact(dev, shape, dtype):
    x = _rows(*shape, dtype=dtype, seed=1)
    for relu in (False, True):
        codes, exps = pkg.lmkan_checkpoint_rows(x.to(dev), relu=relu)
        want = _checkpoint(x, relu)
        assert torch.equal(codes.cpu(), want[0]) and torch.equal(exps.cpu(), want[1])
        values = _values(*want)
        for out in TYPES:
            y = pkg.lmkan_restore_rows(codes, exps, dtype=CODE[out])
            assert y.dtype == DT[out] and torch.equal(y.cpu(), values.to(DT[out]))
    # nearest values: off by half a step of 1/64 of the largest in the block, 1/127 of it at most
    top = torch.nn.functional.pad(x.float().clamp(min=0.0), (0, -shape[1] % 32)).view(shape[0], -1, 32).amax(dim=2).repeat_interleave(32, dim=1)
    assert ((values - x.double().clamp(min=0.0)).abs() <= top[:, :shape[1]].double() / 127).all()


def test_checkpoints_of_extreme_values(dev):
    """Blocks of one magnitude each: from subnormal numbers to the largest, powers of two and ties, zeros of both signs."""
    rows = []
    for scale in [2.0 ** -149, 2.0 ** -140, 2.0 ** -127, 2.0 ** -126, 1e-30, 2.0 ** -10, 1.0, 2.0 ** 20, 1e30, 2.0 ** 126, 1.9 * 2.0 ** 126]:
        v = np.float32(scale) * np.linspace(-1.0, 1.0, 32).astype(np.float32)
        rows += [v, np.abs(v)]
    largest = np.finfo(np.float32).max
    rows.append(np.full(32, largest, np.float32) * np.linspace(-1, 1, 32).astype(np.float32))
    rows.append(np.array([largest] + [largest / 2] * 31, np.float32))
    rows.append(np.array([127.0] + [k + 0.5 for k in range(31)], np.float32))          # ties to even
    rows.append(np.array([127.5] + [k + 0.5 for k in range(31)], np.float32))          # the largest would be 128: a step of 2
    rows.append(np.array([np.nextafter(np.float32(127.5), np.float32(0))] + [1.5] * 31, np.float32))
    rows.append(np.array([64.0] + [0.5, 0.25, -0.5, 1.5] + [-0.0] * 27, np.float32))
    rows.append(np.zeros(32, np.float32))
    rows.append(np.full(32, -0.0, np.float32))
    x = torch.from_numpy(np.stack(rows))
    for relu in (False, True):
        codes, exps = pkg.lmkan_checkpoint_rows(x.to(dev), relu=relu)
        want = _checkpoint(x, relu)
        assert torch.equal(exps.cpu(), want[1]) and torch.equal(codes.cpu(), want[0])
        assert torch.equal(pkg.lmkan_restore_rows(codes, exps).cpu(), _values(*want).float())


def test_blocks_that_are_not_finite_become_nan_and_leave_the_others_alone(dev):
    x = _rows(6, 150, seed=3)
    x[0, 40], x[1, 149], x[2, 0], x[3, 64:96] = float("nan"), float("inf"), -float("inf"), float("nan")
    codes, exps = pkg.lmkan_checkpoint_rows(x.to(dev))
    want = _checkpoint(x)
    assert torch.equal(codes.cpu(), want[0]) and torch.equal(exps.cpu(), want[1])
    y = pkg.lmkan_restore_rows(codes, exps, weight=torch.full((150,), 2.0, device=dev), relu=True).cpu()
    nan = torch.isnan(_values(*want))
    assert int(nan.sum()) == 32 + 22 + 32 + 32 and torch.equal(torch.isnan(y), nan)
    x = x.clamp(max=0.0)
    codes, exps = pkg.lmkan_checkpoint_rows(x.to(dev), relu=True)                       # max(NaN, 0) is NaN, max(-inf, 0) is 0
    assert int((exps.cpu() == 255).sum()) == 2 and int(exps.cpu().long().sum()) == 510


@pytest.mark.parametrize("shape", [(5, 70), (3, 1024), (300, 33)], ids=str)
@pytest.mark.parametrize("dtype", TYPES)
def test_restore_with_affine_and_relu(dev, shape, dtype):
    codes, exps = _checkpoint(_rows(*shape, seed=4))
    w, b = _randn(shape[1], seed=5), _randn(shape[1], seed=6)
    v = _values(codes, exps)
    for weight, bias, relu in [(w, b, False), (w, b, True), (w, None, False), (None, b, True), (None, None, True)]:
        want = v * (1.0 if weight is None else weight.double()) + (0.0 if bias is None else bias.double())
        want = want.clamp(min=0.0) if relu else want
        y = pkg.lmkan_restore_rows(codes.to(dev), exps.to(dev), weight=None if weight is None else weight.to(dev),
                                   bias=None if bias is None else bias.to(dev), relu=relu, dtype=CODE[dtype])
        _within(y, want, _out(want, dtype) + 2 * U * want.abs())


# ---- layer norm ------------------------------------------------------------------------------------------------------

EPS = float(np.float32(1e-5))   # the descriptor's eps is a float32


def _statistics(x):
    x = x.double()
    mean = x.mean(dim=1, keepdim=True)
    return mean, 1.0 / torch.sqrt((x - mean).square().mean(dim=1, keepdim=True) + EPS)


def _check_norm(dev, x, dtype, weight, bias, keep, eps=EPS):
    x_dtype = {v: k for k, v in DT.items()}[x.dtype]
    desc = pkg.NormDesc(x.shape[1], x_dtype=CODE[x_dtype], y_dtype=CODE[dtype], eps=eps)
    on = [None if t is None else t.to(dev) for t in (weight, bias)]
    y, stats, kept = pkg.lmkan_layer_norm(desc, x.to(dev), *on, keep=keep)
    mean, rstd = _statistics(x)
    xd = x.double()
    spread = xd.abs().amax(dim=1, keepdim=True)
    _within(stats, torch.cat([mean, rstd], dim=1), torch.cat([U * mean.abs() + 2.0 ** -50 * spread, 1.01 * U * rstd], dim=1), "stats")
    hat = (xd - mean) * rstd
    w = torch.ones(x.shape[1]).double() if weight is None else weight.double()
    want = hat * w + (0.0 if bias is None else bias.double())
    _within(y, want, (U * mean.abs() * rstd + 4 * U * hat.abs()) * w.abs() + U * want.abs() + _out(want, dtype), "y")
    assert (kept is not None) == keep
    if keep:
        hat32 = (x.float() - mean.float()) * rstd.float()
        codes, exps = _checkpoint(hat32)
        assert torch.equal(kept[0].cpu(), codes) and torch.equal(kept[1].cpu(), exps)
    return y, stats, kept


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_layer_norm_matches_float64(dev, shape, dtype):
    x = _rows(*shape, dtype=dtype, seed=7)
    w, b = _randn(shape[1], seed=8), _randn(shape[1], seed=9)
    _check_norm(dev, x, dtype, w, b, keep=True)
    _check_norm(dev, x, dtype, None, None, keep=False)


@pytest.mark.parametrize("x_dtype", TYPES)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", [(37, 50), (6, 640), (2, 5000), (2, 40000)], ids=str)
def test_layer_norm_in_every_pair_of_types(dev, x_dtype, dtype, shape):
    x = _rows(*shape, dtype=x_dtype, seed=10)
    _check_norm(dev, x, dtype, _randn(shape[1], seed=11), None, keep=True)
    _check_norm(dev, x, dtype, None, _randn(shape[1], seed=11), keep=False)


@pytest.mark.parametrize("cols", [4, 40, 1000, 6000, 30000])
def test_rows_with_large_means_and_magnitudes(dev, cols):
    """Offsets of up to ten thousand times the spread; magnitudes whose squares exceed float32, or vanish in eps."""
    x = torch.cat([_randn(2, cols, seed=12) + 1e4, 1e-3 * _randn(2, cols, seed=13) - 7.0, 1e30 * _randn(2, cols, seed=14),
                   1e-30 * _randn(2, cols, seed=15), torch.full((1, cols), 3.25), torch.zeros((1, cols))])
    y, stats, _ = _check_norm(dev, x, "f32", None, None, keep=True)
    assert torch.equal(y[-2:].cpu(), torch.zeros((2, cols)))


def test_a_row_that_is_not_finite_stays_alone(dev):
    for cols in (20, 700, 9000):
        x = _rows(5, cols, seed=16)
        clean = x.clone()
        x[1, 3], x[3, -1] = float("nan"), float("inf")
        y, stats, kept = pkg.lmkan_layer_norm(pkg.NormDesc(cols), x.to(dev), keep=True)
        back = pkg.lmkan_restore_rows(*kept)
        want, _, want_kept = pkg.lmkan_layer_norm(pkg.NormDesc(cols), clean.to(dev), keep=True)
        for r in range(5):
            if r in (1, 3):
                assert torch.isnan(y[r]).all() and torch.isnan(back[r]).all()
            else:
                assert torch.equal(y[r], want[r]) and torch.equal(kept[0][r], want_kept[0][r])


@pytest.mark.parametrize("shape", [(3, 20), (9, 1024), (2, 30000)], ids=str)
def test_layer_norm_in_place(dev, shape):
    x, w = _rows(*shape, seed=17).to(dev), _randn(shape[1], seed=18).to(dev)
    want, _, kept = pkg.lmkan_layer_norm(pkg.NormDesc(shape[1]), x, w, keep=True)
    again, _, kept_again = pkg.lmkan_layer_norm(pkg.NormDesc(shape[1]), x, w, y=x, keep=True)
    assert again.data_ptr() == x.data_ptr() and torch.equal(want, x)
    assert torch.equal(kept[0], kept_again[0]) and torch.equal(kept[1], kept_again[1])


def _norm_gradients(hat, rstd, gy, weight):
    d = gy if weight is None else gy * weight
    dm, dh = d.mean(dim=1, keepdim=True), (d * hat).mean(dim=1, keepdim=True)
    gx = rstd * (d - dm - hat * dh)
    k = hat.shape[1] / 64 + 48
    tol = rstd * U * (6 * d.abs() + (k + 4) * d.abs().mean(dim=1, keepdim=True) + (k + 8) * hat.abs() * (d * hat).abs().mean(dim=1, keepdim=True))
    return gx, tol


def _check_norm_backward(dev, shape, x_dtype, y_dtype, kept, affine, seed=20):
    rows, cols = shape
    desc = pkg.NormDesc(cols, x_dtype=CODE[x_dtype], y_dtype=CODE[y_dtype], eps=EPS)
    x = _rows(rows, cols, x_dtype, seed=seed)
    gy = (1e-3 * _randn(rows, cols, seed=seed + 5)).to(DT[y_dtype])
    weight = _randn(cols, seed=seed + 6) if affine else None
    mean, rstd = (t.float() for t in _statistics(x))
    stats = torch.cat([mean, rstd], dim=1)
    checkpoint = _checkpoint((x.float() - mean) * rstd)
    hat = _values(*checkpoint) if kept else (x.double() - mean.double()) * rstd.double()
    want, tol = _norm_gradients(hat, rstd.double(), gy.double(), None if weight is None else weight.double())
    got = pkg.lmkan_layer_norm_backward(desc, gy.to(dev), stats.to(dev), x=None if kept else x.to(dev),
                                        kept=tuple(t.to(dev) for t in checkpoint) if kept else None,
                                        weight=None if weight is None else weight.to(dev))
    assert got[0].dtype == DT[x_dtype]
    _within(got[0], want, tol + _out(want, x_dtype), "grad_x")
    k = min(rows, 1300) + 8
    g = gy.double()
    _within(got[1], (g * hat).sum(dim=0), (k + 3) * U * (g * hat).abs().sum(dim=0) + 1e-44, "grad_weight")
    _within(got[2], g.sum(dim=0), k * U * g.abs().sum(dim=0) + 1e-44, "grad_bias")
    return desc, gy, stats, x, checkpoint, weight, got


@pytest.mark.parametrize("shape", SHAPES + [(4099, 64), (20000, 40), (3000, 129)], ids=str)
@pytest.mark.parametrize("kept", [False, True], ids=["rows", "kept"])
def test_layer_norm_backward_matches_float64(dev, shape, kept):
    _check_norm_backward(dev, shape, "f32", "f32", kept, affine=True)
    _check_norm_backward(dev, shape, "bf16", "bf16", kept, affine=False, seed=40)


@pytest.mark.parametrize("shape", [(3, 8200), (5, 9001), (2, 12345), (530, 8193), (300, 16384), (4, 16385)], ids=str)
@pytest.mark.parametrize("types", ["f32 f32", "bf16 bf16", "f16 f32"])
def test_rows_on_either_side_of_what_registers_hold(dev, shape, types):
    x_dtype, y_dtype = types.split()
    x = _rows(*shape, dtype=x_dtype, seed=65)
    w, b = _randn(shape[1], seed=66), _randn(shape[1], seed=67)
    _check_norm(dev, x, y_dtype, w, b, keep=True)
    _check_norm(dev, x, y_dtype, None, None, keep=False)
    for kept in (False, True):
        _check_norm_backward(dev, shape, x_dtype, y_dtype, kept, affine=True, seed=68)


@pytest.mark.parametrize("x_dtype", TYPES)
@pytest.mark.parametrize("y_dtype", TYPES)
@pytest.mark.parametrize("shape", [(37, 50), (6, 640), (3, 5000), (2, 40000)], ids=str)
def test_layer_norm_backward_in_every_pair_of_types(dev, x_dtype, y_dtype, shape):
    for kept in (False, True):
        _check_norm_backward(dev, shape, x_dtype, y_dtype, kept, affine=True, seed=60)


@pytest.mark.parametrize("shape", [(5, 40), (300, 1024), (3, 30000)], ids=str)
@pytest.mark.parametrize("kept", [False, True], ids=["rows", "kept"])
def test_parts_of_the_backward_call(dev, shape, kept):
    """Every subset of the gradients gives the same bits; accumulation adds; nothing else is written."""
    desc, gy, stats, x, checkpoint, weight, got = _check_norm_backward(dev, shape, "f32", "f32", kept, affine=True, seed=80)
    args = dict(x=None if kept else x.to(dev), kept=tuple(t.to(dev) for t in checkpoint) if kept else None, weight=weight.to(dev))
    gy, stats = gy.to(dev), stats.to(dev)
    for need in range(8):
        flags = [bool(need & 1), bool(need & 2), bool(need & 4)]
        part = pkg.lmkan_layer_norm_backward(desc, gy, stats, **args, need_grad_x=flags[0], need_grad_weight=flags[1], need_grad_bias=flags[2])
        for p, g, f in zip(part, got, flags):
            assert (p is None) == (not f) and (p is None or torch.equal(p, g))
    base = [_randn(shape[1], seed=90).to(dev), _randn(shape[1], seed=91).to(dev)]
    sums = [t.clone() for t in base]
    pkg.lmkan_layer_norm_backward(desc, gy, stats, **args, grad_weight=sums[0], grad_bias=sums[1], accumulate=True)
    for s, b, g in zip(sums, base, got[1:]):
        assert torch.equal(s, b + g)


def test_norm_gradients_against_differences(dev):
    """The gradient of sum(y c), by central differences of the operator's own forward pass."""
    rows, cols = 3, 37
    x, w, b, c = _rows(rows, cols, seed=100).double(), _randn(cols, seed=101).double(), _randn(cols, seed=102).double(), _randn(rows, cols, seed=103).double()
    desc = pkg.NormDesc(cols, eps=1e-3)
    y, stats, _ = pkg.lmkan_layer_norm(desc, x.float().to(dev), w.float().to(dev), b.float().to(dev))
    gx, gw, gb = pkg.lmkan_layer_norm_backward(desc, c.float().to(dev), stats, x=x.float().to(dev), weight=w.float().to(dev))

    def value(x_, w_, b_):
        got = pkg.lmkan_layer_norm(desc, x_.float().to(dev), w_.float().to(dev), b_.float().to(dev))[0]
        return float((got.cpu().double() * c).sum())
    h = 2.0 ** -6
    for i, j in [(0, 0), (1, 17), (2, 36)]:
        for which, grad in ((0, gx[i, j]), (1, gw[j]), (2, gb[j])):
            at = [x.clone(), w.clone(), b.clone()]
            to = at[which][i, j:j + 1] if which == 0 else at[which][j:j + 1]
            to += h
            up = value(*at)
            to -= 2 * h
            down = value(*at)
            # rounding of the values (111 terms of about 1, off by 2^-22 in all) over 2 h, and h^2 of the third derivative
            assert abs((up - down) / (2 * h) - float(grad)) <= 111 * 2.0 ** -22 / (2 * h) + 20 * h * h


def test_norm_without_rows(dev):
    desc, none = pkg.NormDesc(24), torch.zeros((0, 24), device=dev)
    y, stats, kept = pkg.lmkan_layer_norm(desc, none, keep=True)
    assert y.shape == (0, 24) and stats.shape == (0, 2) and kept[0].shape == (0, 24) and kept[1].shape == (0, 1)
    gw, gb = torch.full((24,), 3.0, device=dev), torch.full((24,), 4.0, device=dev)
    pkg.lmkan_layer_norm_backward(desc, none, stats, x=none, grad_weight=gw, grad_bias=gb, accumulate=True)
    assert float(gw.min()) == 3.0 and float(gb.min()) == 4.0
    _, gw, gb = pkg.lmkan_layer_norm_backward(desc, none, stats, kept=kept, grad_weight=gw, grad_bias=gb)
    assert not gw.any() and not gb.any()


# ---- the linear term's gradient --------------------------------------------------------------------------------------

def _check_grad(dev, batch, n_in, n_out, dtype, relu, bias, seed=110, gradient=None):
    codes, exps = _checkpoint(_rows(batch, n_in, seed=seed)) if batch else (torch.zeros((0, n_in), dtype=torch.int8), torch.zeros((0, -(-n_in // 32)), dtype=torch.uint8))
    gy = (1e-3 * _randn(batch, n_out, seed=seed + 1)).to(DT[dtype]) if gradient is None else gradient
    desc = pkg.LinearDesc(n_in, n_out, y_dtype=CODE[dtype], relu=relu)
    gw, gb = pkg.lmkan_linear_grad(desc, codes.to(dev), exps.to(dev), gy.to(dev), need_grad_bias=bias)
    v, g = _values(codes, exps), gy.double()
    v = v.clamp(min=0.0) if relu else v
    size = torch.sqrt(g.square().T @ v.square())
    _within(gw, g.T @ v, (batch / 4 + 64) * U * size + 1e-44, "grad_weight")
    assert (gb is not None) == bias
    if bias:
        _within(gb, g.sum(dim=0), (batch / 4 + 64) * U * g.square().sum(dim=0).sqrt() + 1e-44, "grad_bias")
    return desc, codes.to(dev), exps.to(dev), gy.to(dev), gw, gb


GRADS = [(0, 8, 4), (1, 1, 1), (1, 40, 24), (2, 33, 5), (31, 64, 64), (32, 128, 128), (33, 127, 129), (64, 32, 1), (100, 500, 333), (257, 100, 7),
         (1000, 16, 16), (4097, 64, 32), (5000, 130, 70), (300, 1, 500), (300, 500, 1), (20000, 40, 24), (1024, 512, 512), (640, 1030, 260)]


@pytest.mark.parametrize("shape", GRADS, ids=str)
@pytest.mark.parametrize("dtype", TYPES)
def test_linear_grad_matches_float64(dev, shape, dtype):
    _check_grad(dev, *shape, dtype, relu=True, bias=True)
    _check_grad(dev, *shape, dtype, relu=False, bias=False, seed=120)


@pytest.mark.parametrize("shape", [(70, 2048, 4352), (130, 2049, 4101), (1, 4096, 4160)], ids=str)
@pytest.mark.parametrize("dtype", TYPES)
def test_linear_grad_of_more_tiles_than_units(dev, shape, dtype):
    desc, codes, exps, gy, gw, gb = _check_grad(dev, *shape, dtype, relu=True, bias=True, seed=125)
    base = torch.ones_like(gw), torch.ones_like(gb)
    pkg.lmkan_linear_grad(desc, codes, exps, gy, grad_weight=base[0], grad_bias=base[1], accumulate=True)
    assert torch.equal(base[0], 1 + gw) and torch.equal(base[1], 1 + gb)


@pytest.mark.parametrize("dtype", TYPES)
def test_products_keep_the_bits_of_the_gradient(dev, dtype):
    """One row: every element is one product, off by 2^-24 for the bits of a float32 gradient that are kept and 2^-24 for
    the product (24 bits times 7)."""
    codes, exps = _checkpoint(_rows(1, 200, seed=130))
    gy = (_randn(1, 90, seed=131) * torch.exp2(torch.randint(-60, 60, (1, 90), generator=torch.Generator().manual_seed(132)).float())).to(DT[dtype])
    gy = gy.nan_to_num(posinf=1.0, neginf=-1.0)
    gw, _ = pkg.lmkan_linear_grad(pkg.LinearDesc(200, 90, y_dtype=CODE[dtype]), codes.to(dev), exps.to(dev), gy.to(dev))
    want = gy.double().T @ _values(codes, exps)
    _within(gw, want, 2 * U * want.abs() + 2.0 ** -126, "grad_weight")


def test_gradients_of_any_size_beside_each_other(dev):
    """Rows of the batch whose gradients and activations lie many powers of two apart, rows of zeros among them."""
    g = torch.Generator().manual_seed(140)
    gy = _randn(300, 70, seed=141) * torch.exp2(torch.randint(-30, 30, (300, 1), generator=g).float())
    gy[::7] = 0.0
    _check_grad(dev, 300, 90, 70, "f32", True, True, seed=142, gradient=gy)


@pytest.mark.parametrize("shape", [(50, 40, 24), (3000, 256, 200)], ids=str)
def test_linear_grad_accumulates_and_repeats(dev, shape):
    desc, codes, exps, gy, gw, gb = _check_grad(dev, *shape, "f32", True, True, seed=150)
    again = pkg.lmkan_linear_grad(desc, codes, exps, gy)
    assert torch.equal(again[0], gw) and torch.equal(again[1], gb)
    base = [_randn(*gw.shape, seed=151).to(dev), _randn(*gb.shape, seed=152).to(dev)]
    sums = [t.clone() for t in base]
    pkg.lmkan_linear_grad(desc, codes, exps, gy, grad_weight=sums[0], grad_bias=sums[1], accumulate=True)
    assert torch.equal(sums[0], base[0] + gw) and torch.equal(sums[1], base[1] + gb)
    sums[0].copy_(base[0])
    pkg.lmkan_linear_grad(desc, codes, exps, gy, need_grad_bias=False, grad_weight=sums[0], accumulate=True)
    assert torch.equal(sums[0], base[0] + gw)


def test_linear_grad_of_values_that_are_not_finite(dev):
    """A block that stands for NaN reaches its 32 columns, a gradient that is not finite its output, and no other."""
    x = _rows(70, 100, seed=160)
    x[5, 40] = float("nan")
    codes, exps = _checkpoint(x)
    gy = _randn(70, 50, seed=161)
    gy[9, 7] = float("inf")
    for relu in (False, True):
        gw, gb = pkg.lmkan_linear_grad(pkg.LinearDesc(100, 50, relu=relu), codes.to(dev), exps.to(dev), gy.to(dev))
        bad = ~torch.isfinite(gw.cpu())
        assert bad[:, 32:64].all() and bad[7].all()
        bad[:, 32:64] = False
        bad[7] = False
        assert not bad.any()
        assert not torch.isfinite(gb[7]) and int(torch.isfinite(gb).sum()) == 49


# ---- adapters --------------------------------------------------------------------------------------------------------

def _adapters(batch, n_in, n_out, rank, count, w="f32", x="f32", y="f32", seed=170, index=None):
    a = (_randn(count, rank, n_in, seed=seed) / n_in ** 0.5).to(DT[w])
    b = _randn(count, n_out, rank, seed=seed + 1).to(DT[w])
    scale = 0.5 + torch.rand((count,), generator=torch.Generator().manual_seed(seed + 2))
    if index is None:
        index = torch.randint(-1, count + 1, (batch,), generator=torch.Generator().manual_seed(seed + 3)).int()   # -1 and count: none
    return _rows(batch, n_in, x, seed=seed + 4), index.int(), a, b, _randn(batch, n_out, seed=seed + 5).to(DT[y]), scale


def _check_adapters(dev, data, relu, scaled, w="f32", x_type="f32", y_type="f32"):
    x, index, a, b, y, scale = data
    count, rank, n_in = a.shape
    n_out = b.shape[1]
    desc = pkg.AdapterDesc(count, rank, n_in, n_out, dtype=CODE[w], x_dtype=CODE[x_type], y_dtype=CODE[y_type], relu=relu)
    got = y.clone().to(dev)
    out = pkg.lmkan_adapters_add(desc, x.to(dev), index.to(dev), a.to(dev), b.to(dev), got, scale=scale.to(dev) if scaled else None)
    assert out.data_ptr() == got.data_ptr()
    xd = x.double().clamp(min=0.0) if relu else x.double()
    want, size = y.double().clone(), torch.zeros(y.shape, dtype=torch.float64)
    has = (index >= 0) & (index < count)
    for r in index[has].unique().tolist():
        n = torch.nonzero(index == r)[:, 0]
        s = float(scale[r]) if scaled else 1.0
        ad, bd = a[r].double(), b[r].double()
        want[n] += s * ((xd[n] @ ad.T) @ bd.T)
        size[n] = s * ((xd[n].abs() @ ad.abs().T) @ bd.abs().T)
    assert torch.equal(got[~has].cpu(), y[~has])                       # bit for bit
    _within(got[has], want[has], ((n_in + rank + 16) * U * size + 2 * U * want.abs() + _out(want, y_type))[has], "y")
    return desc, got


ADAPTERS = [(1, 1, 1, 1, 1), (1, 64, 64, 8, 4), (1, 4096, 100, 16, 3), (3, 37, 19, 5, 2), (16, 128, 128, 16, 4), (17, 130, 70, 17, 3), (48, 256, 300, 33, 20),
            (65, 100, 33, 64, 65), (200, 64, 500, 100, 5), (130, 500, 40, 256, 2), (1000, 96, 72, 7, 300), (600, 1000, 16, 1, 1), (33, 7, 1100, 128, 1),
            (2049, 40, 24, 12, 6), (300, 16, 16, 4, 8192), (3000, 64, 48, 8, 8192), (40000, 24, 20, 3, 50)]


@pytest.mark.parametrize("shape", ADAPTERS, ids=str)
def test_adapters_match_float64(dev, shape):
    data = _adapters(*shape)
    _check_adapters(dev, data, relu=False, scaled=True)
    _check_adapters(dev, data, relu=True, scaled=False)


@pytest.mark.parametrize("w", TYPES)
@pytest.mark.parametrize("x", TYPES)
@pytest.mark.parametrize("y", TYPES)
def test_adapters_in_every_type(dev, w, x, y):
    for shape in [(5, 100, 60, 6, 3), (70, 128, 96, 16, 3), (300, 64, 130, 40, 2)]:
        _check_adapters(dev, _adapters(*shape, w=w, x=x, y=y, seed=190), True, True, w, x, y)


@pytest.mark.parametrize("rank", [1, 6, 8, 16, 20, 32, 48, 64, 65, 100, 128, 129, 200, 256])
@pytest.mark.parametrize("types", ["f32 f32 f32", "bf16 bf16 bf16", "f16 f16 f32", "bf16 f32 f32", "f32 f16 bf16"])
def test_adapters_of_every_rank_with_many_rows(dev, rank, types):
    """More rows than one launch takes: sorted by adapter, a few hundred of each and some tiles not full."""
    w, x, y = types.split()
    for n_in, n_out, relu in [(256, 160, True), (333, 77, False), (1200, 520, False)]:
        _check_adapters(dev, _adapters(700, n_in, n_out, rank, 3, w=w, x=x, y=y, seed=195), relu, True, w, x, y)


@pytest.mark.parametrize("kind", ["one", "none", "runs", "last", "beyond"])
def test_arrangements_of_requests(dev, kind):
    batch, count = 500, 9
    index = {"one": torch.full((batch,), 4), "none": torch.full((batch,), -1), "runs": torch.arange(batch) // 77, "last": torch.where(torch.arange(batch) == 499, 8, -1),
             "beyond": torch.tensor([-2 ** 31, 2 ** 31 - 1, 9, 8, 0])[torch.arange(batch) % 5]}[kind]
    _check_adapters(dev, _adapters(batch, 80, 50, 10, count, index=index, seed=200), False, True)


def test_adapters_with_values_that_are_not_finite_stay_in_their_rows(dev):
    data = _adapters(40, 60, 30, 6, 3, seed=210, index=torch.arange(40) % 3)
    x, index, a, b, y, scale = data
    desc, clean = _check_adapters(dev, data, False, True)
    x, a = x.clone(), a.clone()
    x[7, 5] = float("nan")
    a[2, 0, 0] = float("inf")
    got = pkg.lmkan_adapters_add(desc, x.to(dev), index.to(dev), a.to(dev), b.to(dev), y.clone().to(dev), scale=scale.to(dev))
    for n in range(40):
        if n == 7:
            assert torch.isnan(got[n]).all()
        elif n % 3 == 2:
            assert not torch.isfinite(got[n]).any()
        else:
            assert torch.equal(got[n], clean[n])


@pytest.mark.parametrize("types", ["f32 f32 f32", "bf16 bf16 bf16", "f16 f16 f32", "f32 f16 bf16"])
def test_many_rows_with_values_that_are_not_finite_stay_in_their_rows(dev, types):
    w, x_type, y_type = types.split()
    data = _adapters(900, 128, 64, 24, 3, w=w, x=x_type, y=y_type, seed=212, index=torch.arange(900) % 3)
    x, index, a, b, y, scale = data
    desc, clean = _check_adapters(dev, data, False, True, w, x_type, y_type)
    x, a, b, y = x.clone(), a.clone(), b.clone(), y.clone()
    x[7, 5] = float("nan")
    x[9, 127] = float("-inf")
    a[2, 0, 0] = float("inf")
    b[1, 63, 23] = float("inf")
    y[12, 3] = float("nan")
    got = pkg.lmkan_adapters_add(desc, x.to(dev), index.to(dev), a.to(dev), b.to(dev), y.to(dev), scale=scale.to(dev)).cpu()
    bad = ~torch.isfinite(got)
    want = torch.zeros(900, 64, dtype=torch.bool)
    want[7] = want[9] = want[2::3] = True
    want[1::3, 63] = want[12, 3] = True
    assert torch.equal(bad, want)
    assert torch.equal(got[~want], clean.cpu()[~want])


@pytest.mark.parametrize("small", ["x", "a", "b"])
@pytest.mark.parametrize("batch", [6, 900])
def test_float16_numbers_below_the_smallest_normal_one_count(dev, small, batch):
    """Multiples of 2^-24 are factors like any other."""
    x, index, a, b, y, scale = _adapters(batch, 128, 64, 16, 3, w="f16", x="f16", y="f32", seed=215, index=torch.arange(batch) % 3)
    tiny = {"x": x, "a": a, "b": b}[small]
    tiny.copy_(tiny * 2.0 ** -18)
    _check_adapters(dev, (x, index, a, b, torch.zeros_like(y), scale), False, True, "f16", "f16", "f32")


# ---- all of them -----------------------------------------------------------------------------------------------------

def _guarded(t, dev, shift):
    """A copy of `t` that starts `shift` elements into a buffer of its own, and a check of what lies around it."""
    n = t.numel()
    fill = 77
    buf = torch.full((n + shift + 64,), fill, dtype=t.dtype, device=dev)
    view = buf[shift:shift + n].view(t.shape)
    view.copy_(t.to(dev))
    return view, lambda: bool((buf[:shift] == fill).all()) and bool((buf[shift + n:] == fill).all())


@pytest.mark.parametrize("shape", [(3, 40), (37, 129), (70, 1024), (2, 9001)], ids=str)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shift", [1, 3, 8])
def test_pointers_anywhere_and_nothing_written_beyond(dev, shape, dtype, shift):
    """Tensors that start on an element's boundary only: the same results, and nothing around an output changes."""
    rows, cols = shape
    code, n_out = CODE[dtype], 37
    x, w, b = _rows(rows, cols, dtype, seed=220).to(dev), _randn(cols, seed=221).to(dev), _randn(cols, seed=222).to(dev)
    gy, gl = (1e-3 * _randn(rows, cols, seed=223)).to(DT[dtype]).to(dev), _randn(rows, n_out, seed=224).to(DT[dtype]).to(dev)
    desc, linear = pkg.NormDesc(cols, x_dtype=code, y_dtype=code), pkg.LinearDesc(cols, n_out, y_dtype=code)
    adapters = pkg.AdapterDesc(2, 5, cols, n_out, dtype=code, x_dtype=code, y_dtype=code)
    a, bb = _randn(2, 5, cols, seed=225).to(DT[dtype]).to(dev), _randn(2, n_out, 5, seed=226).to(DT[dtype]).to(dev)
    index = (torch.arange(rows) % 2).int().to(dev)
    y, stats, kept = pkg.lmkan_layer_norm(desc, x, w, b, keep=True)
    gx, gw, gb = pkg.lmkan_layer_norm_backward(desc, gy, stats, x=x, weight=w)
    back = pkg.lmkan_restore_rows(*kept, weight=w, bias=b, dtype=code)
    lw, lb = pkg.lmkan_linear_grad(linear, *kept, gl)
    added = pkg.lmkan_adapters_add(adapters, x, index, a, bb, gl.clone())
    put = lambda t: _guarded(t, dev, shift)[0]
    checks = []

    def out(like):
        view, check = _guarded(torch.zeros_like(like), dev, shift)
        checks.append(check)
        return view
    y2, stats2, kept2 = pkg.lmkan_layer_norm(desc, put(x), put(w), put(b), y=out(y), keep=True)
    moved = put(kept[0]), put(kept[1])
    gx2, gw2, gb2 = pkg.lmkan_layer_norm_backward(desc, put(gy), put(stats), x=put(x), weight=put(w), grad_x=out(gx), grad_weight=out(gw), grad_bias=out(gb))
    back2 = pkg.lmkan_restore_rows(*moved, weight=put(w), bias=put(b), dtype=code, y=out(back))
    lw2, lb2 = pkg.lmkan_linear_grad(linear, *moved, put(gl), grad_weight=out(lw), grad_bias=out(lb))
    added2, check = _guarded(gl, dev, shift)
    checks.append(check)
    pkg.lmkan_adapters_add(adapters, put(x), put(index), put(a), put(bb), added2)
    for got, want in [(y2, y), (stats2, stats), (kept2[0], kept[0]), (kept2[1], kept[1]), (back2, back)]:
        assert torch.equal(got, want)
    # sums whose order may go by the alignment: both within their bounds of the exact sum
    hat = (x.cpu().double() - stats[:, :1].cpu().double()) * stats[:, 1:].cpu().double()
    g, k = gy.cpu().double(), 2 * (min(rows, 1300) + 11) * U
    want, tol = _norm_gradients(hat, stats[:, 1:].cpu().double(), g, w.cpu().double())
    _within(gx2, gx.cpu().double(), 2 * tol + 2 * _out(want, dtype), "grad_x")
    _within(gw2, gw.cpu().double(), k * (g * hat).abs().sum(dim=0), "grad_weight")
    _within(gb2, gb.cpu().double(), k * g.abs().sum(dim=0), "grad_bias")
    v, g = _values(kept[0].cpu(), kept[1].cpu()), gl.cpu().double()
    _within(lw2, lw.cpu().double(), 2 * (rows / 4 + 64) * U * torch.sqrt(g.square().T @ v.square()), "the linear term's weight")
    _within(lb2, lb.cpu().double(), 2 * (rows / 4 + 64) * U * g.square().sum(dim=0).sqrt(), "the linear term's bias")
    r = index.cpu().long()
    low = torch.einsum("nki,ni->nk", a.cpu().double().abs()[r], x.cpu().double().abs())
    size = torch.einsum("njk,nk->nj", bb.cpu().double().abs()[r], low)
    _within(added2, added.cpu().double(), 2 * ((cols + 5 + 16) * U * size + 2 * U * added.cpu().double().abs() + _out(added.cpu().double(), dtype)), "y")
    assert all(c() for c in checks)


def _chain(dev, rows=96, n_in=64, n_out=40, seed=230):
    """Norm, linear term, adapters and both backward calls, as a program makes them; returns a function of nothing."""
    x, w, b = _rows(rows, n_in, seed=seed).to(dev), (1 + 0.1 * _randn(n_in, seed=seed + 1)).to(dev), _randn(n_in, seed=seed + 2).to(dev)
    weight, gy = _randn(n_out, n_in, seed=seed + 3).to(dev), (1e-2 * _randn(rows, n_out, seed=seed + 4)).to(dev)
    norm, linear = pkg.NormDesc(n_in), pkg.LinearDesc(n_in, n_out, relu=True)
    adapters = pkg.AdapterDesc(3, 8, n_in, n_out, relu=True)
    a, up = _randn(3, 8, n_in, seed=seed + 5).to(dev), _randn(3, n_out, 8, seed=seed + 6).to(dev)
    index = (torch.arange(rows) % 4 - 1).int().to(dev)
    codes, scale = pkg.lmkan_quantize_rows(weight)

    def run(stream=None):
        z, stats, kept = pkg.lmkan_layer_norm(norm, x, w, b, keep=True, stream=stream)
        z_kept = pkg.lmkan_checkpoint_rows(z, stream=stream)
        y = pkg.lmkan_linear_i8(linear, z, codes, scale, stream=stream)
        pkg.lmkan_adapters_add(adapters, z, index, a, up, y, stream=stream)
        grad_weight, grad_bias = pkg.lmkan_linear_grad(linear, *z_kept, gy, stream=stream)
        back = pkg.lmkan_restore_rows(*z_kept, stream=stream)
        grad_x, grad_w, grad_b = pkg.lmkan_layer_norm_backward(norm, back, stats, kept=kept, weight=w, stream=stream)
        return z, y, grad_weight, grad_bias, back, grad_x, grad_w, grad_b
    return run


@pytest.mark.parametrize("rows", [96, 3000])
def test_chain_on_other_streams(dev, rows):
    run = _chain(dev, rows)
    want = run()
    torch.cuda.synchronize()
    side, other = torch.cuda.Stream(), torch.cuda.Stream()
    first, second = run(stream=side), run(stream=other)             # two at once
    with torch.cuda.stream(side):
        third = run()
    torch.cuda.synchronize()
    for got in (first, second, third):
        assert all(torch.equal(g, t) for g, t in zip(got, want))


@pytest.mark.parametrize("rows", [96, 3000])
def test_chain_in_a_graph(dev, rows):
    run = _chain(dev, rows)
    want = run()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    for _ in range(4):
        for g in got:
            g.fill_(7)
        graph.replay()
        assert all(torch.equal(g, t) for g, t in zip(run(), want))      # eager work between replays
        torch.cuda.synchronize()
        assert all(torch.equal(g, t) for g, t in zip(got, want))


def test_chain_against_autograd(dev):
    """A normalised linear layer's gradients through both backward calls from checkpoints, against autograd in float64 on the
    values that the checkpoints stand for."""
    rows, n_in, n_out = 150, 96, 50
    x, w, b = _rows(rows, n_in, seed=240), 1 + 0.1 * _randn(n_in, seed=241), 0.1 * _randn(n_in, seed=242)
    weight, gy = _randn(n_out, n_in, seed=243), 1e-2 * _randn(rows, n_out, seed=244)
    z, stats, kept = pkg.lmkan_layer_norm(pkg.NormDesc(n_in), x.to(dev), w.to(dev), b.to(dev), keep=True)
    z_kept = pkg.lmkan_checkpoint_rows(z)
    gw, gb = pkg.lmkan_linear_grad(pkg.LinearDesc(n_in, n_out, relu=True), *z_kept, gy.to(dev))
    zv = _values(z_kept[0].cpu(), z_kept[1].cpu()).requires_grad_()
    wd, bd = weight.double().requires_grad_(), torch.zeros(n_out, dtype=torch.float64, requires_grad=True)
    y = zv.clamp(min=0.0) @ wd.T + bd
    y.backward(gy.double())
    # as in test_linear_grad: (n / 4 + 64) u of the root of the sum of squares; relative to the whole
    assert float((gw.cpu().double() - wd.grad).norm() / wd.grad.norm()) <= (rows / 4 + 64) * U * 2
    assert float((gb.cpu().double() - bd.grad).norm() / bd.grad.norm()) <= (rows / 4 + 64) * U * 2
    gz = zv.grad.float()
    gx, gnw, gnb = pkg.lmkan_layer_norm_backward(pkg.NormDesc(n_in), gz.to(dev), stats, kept=kept, weight=w.to(dev))
    hat = _values(kept[0].cpu(), kept[1].cpu())
    want, tol = _norm_gradients(hat, stats[:, 1:].cpu().double(), gz.double(), w.double())
    _within(gx, want, tol + _out(want, "f32"))
    # and against the rows themselves: hat is off by 1/127 of a block's largest element at most, here a hundredth of the norm
    exact = x.double().requires_grad_()
    torch.nn.functional.layer_norm(exact, (n_in,), w.double(), b.double(), EPS).backward(gz.double())
    assert float((gx.cpu().double() - exact.grad).norm() / exact.grad.norm()) <= 0.01


def test_normalised_layer_of_the_example(dev):
    """The example's training step runs, and its gradients are those of the formulas at the values that the checkpoint
    stands for; its answers with adapters are the plain ones plus the adapters' products."""
    from paper_2509_07103_amd import preconditioned
    losses, off = preconditioned.run(3, 256, 32, 24, 7, normalised=True)
    assert len(losses) == 3 and all(np.isfinite(losses)) and off < 0.1
    rows, n_in, n_out = 200, 64, 40
    model = preconditioned.NormalisedLayer(n_in, n_out, 8, 0.3, dev)
    x, gy = _rows(rows, n_in, seed=250), 1e-2 * _randn(rows, n_out, seed=251)
    _, saved = model.forward(x.to(dev))
    grad_x, grad_table, grad_weight = model.gradients(saved, gy.to(dev))
    stats, kept = saved
    z = _values(kept[0].cpu(), kept[1].cpu())
    w, g = model.weight.cpu().double(), gy.double()
    relu = z.clamp(min=0.0)
    _within(grad_weight, g.T @ relu, (rows / 4 + 64) * U * torch.sqrt(g.square().T @ relu.square()) + 1e-44, "grad_weight")
    # (a table of zeros: the layer itself passes nothing back); the product of float32 on the way is off by n_out u of the
    # magnitudes, which the norm's backward pass takes to at most three times that of a row
    gz = (g @ w) * (z > 0)
    want, tol = _norm_gradients(z, stats[:, 1:].cpu().double(), gz, None)
    size = (g.abs() @ w.abs()).amax(dim=1, keepdim=True) * stats[:, 1:].cpu().double() * (1 + z.abs())
    _within(grad_x, want, tol + 3 * n_out * U * size, "grad_x")
    _, table = pkg.lmkan_backward(model.layer, pkg.lmkan_restore_rows(*kept), model.table, (0.3 * gy).to(dev), need_grad_x=False)
    assert float((table - grad_table).norm() / table.norm()) <= 1e-5
    model.freeze()
    adapters = preconditioned.random_adapters(3, 8, n_in, n_out, dev)
    index = (torch.arange(rows) % 4 - 1).int()
    plain, adapted = model.answer(x.to(dev)), model.answer(x.to(dev), adapters, index.to(dev))
    assert torch.equal(plain[::4], adapted[::4])                        # no adapter
    zf, _, _ = pkg.lmkan_layer_norm(model.norm, x.to(dev))
    zd, a, b = zf.cpu().double().clamp(min=0.0), adapters[1].cpu().double(), adapters[2].cpu().double()
    for n in range(1, rows, 17):
        r = int(index[n])
        if r >= 0:
            add = b[r] @ (a[r] @ zd[n])
            size = b[r].abs() @ (a[r].abs() @ zd[n])
            want = plain[n].cpu().double() + add
            _within(adapted[n], want, (n_in + 8 + 16) * U * size + 2 * U * want.abs())


def test_offsets_beyond_32_bits(dev):
    """Matrices of more than 2^31 elements: their last rows come out as they do alone."""
    rows, cols, last = 16 * 1024 + 256, 131070, 4
    gen = torch.Generator(device=dev).manual_seed(260)
    x = torch.empty((rows, cols), dtype=torch.float16, device=dev).normal_(generator=gen)
    end = x[-last:]                                                     # (aligned as the first row is)
    assert x.numel() > 2 ** 31 and end.data_ptr() % 16 == x.data_ptr() % 16
    desc = pkg.NormDesc(cols, x_dtype=pkg.LMKAN_F16, y_dtype=pkg.LMKAN_F16)
    y, stats, kept = pkg.lmkan_layer_norm(desc, x, keep=True)
    y_end, stats_end, kept_end = pkg.lmkan_layer_norm(desc, end, keep=True)
    for got, want in [(y, y_end), (stats, stats_end), (kept[0], kept_end[0]), (kept[1], kept_end[1])]:
        assert torch.equal(got[-last:], want)
    codes, exps = pkg.lmkan_checkpoint_rows(x, relu=True)
    of_end = pkg.lmkan_checkpoint_rows(end, relu=True)
    assert torch.equal(codes[-last:], of_end[0]) and torch.equal(exps[-last:], of_end[1])
    pkg.lmkan_restore_rows(codes, exps, dtype=pkg.LMKAN_F16, y=y)
    assert torch.equal(y[-last:], pkg.lmkan_restore_rows(*of_end, dtype=pkg.LMKAN_F16))
    for given in ({"x": x}, {"kept": kept}):
        alone = {"x": end} if "x" in given else {"kept": kept_end}
        grad_x, grad_weight, grad_bias = pkg.lmkan_layer_norm_backward(desc, y, stats, **given)
        assert torch.equal(grad_x[-last:], pkg.lmkan_layer_norm_backward(desc, y[-last:], stats_end, **alone)[0])
        del grad_x
    # one row that is not zero: each sum is one product
    linear = pkg.LinearDesc(cols, 3)
    gy = torch.zeros((rows, 3), device=dev)
    gy[-1] = torch.tensor([1.5, -0.3, 7.0], device=dev)
    for got, want in zip(pkg.lmkan_linear_grad(linear, codes, exps, gy), pkg.lmkan_linear_grad(linear, of_end[0], of_end[1], gy[-last:])):
        assert torch.equal(got, want)
    y.zero_()                                                           # .. and with the gradient's own offsets
    y[-1] = x[0]
    few = pkg.lmkan_checkpoint_rows(_randn(rows, 3, seed=261).to(dev))
    got = pkg.lmkan_linear_grad(pkg.LinearDesc(3, cols, y_dtype=pkg.LMKAN_F16), *few, y)[0]
    assert torch.equal(got, x[0].float()[:, None] * pkg.lmkan_restore_rows(*few)[-1])   # (11 bits times 7: exact)
    # adapters: n_in u of the sum of magnitudes and the rest, as ever
    a = (_randn(2, 3, cols, seed=262) / cols ** 0.5).half()
    b, index = _randn(2, 5, 3, seed=263).half(), torch.arange(rows, dtype=torch.int32) % 2
    out = pkg.lmkan_adapters_add(pkg.AdapterDesc(2, 3, cols, 5, dtype=pkg.LMKAN_F16, x_dtype=pkg.LMKAN_F16), x, index.to(dev), a.to(dev), b.to(dev),
                                 torch.zeros((rows, 5), device=dev))
    for n in list(range(3)) + list(range(rows - 3, rows)):
        xd, ad, bd = x[n].cpu().double(), a[n % 2].double(), b[n % 2].double()
        size = bd.abs() @ (ad.abs() @ xd.abs())
        _within(out[n], bd @ (ad @ xd), (cols + 3 + 16) * U * size, f"row {n}")
