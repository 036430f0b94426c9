"""The operators of the dense matrices at the ends of their documented ranges: sizes, magnitudes, schedules.

Tolerances are those of test_gpu_dense.py: 4e-5 of the result's norm for five steps, and the unit roundoff of a
16-bit result."""
import numpy as np
import pytest
import torch

import paper_2509_07103_amd as pkg
from test_gpu_dense import CODE, DT, TOL, UNIT, _codes, _far, _gradient, _reference, _rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    pkg.lib()
    return torch.device("cuda:0")


def _polynomial(gram, schedule):
    """The matrix P of X_k = P X_0 from the Gram matrix of X_0, float64."""
    p = torch.eye(gram.shape[0], dtype=torch.float64, device=gram.device)
    for a, b, c in schedule:
        a, b, c = (float(torch.tensor(v, dtype=torch.float32)) for v in (a, b, c))
        step = b * gram + c * gram @ gram
        step.diagonal().add_(a)
        gram = step @ gram @ step
        p = step @ p
    return p


def test_rows_of_more_than_2_to_the_25(dev):
    """A panel of X by columns is longer than 4 GiB: n a little over 2^25 (8.7 GB a matrix, 44 GB in all)."""
    m, n = 65, (1 << 25) + 10
    g = torch.Generator(device=dev).manual_seed(1)
    x = torch.randn((1, m, n), device=dev, generator=g)
    pieces = [(c, min(c + (1 << 20), n)) for c in range(0, n, 1 << 20)]
    gram = torch.zeros((m, m), dtype=torch.float64, device=dev)
    for c, d in pieces:
        v = x[0, :, c:d].double()
        gram += v @ v.t().contiguous()
    norm = float(gram.trace()) ** 0.5 + 1e-7
    p = _polynomial(gram / norm ** 2, pkg.QUINTIC_SCHEDULE) / norm
    got = pkg.lmkan_orthogonalize(pkg.MatrixDesc(1, m, n), x)
    worst = 0.0
    for c, d in pieces:
        want = p @ x[0, :, c:d].double()
        off = got[0, :, c:d].double() - want
        whole = (d - c) // 64 * 64                      # 64 columns at a time: a tile's
        for part in (slice(0, whole), slice(whole, d - c)):
            if part.start < part.stop:
                o, w = (t[:, part].reshape(m, -1, min(64, part.stop - part.start)).square().sum(dim=(0, 2)) for t in (off, want))
                worst = max(worst, float((o / w).max()) ** 0.5)
    assert worst <= TOL


def test_more_matrices_than_a_launch_takes(dev):
    """2^21 matrices of one workgroup each to a launch: the second launch starts where the first ended."""
    n = (1 << 21) + 77
    g = torch.Generator(device=dev).manual_seed(2)
    x = torch.randn((n, 1, 3), device=dev, generator=g)

    def steps(v):
        v = v / (v.norm(dim=2, keepdim=True) + 1e-7)
        for a, b, c in pkg.QUINTIC_SCHEDULE:
            s2 = v.square().sum(dim=2, keepdim=True)
            v = (a + b * s2 + c * s2 * s2) * v
        return v
    want = steps(x.double())
    got = pkg.lmkan_orthogonalize(pkg.MatrixDesc(n, 1, 3), x)
    assert float(((got.double() - want).norm(dim=2) / want.norm(dim=2)).max()) <= TOL
    m, w = torch.zeros_like(x), x.clone()
    pkg.lmkan_muon_step(pkg.MatrixDesc(n, 1, 3), pkg.MuonParams(lr=0.5, momentum=0.5, nesterov=False), x, m, w)
    assert torch.equal(m, 0.5 * x)
    want = steps(0.5 * x.double())
    off = (w.double() - (x.double() - 0.5 * want)).norm(dim=2)
    assert bool((off <= 4 * 2.0 ** -24 * x.double().norm(dim=2) + 0.5 * TOL * want.norm(dim=2)).all())


@pytest.mark.parametrize("rows,cols", [((1 << 23) + 21, 3), ((1 << 21) + 13, 2049)])
def test_more_rows_than_a_launch_takes(dev, rows, cols):
    """Four rows of up to 2048 values to a workgroup, or one longer one, 2^21 workgroups to a launch."""
    g = torch.Generator(device=dev).manual_seed(3)
    x = torch.empty((rows, cols), dtype=torch.float16, device=dev).normal_(generator=g)
    codes, scale = pkg.lmkan_quantize_rows(x)
    for at in range(0, rows, 1 << 19):
        v = x[at:at + (1 << 19)].float()
        top = v.abs().amax(dim=1, keepdim=True)
        full = torch.full_like(top, 127.0)
        f = torch.where(top > 0, full / top, torch.zeros_like(top))
        assert torch.equal(codes[at:at + (1 << 19)].float(), torch.round(v * f))
        assert torch.equal(scale[at:at + (1 << 19)], (top / full)[:, 0])


def test_linear_i8_of_more_rows_and_weights_than_a_launch_takes(dev):
    """Rows to codes in two launches, and weights to aligned rows in two."""
    for batch, n_in, n_out in (((1 << 23) + 21, 3, 2), (70, 2051, (1 << 20) + 5)):
        g = torch.Generator(device=dev).manual_seed(4)
        x = torch.empty((batch, n_in), dtype=torch.float16, device=dev).normal_(generator=g)
        w = torch.randint(-127, 128, (n_out, n_in), device=dev, generator=g, dtype=torch.int8)
        ws = torch.rand((n_out,), device=dev, generator=g)
        got = pkg.lmkan_linear_i8(pkg.LinearDesc(n_in, n_out, pkg.LMKAN_F16, pkg.LMKAN_F32), x, w, ws)
        codes, scale = pkg.lmkan_quantize_rows(x)
        codes = codes.float()                            # sums below 2^24 or exact in float64
        for at in range(0, n_out, 1 << 17):
            for r in range(0, batch, 1 << 21):
                part = slice(r, r + (1 << 21)), slice(at, at + (1 << 17))
                want = codes[part[0]].double() @ w[part[1]].double().t().contiguous() * scale[part[0]].double()[:, None] * ws[part[1]].double()
                off = (got[part].double() - want).abs()
                assert bool((off <= 4 * 2.0 ** -24 * want.abs() + 1e-30).all())


def _on_device(x, schedule, eps=1e-7):
    """_reference for larger shapes: the same steps in float64 on the device, factors contiguous."""
    x = x.double()
    flip = x.shape[1] > x.shape[2]
    x = x.mT.contiguous() if flip else x
    x = x / (x.square().sum(dim=(1, 2), keepdim=True).sqrt() + eps)
    for a, b, c in np.asarray(schedule, dtype=np.float32).astype(np.float64).reshape(-1, 3):
        gram = x @ x.mT.contiguous()
        x = a * x + (b * gram + c * gram @ gram) @ x
    return x.mT.contiguous() if flip else x


# short sides above 512 with 128 tiles of 256 or more, 257 to 512 with 512 tiles of 128; joins of both
@pytest.mark.parametrize("shape", [(1, 4097, 4099), (16, 1025, 1100), (40, 700, 513), (100, 300, 420), (90, 500, 290)],
                         ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_orthogonalize_in_the_larger_tiles(dev, shape, dtype):
    g = torch.Generator(device=dev).manual_seed(sum(shape))
    x = torch.randn(shape, device=dev, generator=g)
    x += 0.5 * torch.randn((*shape[:2], 2), device=dev, generator=g) @ torch.randn((shape[0], 2, shape[2]), device=dev, generator=g)
    x = x.to(DT[dtype])
    got = pkg.lmkan_orthogonalize(pkg.MatrixDesc(*shape, dtype=CODE[dtype]), x)
    assert _far(got, _on_device(x, pkg.QUINTIC_SCHEDULE).cpu()) <= TOL + (UNIT[dtype] if dtype != "f32" else 0.0)
    assert torch.equal(got, pkg.lmkan_orthogonalize(pkg.MatrixDesc(*shape, dtype=CODE[dtype]), x))


@pytest.mark.parametrize("shape", [(16500, 65, 66), (16390, 70, 68), (32800, 1, 4097), (32780, 4100, 2)], ids=lambda s: "x".join(map(str, s)))
def test_batches_in_parts(dev, shape):
    """More matrices than share the workspace at a time."""
    g = torch.Generator(device=dev).manual_seed(6)
    grad = torch.randn(shape, device=dev, generator=g).to(torch.bfloat16)
    m, w = torch.randn(shape, device=dev, generator=g), torch.zeros(shape, device=dev)
    held = m.clone()
    p = pkg.MuonParams(lr=0.5, momentum=0.5, nesterov=True)
    pkg.lmkan_muon_step(pkg.MatrixDesc(*shape, dtype=pkg.LMKAN_BF16), p, grad, m, w)
    for at in range(0, shape[0], 2048):
        part = slice(at, at + 2048)
        moved = 0.5 * held[part].double() + 0.5 * grad[part].double()
        assert float((m[part].double() - moved).abs().max()) <= 4 * 2.0 ** -24 * float(held.abs().max() + grad.abs().max())
        want = -0.5 * _on_device(0.5 * moved + 0.5 * grad[part].double(), pkg.QUINTIC_SCHEDULE)
        assert _far(w[part], want.cpu()) <= TOL


@pytest.mark.parametrize("batch,n_in,n_out", [(8200, 1000, 1030), (4097, 2050, 2052), (9001, 16, 1025), (3000, 333, 4101)])
@pytest.mark.parametrize("x_dtype,y_dtype", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f32")])
@pytest.mark.parametrize("relu,bias,beta", [(False, False, 0.0), (True, True, 0.25)])
def test_linear_i8_in_the_larger_tiles(dev, batch, n_in, n_out, x_dtype, y_dtype, relu, bias, beta):
    """512 tiles of 128 and more."""
    g = torch.Generator().manual_seed(batch + n_in + n_out)
    x = _rows(batch, n_in, 41, x_dtype)
    w = torch.randint(-127, 128, (n_out, n_in), generator=g, dtype=torch.int8)
    ws = (0.5 + torch.rand((n_out,), generator=g)) / (73.0 * n_in ** 0.5)
    b = torch.randn((n_out,), generator=g).to(dev) if bias else None
    y = torch.randn((batch, n_out), generator=g).to(DT[y_dtype]).to(dev) if beta else None
    codes, _ = _codes(x, relu)
    top = x.float().clamp(min=0) if relu else x.float().abs()
    want = torch.from_numpy(codes).to(dev).double() @ w.to(dev).double().t().contiguous()
    want *= (top.amax(dim=1).double()[:, None] / 127.0).to(dev) * ws.to(dev).double()
    size = want.abs()
    if bias:
        want, size = want + b.double(), size + b.double().abs()
    if beta:
        want, size = want + beta * y.double(), size + beta * y.double().abs()
    got = pkg.lmkan_linear_i8(pkg.LinearDesc(n_in, n_out, CODE[x_dtype], CODE[y_dtype], relu=relu), x.to(dev), w.to(dev), ws.to(dev),
                              bias=b, beta=beta, y=y)
    most = 8 * 2.0 ** -24 * size + (UNIT[y_dtype] if y_dtype != "f32" else 0.0) * want.abs() * 1.001
    off = (got.double() - want).abs()
    assert bool((off <= most + 1e-30).all()), float((off / (most + 1e-30)).max())


SHRINKING = [[(0.0, 0.0, 0.0)], [(0.0, 0.0, 0.0)] + list(pkg.QUINTIC_SCHEDULE[:2]), list(pkg.QUINTIC_SCHEDULE[:2]) + [(0.0, 0.0, 0.0)],
             [(1e-20, 0.0, 0.0)], [(1e-20, 0.0, 0.0), (2.0, -1.5, 0.5)], [(1e-12, -5e-13, 0.0), (1e-12, 0.0, 0.0), (60.0, 0.0, 0.0)],
             [(0.0, 1e-3, 0.0)] * 2, [(1.5, -0.5, 0.0)] * 2 + [(1e-19, 0.0, 0.0)] * 2, [(0.5, 0.0, 0.0)] * 32]


@pytest.mark.parametrize("schedule", SHRINKING, ids=range(len(SHRINKING)))
@pytest.mark.parametrize("shape", [(3, 24, 40), (3, 40, 70), (2, 64, 64), (1, 48, 6000), (1, 30, 6000), (2, 100, 70), (2, 150, 130), (1, 600, 700)],
                         ids=lambda s: "x".join(map(str, s)))
def test_schedules_that_shrink(dev, schedule, shape):
    """Steps of nothing, and steps that take singular values down to 1e-38."""
    x = _gradient(*shape, seed=15)
    got = pkg.lmkan_orthogonalize(pkg.MatrixDesc(*shape), x.to(dev), schedule=schedule)
    want = _reference(x, schedule)
    if not want.any():
        assert torch.equal(got.cpu(), torch.zeros_like(x))
    else:
        assert _far(got, want) <= TOL


SMALL = [(3, 16, 8), (2, 40, 70), (3, 64, 64), (1, 3, 5000), (1, 64, 6000), (6000, 30, 1), (1, 1, 70001)]


@pytest.mark.parametrize("scale,eps", [(1e-18, 1e-30), (1e-24, 1e-30), (1e-30, 1e-36), (1e-36, 1e-40), (1e-24, 1e-24)])
@pytest.mark.parametrize("shape", SMALL + [(2, 65, 70), (2, 250, 333)], ids=lambda s: "x".join(map(str, s)))
def test_small_magnitudes_with_a_smaller_eps(dev, shape, scale, eps):
    """Squares below float32's range; eps is a float32 value.  (Denormals hold fewer bits: they are the input here.)"""
    x = _gradient(*shape, seed=14, scale=scale)
    got = pkg.lmkan_orthogonalize(pkg.MatrixDesc(*shape, eps=eps), x.to(dev))
    assert _far(got, _reference(x, pkg.QUINTIC_SCHEDULE, float(np.float32(eps)))) <= TOL


@pytest.mark.parametrize("shape", [(1, 3, 5000), (1, 64, 6000), (2, 40, 70), (1, 70, 6000)], ids=lambda s: "x".join(map(str, s)))
def test_magnitudes_that_differ_within_a_matrix(dev, shape):
    """Small, ordinary and large columns, in this and the other order: the norm is that of the largest."""
    n = shape[2]
    for order in ((1e-28, 1.0, 1e25), (1e25, 1.0, 1e-28), (1e-28, 1e-27, 1e-28), (1.0, 1e-28, 1.0)):
        x = _gradient(*shape, seed=16, scale=1.0)
        for k, s in enumerate(order):
            x[:, :, k * n // 3:(k + 1) * n // 3] *= s
        got = pkg.lmkan_orthogonalize(pkg.MatrixDesc(*shape, eps=1e-36), x.to(dev))
        assert _far(got, _reference(x, pkg.QUINTIC_SCHEDULE, float(np.float32(1e-36)))) <= TOL


@pytest.mark.parametrize("shape", SMALL + [(2, 65, 70), (2, 250, 333)], ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("steps", [0, 5])
def test_the_largest_magnitudes(dev, shape, steps):
    """Norms beyond float32."""
    x = _gradient(*shape, seed=17, scale=1.0)
    x *= 3e38 / x.abs().max()
    got = pkg.lmkan_orthogonalize(pkg.MatrixDesc(*shape), x.to(dev), schedule=pkg.QUINTIC_SCHEDULE[:steps])
    assert _far(got, _reference(x, pkg.QUINTIC_SCHEDULE[:steps])) <= TOL


@pytest.mark.parametrize("steps", [0, 1, 5])
@pytest.mark.parametrize("eps", [1e-38, 1e-39, 1e-42, 1e-45])
@pytest.mark.parametrize("shape", SMALL + [(2, 65, 70), (2, 250, 333)], ids=lambda s: "x".join(map(str, s)))
def test_zeros_with_the_smallest_eps(dev, shape, eps, steps):
    got = pkg.lmkan_orthogonalize(pkg.MatrixDesc(*shape, eps=eps), torch.zeros(shape, device=dev), schedule=pkg.QUINTIC_SCHEDULE[:steps])
    assert torch.equal(got, torch.zeros_like(got))


@pytest.mark.parametrize("scale", [1e-9, 1e-12, 1e-15, 1e-20])
@pytest.mark.parametrize("shape", [(2, 40, 70), (2, 65, 70), (3, 100, 90), (1, 1500, 96), (2, 250, 333), (1, 600, 700)], ids=lambda s: "x".join(map(str, s)))
def test_gradients_far_below_eps(dev, shape, scale):
    """|U| << eps: X_0 is small and the steps multiply it by a, every product with 22 bits all the same."""
    x = _gradient(*shape, seed=18, scale=scale)
    got = pkg.lmkan_orthogonalize(pkg.MatrixDesc(*shape), x.to(dev))
    assert _far(got, _reference(x, pkg.QUINTIC_SCHEDULE, float(np.float32(1e-7)))) <= TOL


LARGE_FACTORS = ((8.205, -22.9, 16.46), (4.066, -2.861, 0.5184), (3.910, -2.823, 0.5250), (3.286, -2.415, 0.4853), (2.278, -1.620, 0.3985))


@pytest.mark.parametrize("schedule", [pkg.QUINTIC_SCHEDULE, LARGE_FACTORS], ids=["quintic", "large_factors"])
@pytest.mark.parametrize("m,n", [(20, 160), (32, 256), (33, 66), (41, 328), (45, 90), (46, 115), (48, 384), (48, 576), (49, 147), (60, 60), (64, 144), (100, 100),
                                 (128, 2000), (193, 193), (250, 333), (256, 256), (512, 512), (1024, 1024)])
def test_errors_stay_near_those_of_float32_steps(dev, m, n, schedule):
    """At most 1.5 times, geometric mean over matrices: what the steps on one Gram matrix are chosen by."""
    count = max(2, min(64, int(2e6 / (m * n))))
    g = torch.Generator(device=dev).manual_seed(m * 7919 + n)
    x = torch.randn((count, m, n), device=dev, generator=g)
    x += 0.5 * torch.randn((count, m, 2), device=dev, generator=g) @ torch.randn((count, 2, n), device=dev, generator=g)
    want = _on_device(x, schedule)
    plain = x / (x.double().square().sum(dim=(1, 2), keepdim=True).sqrt() + 1e-7).float()
    for a, b, c in schedule:
        gram = plain @ plain.mT.contiguous()
        plain = a * plain + (b * gram + c * (gram @ gram)) @ plain
    got = pkg.lmkan_orthogonalize(pkg.MatrixDesc(count, m, n), x, schedule=schedule)
    far, far_plain = ((t.double() - want).flatten(1).norm(dim=1) / want.flatten(1).norm(dim=1) for t in (got, plain))
    assert float((far / far_plain).log().mean().exp()) <= 1.5


@pytest.mark.parametrize("x_size,w_size", [(1e-36, 1e-4), (1e-35, 1e-6), (1e30, 1e-3), (1.0, 1e-30)])
@pytest.mark.parametrize("batch,n_in,n_out", [(1, 300, 64), (1, 4096, 2100), (5, 300, 64), (300, 300, 64), (300, 300, 61), (70, 4096, 64), (70, 4096, 33)])
def test_linear_i8_of_rows_of_any_magnitude(dev, batch, n_in, n_out, x_size, w_size):
    """Scales whose product lies below float32's normal range: the sum brings it back."""
    g = torch.Generator().manual_seed(batch + n_in + n_out)
    x = x_size * torch.randn((batch, n_in), generator=g)
    w = torch.randint(-127, 128, (n_out, n_in), generator=g, dtype=torch.int8)
    ws = w_size * (0.5 + torch.rand((n_out,), generator=g))
    codes, scale = _codes(x)
    product = codes.astype(np.float64) @ w.numpy().astype(np.float64).T
    want = product * scale.astype(np.float64)[:, None] * ws.numpy().astype(np.float64)
    got = pkg.lmkan_linear_i8(pkg.LinearDesc(n_in, n_out), x.to(dev), w.to(dev), ws.to(dev)).cpu().double().numpy()
    off = np.abs(got - want)
    most = 4 * 2.0 ** -24 * np.abs(want) + 2.0 ** -149
    assert (off <= most).all(), float((off / most).max())
