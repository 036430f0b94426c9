"""The operators of the dense matrices at the ends of their documented ranges: sizes, magnitudes, schedules.

Tolerances are those of test_gpu_dense.py: 4e-5 of the result's norm for five steps, and the unit roundoff of a
16-bit result."""
import pytest
import torch

import paper_2509_07103_amd as pkg

pytestmark = pytest.mark.gpu

TOL = 4e-5


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
