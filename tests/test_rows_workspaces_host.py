"""Workspaces of the operators on rows cover every smaller batch: a program sizes one for its largest batch, and the last
batch of an epoch is a smaller one."""
import random

import pytest

import paper_2509_07103_amd as pkg


def _never_shrinks(size, batches):
    most, where = 0, None
    for n in batches:
        bytes_ = size(n)
        assert bytes_ >= most, f"{bytes_} bytes for {n} rows, {most} for {where}"
        most, where = bytes_, n


def _batches(seed):
    """All sorts of steps up to 70000 rows, the ends of tiles among them."""
    r = random.Random(seed)
    edges = [32 * t + d for t in range(1, 1100) for d in (0, 1)]
    return sorted(set(range(1, 200)) | set(edges) | {r.randrange(1, 70000) for _ in range(1500)} | {32767, 32768, 32769})


@pytest.mark.parametrize("shape", [(8, 64, 4096, 1024), (8, 64, 4096, 333), (3, 1, 100, 24), (8192, 4, 333, 64), (50, 256, 1024, 1024),
                                   (4, 128, 131070, 16), (2, 16, 257, 4096), (16, 33, 2048, 2048)], ids=str)
def test_adapters(shape):
    for dtype in (pkg.LMKAN_F32, pkg.LMKAN_BF16):
        desc = pkg.AdapterDesc(*shape, dtype=dtype)
        _never_shrinks(lambda n: pkg.lmkan_adapters_workspace_bytes(desc, n), _batches(1))
    assert pkg.lmkan_adapters_workspace_bytes(desc, 0) == 0


@pytest.mark.parametrize("shape", [(500, 333), (4096, 1024), (4096, 333), (1024, 1024), (64, 10), (1, 1), (1000, 1000), (2048, 2048), (4096, 4096),
                                   (130, 4000), (8000, 3000)], ids=str)
@pytest.mark.parametrize("y_dtype", [pkg.LMKAN_F32, pkg.LMKAN_F16, pkg.LMKAN_BF16])
def test_linear_gradient(shape, y_dtype):
    desc = pkg.LinearDesc(*shape, y_dtype=y_dtype)
    _never_shrinks(lambda n: pkg.lmkan_linear_grad_workspace_bytes(desc, n), _batches(2))
    # never more than the parts of four workgroups a unit, 256 x 128 float32 each, and their biases
    assert pkg.lmkan_linear_grad_workspace_bytes(desc, 70000) <= 1024 * 256 * 128 * 4 + 512 * shape[1] * 8 + 512


def test_norm_gradients():
    for cols in (1, 333, 1024, 20011):
        desc = pkg.NormDesc(cols)
        _never_shrinks(lambda n: pkg.lmkan_layer_norm_backward_workspace_bytes(desc, n), range(0, 3000))
