"""Launches of the calls on dense matrices, found without a GPU."""
import pytest

from dense_routes import routes
from routes import recorder


@pytest.fixture(scope="module")
def rec(tmp_path_factory):
    return recorder(tmp_path_factory.mktemp("recorder"))


# a launch takes fewer than 2^32 work items along a dimension: the runtime refuses more
@pytest.mark.parametrize("call", [
    dict(fn="quantize", rows=1 << 26, cols=8), dict(fn="quantize", rows=(1 << 31) - 1, cols=1), dict(fn="quantize", rows=1 << 24, cols=2049),
    dict(fn="orthogonalize", batch=1 << 26, rows=4, cols=8), dict(fn="orthogonalize", batch=5600000, rows=64, cols=64),
    dict(fn="muon", batch=(1 << 31) - 1, rows=1, cols=1), dict(fn="orthogonalize", batch=1 << 22, rows=16, cols=600),
    dict(fn="orthogonalize", batch=1 << 26, rows=4, cols=8, schedule=[]), dict(fn="orthogonalize", batch=1 << 25, rows=65, cols=65),
    dict(fn="orthogonalize", batch=1, rows=65, cols=1 << 26), dict(fn="orthogonalize", batch=1 << 22, rows=64, cols=1000),
    dict(fn="linear", batch=1 << 26, n_in=8, n_out=1), dict(fn="linear", batch=1 << 24, n_in=2049, n_out=2),
    dict(fn="linear", batch=(1 << 31) - 1, n_in=1, n_out=1), dict(fn="linear", batch=100, n_in=4097, n_out=4194240),
    dict(fn="linear", batch=1, n_in=131070, n_out=4194240), dict(fn="linear", batch=2, n_in=8, n_out=4194240),
], ids=lambda c: "-".join(str(v) for v in c.values()))
def test_no_launch_is_larger_than_the_runtime_takes(rec, call):
    (status, launches, _), = routes([call], rec)
    assert status == 0 and launches
    for name, grid, threads, _ in launches:
        assert grid[0] * threads < 1 << 32 and grid[1] <= 65535 and grid[2] <= 65535, (name, grid, threads)
