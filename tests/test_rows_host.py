"""Refusals of the operators on rows (norm, checkpoints, linear gradient, adapters), found on the host before anything is
launched."""
import ctypes as C

import pytest
import torch

import paper_2509_07103_amd as pkg
from paper_2509_07103_amd import binding

OK, NULL, SHAPE, UNSUPPORTED, WORKSPACE, ALIGN = 0, 1, 2, 3, 4, 5
ODD = C.c_void_p(0x10001)
BIG = C.c_size_t(1 << 60)


def _at(n):
    """Addresses far apart, never dereferenced: validation comes first."""
    return C.c_void_p((n + 1) << 32)


def _checkpoint(rows=4, cols=40, dtype=0, flags=0, x=_at(0), codes=_at(1), exps=_at(2)):
    return pkg.lib().lmkan_checkpoint_rows(rows, cols, dtype, flags, x, codes, exps, None)


@pytest.mark.parametrize("kw,status", [
    (dict(rows=-1), SHAPE), (dict(cols=0), SHAPE), (dict(cols=131071), SHAPE), (dict(rows=1 << 31), SHAPE),
    (dict(dtype=3), UNSUPPORTED), (dict(flags=2), UNSUPPORTED), (dict(x=None), NULL), (dict(codes=None), NULL),
    (dict(exps=None), NULL), (dict(x=ODD), ALIGN), (dict(x=ODD, dtype=2), ALIGN),
    (dict(codes=_at(0)), UNSUPPORTED), (dict(exps=_at(0)), UNSUPPORTED), (dict(exps=_at(1)), UNSUPPORTED),
    (dict(rows=0, x=None, codes=None, exps=None), OK),
])
def test_checkpoint_refuses(kw, status):
    assert _checkpoint(**kw) == status


def _restore(rows=4, cols=40, dtype=0, flags=0, codes=_at(1), exps=_at(2), weight=_at(3), bias=_at(4), y=_at(5)):
    return pkg.lib().lmkan_restore_rows(rows, cols, dtype, flags, codes, exps, weight, bias, y, None)


@pytest.mark.parametrize("kw,status", [
    (dict(rows=-1), SHAPE), (dict(cols=0), SHAPE), (dict(dtype=-1), UNSUPPORTED), (dict(flags=4), UNSUPPORTED),
    (dict(codes=None), NULL), (dict(exps=None), NULL), (dict(y=None), NULL), (dict(y=ODD), ALIGN), (dict(weight=ODD), ALIGN),
    (dict(bias=ODD), ALIGN), (dict(y=_at(1)), UNSUPPORTED), (dict(y=_at(2)), UNSUPPORTED), (dict(y=_at(3)), UNSUPPORTED),
    (dict(y=_at(4)), UNSUPPORTED), (dict(rows=0, codes=None, exps=None, y=None), OK),
])
def test_restore_refuses(kw, status):
    assert _restore(**kw) == status


def _norm(rows=4, x=_at(0), weight=None, bias=None, y=_at(1), stats=None, codes=None, exps=None, flags=0, **kw):
    d = pkg.NormDesc(**{**dict(cols=40), **kw}).c()
    d.flags = flags
    return pkg.lib().lmkan_layer_norm(C.byref(d), rows, x, weight, bias, y, stats, codes, exps, None)


@pytest.mark.parametrize("kw,status", [
    (dict(rows=-1), SHAPE), (dict(cols=0), SHAPE), (dict(cols=131071), SHAPE), (dict(x_dtype=3), UNSUPPORTED),
    (dict(y_dtype=-1), UNSUPPORTED), (dict(eps=0.0), UNSUPPORTED), (dict(eps=-1.0), UNSUPPORTED),
    (dict(eps=float("nan")), UNSUPPORTED), (dict(eps=float("inf")), UNSUPPORTED), (dict(flags=2), UNSUPPORTED),
    (dict(x=None), NULL), (dict(y=None), NULL), (dict(codes=_at(5)), NULL), (dict(exps=_at(5)), NULL),
    (dict(x=ODD), ALIGN), (dict(y=ODD), ALIGN), (dict(weight=ODD), ALIGN), (dict(bias=ODD), ALIGN), (dict(stats=ODD), ALIGN),
    (dict(x=_at(1), y_dtype=1), UNSUPPORTED),                      # in place in another type
    (dict(y=C.c_void_p((1 << 32) + 8)), UNSUPPORTED),              # shifted
    (dict(stats=_at(0)), UNSUPPORTED), (dict(stats=_at(1)), UNSUPPORTED), (dict(codes=_at(0), exps=_at(6)), UNSUPPORTED),
    (dict(codes=_at(5), exps=_at(5)), UNSUPPORTED), (dict(codes=_at(1), exps=_at(6)), UNSUPPORTED),
    (dict(y=_at(2), weight=_at(2)), UNSUPPORTED), (dict(rows=0, x=None, y=None), OK),
])
def test_layer_norm_refuses(kw, status):
    assert _norm(**kw) == status


def _norm_backward(rows=4, x=_at(0), codes=None, exps=None, stats=_at(3), weight=_at(4), gy=_at(5), gx=_at(6), gw=_at(7), gb=_at(8),
                   ws=_at(9), nbytes=BIG, flags=0, **kw):
    d = pkg.NormDesc(**{**dict(cols=40), **kw}).c()
    d.flags = flags
    return pkg.lib().lmkan_layer_norm_backward(C.byref(d), rows, x, codes, exps, stats, weight, gy, gx, gw, gb, ws, nbytes, None)


@pytest.mark.parametrize("kw,status", [
    (dict(rows=-1), SHAPE), (dict(cols=0), SHAPE), (dict(eps=0.0), UNSUPPORTED), (dict(flags=2), UNSUPPORTED),
    (dict(x=None), NULL), (dict(x=None, codes=_at(1)), NULL), (dict(x=None, exps=_at(1)), NULL), (dict(stats=None), NULL),
    (dict(gy=None), NULL), (dict(codes=_at(1), exps=_at(2)), UNSUPPORTED), (dict(x=ODD), ALIGN), (dict(gy=ODD), ALIGN),
    (dict(stats=ODD), ALIGN), (dict(gx=ODD), ALIGN), (dict(gw=ODD), ALIGN), (dict(gb=ODD), ALIGN), (dict(weight=ODD), ALIGN),
    (dict(gx=_at(0)), UNSUPPORTED), (dict(gx=_at(5)), UNSUPPORTED), (dict(gw=_at(4)), UNSUPPORTED), (dict(gb=_at(7)), UNSUPPORTED),
    (dict(gx=_at(7)), UNSUPPORTED), (dict(ws=None), WORKSPACE), (dict(nbytes=C.c_size_t(0)), WORKSPACE),
    (dict(ws=C.c_void_p(0xa00000010)), ALIGN),
])
def test_layer_norm_backward_refuses(kw, status):
    assert _norm_backward(**kw) == status


def _grad(batch=4, codes=_at(0), exps=_at(1), gy=_at(2), gw=_at(3), gb=_at(4), ws=_at(9), nbytes=BIG, flags=0, **kw):
    d = pkg.LinearDesc(**{**dict(n_in=40, n_out=24), **kw}).c()
    d.flags |= flags
    return pkg.lib().lmkan_linear_grad(C.byref(d), batch, codes, exps, gy, gw, gb, ws, nbytes, None)


@pytest.mark.parametrize("kw,status", [
    (dict(batch=-1), SHAPE), (dict(batch=1 << 31), SHAPE), (dict(n_in=0), SHAPE), (dict(n_out=0), SHAPE), (dict(n_in=131071), SHAPE),
    (dict(n_out=4194241), SHAPE), (dict(y_dtype=3), UNSUPPORTED), (dict(flags=4), UNSUPPORTED), (dict(codes=None), NULL),
    (dict(exps=None), NULL), (dict(gy=None), NULL), (dict(gw=None), NULL), (dict(gy=ODD), ALIGN), (dict(gw=ODD), ALIGN),
    (dict(gb=ODD), ALIGN), (dict(gw=_at(0)), UNSUPPORTED), (dict(gw=_at(2)), UNSUPPORTED), (dict(gb=_at(3)), UNSUPPORTED),
    (dict(batch=0, gw=None), NULL),
])
def test_linear_grad_refuses(kw, status):
    assert _grad(**kw) == status


def test_linear_grad_refuses_workspaces():
    d = pkg.LinearDesc(1024, 1024)
    assert pkg.lmkan_linear_grad_workspace_bytes(pkg.LinearDesc(0, 4), 8) == 0
    if pkg.lmkan_linear_grad_workspace_bytes(d, 8192) > 0:
        big = dict(batch=8192, n_in=1024, n_out=1024)
        assert _grad(ws=None, **big) == WORKSPACE and _grad(nbytes=C.c_size_t(255), **big) == WORKSPACE
        assert _grad(ws=C.c_void_p(0xa00000010), **big) == ALIGN


def _adapters(batch=4, x=_at(0), index=_at(1), a=_at(2), b=_at(3), scale=_at(4), y=_at(5), ws=_at(9), nbytes=BIG, flags=0, **kw):
    d = pkg.AdapterDesc(**{**dict(count=3, rank=4, n_in=40, n_out=24), **kw}).c()
    d.flags |= flags
    return pkg.lib().lmkan_adapters_add(C.byref(d), batch, x, index, a, b, scale, y, ws, nbytes, None)


@pytest.mark.parametrize("kw,status", [
    (dict(batch=-1), SHAPE), (dict(count=0), SHAPE), (dict(count=8193), SHAPE), (dict(rank=0), SHAPE), (dict(rank=257), SHAPE),
    (dict(n_in=0), SHAPE), (dict(n_out=0), SHAPE), (dict(n_in=131071), SHAPE), (dict(n_out=4194241), SHAPE),
    (dict(dtype=3), UNSUPPORTED), (dict(x_dtype=-1), UNSUPPORTED), (dict(y_dtype=5), UNSUPPORTED), (dict(flags=2), UNSUPPORTED),
    (dict(x=None), NULL), (dict(index=None), NULL), (dict(a=None), NULL), (dict(b=None), NULL), (dict(y=None), NULL),
    (dict(x=ODD), ALIGN), (dict(index=ODD), ALIGN), (dict(a=ODD), ALIGN), (dict(b=ODD), ALIGN), (dict(scale=ODD), ALIGN), (dict(y=ODD), ALIGN),
    (dict(y=_at(0)), UNSUPPORTED), (dict(y=_at(1)), UNSUPPORTED), (dict(y=_at(2)), UNSUPPORTED), (dict(y=_at(3)), UNSUPPORTED),
    (dict(y=_at(4)), UNSUPPORTED), (dict(batch=0, x=None, index=None, a=None, b=None, y=None, ws=None, nbytes=C.c_size_t(0)), OK),
])
def test_adapters_refuse(kw, status):
    assert _adapters(**kw) == status


def test_adapters_refuse_workspaces():
    big = dict(batch=4096, n_in=1024, n_out=1024, rank=32, count=8)
    assert pkg.lmkan_adapters_workspace_bytes(pkg.AdapterDesc(8, 32, 1024, 1024), 4096) > 256
    assert _adapters(ws=None, **big) == WORKSPACE and _adapters(nbytes=C.c_size_t(256), **big) == WORKSPACE
    assert _adapters(ws=C.c_void_p(0xa00000010), **big) == ALIGN
    assert pkg.lmkan_adapters_workspace_bytes(pkg.AdapterDesc(0, 32, 1024, 1024), 4096) == 0


def test_missing_descriptors():
    L = pkg.lib()
    p = _at(0)
    assert L.lmkan_layer_norm(None, 1, p, p, p, p, p, p, p, None) == NULL
    assert L.lmkan_layer_norm_backward(None, 1, p, p, p, p, p, p, p, p, p, p, BIG, None) == NULL
    assert L.lmkan_linear_grad(None, 1, p, p, p, p, p, p, BIG, None) == NULL
    assert L.lmkan_adapters_add(None, 1, p, p, p, p, p, p, p, BIG, None) == NULL
    assert L.lmkan_layer_norm_backward_workspace_bytes(None, 4) == L.lmkan_linear_grad_workspace_bytes(None, 4) == 0
    assert L.lmkan_adapters_workspace_bytes(None, 4) == 0


def test_sizes_of_checkpoints():
    assert pkg.lmkan_checkpoint_exps_bytes(5, 64) == 10 and pkg.lmkan_checkpoint_exps_bytes(5, 65) == 15
    assert pkg.lmkan_checkpoint_exps_bytes(5, 0) == pkg.lmkan_checkpoint_exps_bytes(-1, 8) == 0


def test_linear_i8_still_refuses_the_flag_of_the_gradient():
    d = binding._Linear(8, 4, 0, 0, pkg.LMKAN_LINEAR_ACCUMULATE)
    p = _at(0)
    assert pkg.lib().lmkan_linear_i8(C.byref(d), 4, p, p, p, None, 0.0, p, p, BIG, None) == UNSUPPORTED


def test_python_refuses_tensors_that_do_not_fit():
    x, row = torch.zeros((4, 40)), torch.zeros((40,))
    codes, exps, stats = torch.zeros((4, 40), dtype=torch.int8), torch.zeros((4, 2), dtype=torch.uint8), torch.zeros((4, 2))
    norm, linear, adapters = pkg.NormDesc(40), pkg.LinearDesc(40, 24), pkg.AdapterDesc(3, 4, 40, 24)
    calls = [
        lambda: pkg.lmkan_checkpoint_rows(x),                                                    # not on the device
        lambda: pkg.lmkan_checkpoint_rows(x.double()),
        lambda: pkg.lmkan_checkpoint_rows(row),
        lambda: pkg.lmkan_restore_rows(codes, exps),
        lambda: pkg.lmkan_restore_rows(codes, exps, dtype=7),
        lambda: pkg.lmkan_restore_rows(codes[0], exps),
        lambda: pkg.lmkan_layer_norm(norm, x),
        lambda: pkg.lmkan_layer_norm(norm, row),
        lambda: pkg.lmkan_layer_norm_backward(norm, x, stats, x=x),
        lambda: pkg.lmkan_layer_norm_backward(norm, x, stats),                                   # neither rows nor checkpoint
        lambda: pkg.lmkan_layer_norm_backward(norm, x, stats, x=x, kept=(codes, exps)),          # both
        lambda: pkg.lmkan_layer_norm_backward(norm, x, stats, x=x, accumulate=True),             # nothing to add to
        lambda: pkg.lmkan_linear_grad(linear, codes, exps, torch.zeros((4, 24))),
        lambda: pkg.lmkan_linear_grad(linear, codes, exps, torch.zeros((4, 24)), accumulate=True),
        lambda: pkg.lmkan_adapters_add(adapters, x, torch.zeros((4,), dtype=torch.int32), torch.zeros((3, 4, 40)), torch.zeros((3, 24, 4)),
                                       torch.zeros((4, 24))),
    ]
    for k, call in enumerate(calls):
        with pytest.raises(ValueError):
            call()
            print("not refused:", k)
