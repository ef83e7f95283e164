"""Argument checks of the layer norm, of the lists of tensors and of the normalised paths at the C ABI, which need no GPU:
a call that is refused has launched nothing."""
import ctypes

import numpy as np
import pytest

from paper_2301_08527_amd import rocket

P = ctypes.c_void_p(4096)
BIG = 1 << 40
E, W = rocket.ROCKET_EINVAL, rocket.ROCKET_EWORKSPACE


def test_layer_norm_refusals():
    lib = rocket.load_library()

    def norm(x=P, dtype=0, rows=4, planes=2, n=30, eps=1e-5, y=P, mean=None, rstd=None, ws=P, size=BIG):
        return lib.rocket_layer_norm(x, dtype, rows, planes, n, P, P, eps, y, mean, rstd, ws, size, None)

    for bad in (dict(x=None), dict(y=None), dict(dtype=3), dict(dtype=-1), dict(rows=0), dict(planes=0), dict(n=0), dict(n=-5), dict(planes=65536), dict(n=2**30 + 1), dict(eps=0.0),
                dict(eps=-1.0), dict(eps=float("inf")), dict(eps=float("nan")), dict(mean=P), dict(rstd=P), dict(x=ctypes.c_void_p(4098)),
                dict(y=ctypes.c_void_p(4097), dtype=1)):
        assert norm(**bad) == E, bad
        assert rocket.rocket_last_error().startswith("rocket_layer_norm: ")

    def back(x=P, dy=P, dtype=0, rows=4, planes=2, n=30, mean=P, rstd=P, dx=P, ws=P, size=BIG):
        return lib.rocket_layer_norm_backward(x, dy, dtype, rows, planes, n, P, mean, rstd, dx, P, P, ws, size, None)

    for bad in (dict(x=None), dict(dy=None), dict(dx=None), dict(mean=None), dict(rstd=None), dict(dtype=7), dict(rows=0), dict(planes=0), dict(n=0),
                dict(dy=ctypes.c_void_p(4099), dtype=2), dict(dx=ctypes.c_void_p(4098))):
        assert back(**bad) == E, bad
    need = lib.rocket_layer_norm_workspace_bytes(4, 2, 30, 1)
    assert need > 0 and need % 256 == 0
    for bad in (dict(ws=None), dict(size=need - 1), dict(ws=ctypes.c_void_p(4100))):
        assert back(**bad) == W, bad
    for sizes in ((0, 1, 1), (1, 0, 1), (1, 1, 0), (-1, 1, 1)):
        assert lib.rocket_layer_norm_workspace_bytes(*sizes, 0) == 0 and lib.rocket_layer_norm_workspace_bytes(*sizes, 1) == 0


@pytest.mark.parametrize("rows,planes,n", [(1, 1, 2**30), (2**31 - 1, 1, 1), (2**31 - 1, 3, 2**30), (65535, 65535, 100), (1, 2**31 - 1, 7), (1, 1, 2**30 + 1)])
def test_workspace_sizes_do_not_wrap(rows, planes, n):
    """sizes are 64-bit throughout: more rows or values never need less"""
    lib = rocket.load_library()
    for backward in (0, 1):
        need = lib.rocket_layer_norm_workspace_bytes(rows, planes, n, backward)
        if planes > 65535 or n > 2**30:      # refused by the calls
            assert need == 0
            continue
        assert need % 256 == 0 and (need > 0 or not backward)
        assert need >= lib.rocket_layer_norm_workspace_bytes(max(1, rows // 4096), planes, n, backward)
        if n > 1 << 20:         # rows in parts: a record for each
            assert need >= 16 * rows * planes


def _list(*records):
    kind = np.dtype([("data", np.uint64), ("count", np.int64), ("dtype", np.int32), ("reserved", np.int32)])
    return np.array([r + (0,) for r in records], dtype=kind)


def test_lists_of_tensors():
    lib = rocket.load_library()

    def at(a):
        return None if a is None else a.ctypes.data

    good = _list((4096, 100, 0), (8192, 0, 1), (12290, 3, 2))
    need = lib.rocket_grad_workspace_bytes(at(good), 3)
    assert need > 0 and need % 256 == 0
    for bad in (_list((0, 5, 0)), _list((4096, -1, 0)), _list((4096, 5, 3)), _list((4098, 5, 0)), _list((4097, 5, 1)), _list((4096, 2**43, 0)), None):
        assert lib.rocket_grad_workspace_bytes(at(bad), 1) == 0
        assert lib.rocket_grad_norm(at(bad), 1, 1.0, P, P, BIG, None) == E
        assert lib.rocket_grad_clip(at(bad), None, 1, 1.0, P, P, BIG, None) == E
        assert lib.rocket_sgd_tensors(at(bad), at(_list((4096, 5, 0))), None, 1, 0.1, None, None) == E
    assert lib.rocket_grad_norm(at(good), 0, 1.0, P, P, BIG, None) == E
    assert lib.rocket_grad_norm(at(good), -3, 1.0, P, P, BIG, None) == E
    for m in (0.0, -1.0, float("nan")):
        assert lib.rocket_grad_norm(at(good), 3, m, P, P, BIG, None) == E
    assert lib.rocket_grad_norm(at(good), 3, 1.0, None, P, BIG, None) == E
    assert lib.rocket_grad_norm(at(good), 3, 1.0, P, None, BIG, None) == W
    assert lib.rocket_grad_norm(at(good), 3, 1.0, P, P, need - 1, None) == W
    assert lib.rocket_grad_norm(at(good), 3, 1.0, P, ctypes.c_void_p(4100), BIG, None) == W
    other = _list((4096, 100, 0), (8192, 1, 1), (12290, 3, 2))
    assert lib.rocket_grad_clip(at(good), at(other), 3, 1.0, P, P, BIG, None) == E and "tensor 1" in rocket.rocket_last_error()
    other = _list((4096, 100, 0), (8192, 0, 2), (12290, 3, 2))
    assert lib.rocket_grad_clip(at(good), at(other), 3, 1.0, P, P, BIG, None) == E
    f32 = _list((4096, 100, 0), (8192, 0, 0), (12288, 3, 0))
    assert lib.rocket_sgd_tensors(at(good), at(good), None, 3, 0.1, P, None) == E           # parameters are float32
    assert lib.rocket_sgd_tensors(at(f32), at(good), at(good), 3, 0.1, P, None) == E
    assert lib.rocket_sgd_tensors(at(f32), at(good), None, 3, float("nan"), P, None) == E
    h = rocket.rocket_make_kernels(1, 10, 2, 100)
    assert lib.rocket_sgd_update_clipped(h.handle, P, P, 0.1, 0, None, None) == E
    assert lib.rocket_sgd_update_clipped(h.handle, None, P, 0.1, 0, P, None) == E
    assert lib.rocket_sgd_update_clipped(h.handle, P, P, float("nan"), 0, P, None) == E


@pytest.mark.parametrize("more", [0, 300])
def test_what_is_written_overlaps_nothing(more):
    """the same tensor twice, one that reaches into the next, results in another's place; addresses that a GPU call would
    fault on are never reached"""
    lib = rocket.load_library()
    rest = [((1 << 30) + 4096 * i, 10, 0) for i in range(more)]
    rest2 = [((1 << 31) + 4096 * i, 10, 0) for i in range(more)]
    n = 2 + more

    def clip(grads, out):
        g, o = _list(*(grads + rest)), None if out is None else _list(*(out + rest2))
        return lib.rocket_grad_clip(g.ctypes.data, None if o is None else o.ctypes.data, n, 1.0, P, P, BIG, None)

    def sgd(params, grads, out):
        p, g, o = _list(*(params + rest)), _list(*(grads + rest)), None if out is None else _list(*(out + rest2))
        return lib.rocket_sgd_tensors(p.ctypes.data, g.ctypes.data, None if o is None else o.ctypes.data, n, 0.1, None, None)

    a, b, c, d = (4096, 100, 0), (8192, 100, 0), (16384, 100, 0), (32768, 100, 0)
    inside = (4096 + 396, 100, 0)          # begins in a's last value
    for grads, out in (([a, a], None), ([a, inside], None), ([a, b], [c, c]), ([a, b], [b, a]), ([a, b], [c, inside]), ([a, b], [inside, c]),
                       ([a, a], [a, c])):
        assert clip(grads, out) == E and "overlap" in rocket.rocket_last_error(), (grads, out)
    for params, grads, out in (([a, a], [c, d], None), ([a, b], [a, c], None), ([a, b], [c, inside], None), ([a, b], [c, d], [d, (65536, 100, 0)]),
                               ([a, b], [c, d], [b, (65536, 100, 0)])):
        assert sgd(params, grads, out) == E and "overlap" in rocket.rocket_last_error(), (params, grads, out)


@pytest.mark.parametrize("tensors", [1, 95, 96, 97, 1000])
def test_workspace_of_many_tensors(tensors):
    """a partial sum per workgroup: it grows with the values, not with the tensors alone"""
    lib = rocket.load_library()
    few = _list(*[(4096, 1, 0)] * tensors)
    many = _list(*[(4096, 1 << 20, 0)] * tensors)
    a, b = (lib.rocket_grad_workspace_bytes(v.ctypes.data, tensors) for v in (few, many))
    assert 0 < a <= b < 1 << 22


def test_normed_paths_refuse():
    lib = rocket.load_library()
    h = rocket.rocket_make_kernels(1, 10, 2, 100)

    def infer(handle=h.handle, x=P, B=4, mask=3, eps=1e-5, coef=P, icpt=P, feats=P, pred=P, ws=P, size=BIG):
        return lib.rocket_infer_normed(handle, x, 0, B, mask, 10.0, -3.0, P, P, eps, coef, icpt, feats, pred, ws, size, None)

    for bad in (dict(handle=None), dict(x=None), dict(B=0), dict(mask=0), dict(mask=8), dict(eps=0.0), dict(coef=None), dict(icpt=None), dict(feats=None),
                dict(pred=None)):
        assert infer(**bad) == E, bad
    need = lib.rocket_infer_normed_workspace_bytes(h.handle, 4, 3)
    assert need >= rocket.rocket_workspace_bytes(h, 4, 3) + 4 * 4 * 20 and need % 256 == 0
    assert infer(size=need - 1) == W and infer(ws=None) == W
    assert lib.rocket_infer_normed_workspace_bytes(h.handle, 0, 3) == 0 and lib.rocket_infer_normed_workspace_bytes(None, 1, 3) == 0

    def train(handle=h.handle, x=P, B=4, mask=5, nw=P, nb=P, eps=1e-5, coef=P, icpt=P, y=P, lr=0.1, max_norm=1.0, ws=P, size=BIG):
        return lib.rocket_train_step_normed(handle, x, 0, B, mask, 10.0, -3.0, nw, nb, eps, coef, icpt, y, lr, 0, max_norm, P, P, ws, size, None)

    for bad in (dict(handle=None), dict(x=None), dict(B=0), dict(B=65536), dict(mask=3), dict(mask=0), dict(nw=None), dict(nb=None), dict(eps=-1.0),
                dict(coef=None), dict(icpt=None), dict(y=None), dict(lr=float("inf")), dict(max_norm=0.0), dict(max_norm=float("nan"))):
        assert train(**bad) == E, bad
    need = lib.rocket_train_normed_workspace_bytes(h.handle, 4, 5)
    assert need > rocket.rocket_train_workspace_bytes(h, 4, 5) and need % 256 == 0
    assert train(size=need - 1) == W and train(ws=None) == W
    assert lib.rocket_train_normed_workspace_bytes(h.handle, 0, 5) == 0
