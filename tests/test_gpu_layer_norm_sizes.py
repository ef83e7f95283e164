"""The layer norm at sizes where its launches, its sums over rows and its ranges end (rocket_layer_norm, rocket_layer_norm_backward).
Needs an MI355X."""
import math

import pytest

from paper_2301_08527_amd import rocket

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,lanes", [(2, 4), (258, 64)])
def test_in_place_over_several_launches(n, lanes):
    """Three planes, so that the groups of lanes of a launch (2^20 workgroups of 256 / lanes groups, four examples to each) do not fill its
    last workgroup.  Row 7,001 i + k is row k, and so are its results, in place as elsewhere, bit for bit."""
    import torch
    planes, period = 3, 7001
    rows = (1 << 20) * (256 // lanes) // planes * 4 + 5
    again = -(-rows // period)
    print("layer norm in place", rows, planes, n, flush=True)
    g = torch.Generator(device="cuda")
    g.manual_seed(n)
    small = (3.0 + 2.0 * torch.randn((period, planes * n), generator=g, device="cuda")).to(torch.bfloat16)
    w, b = 1.5 + torch.rand(planes * n, generator=g, device="cuda"), 0.25 + torch.rand(planes * n, generator=g, device="cuda")
    mean, rstd = torch.empty((2, period, planes), device="cuda")
    want = rocket.rocket_layer_norm(small, w, b, planes=planes, mean=mean, rstd=rstd)
    x = small.repeat(again, 1)[:rows]
    assert x.is_contiguous()
    ms, rs = torch.empty((rows, planes), device="cuda"), torch.empty((rows, planes), device="cuda")
    rocket.rocket_layer_norm(x, w, b, planes=planes, y=x, mean=ms, rstd=rs)
    for got, one in ((x, want), (ms, mean), (rs, rstd)):
        whole = rows // period * period
        assert bool((got[:whole].view(-1, period, got.shape[1]) == one).all())
        assert torch.equal(got[whole:], one[:rows - whole])


@pytest.mark.parametrize("dtype,far", [("float32", False), ("float32", True), ("bfloat16", False)])
@pytest.mark.parametrize("rows,n", [(3, 8), (3, 301), (3, 1500), (3, 10000), (259, 65001), (3, 200001)])
def test_rows_as_large_as_their_squares_allow(rows, n, dtype, far):
    """n D^2 just below 3e38, D the largest distance from the mean and 1e-5 times the largest value: values of +-D, or, `far`, values whose
    mean's rounding takes nearly half of it.

    Tolerances: a sum adds at most 138 numbers one after the other (128 values of a lane, 6 exchanges, 4 joins), each addition off by
    U = 2^-24.  The first sum's rounding, `off` in units of the spread, is in the distances that the second one adds: it makes their
    mean's error (1 + off), that of their squares (1 + off^2) times as large.  The backward pass is given that r, three times in h c2."""
    import torch
    U, half = 2.0 ** -24, torch.finfo(getattr(torch, dtype)).eps / 2
    g = torch.Generator(device="cuda")
    g.manual_seed(n)
    most = math.sqrt(2.99e38 / n)
    w, b = 0.5 + torch.rand(n, generator=g, device="cuda"), torch.randn(n, generator=g, device="cuda")
    dy = torch.randn((rows, n), generator=g, device="cuda").to(getattr(torch, dtype))
    if far:
        x = 0.45e5 * most + 0.27 * most * (2.0 * torch.rand((rows, n), generator=g, device="cuda") - 1.0)
    else:
        x = 0.99 * most * (1.0 - 2.0 * (torch.arange(n, device="cuda") % 2)).repeat(rows, 1)
    x = x.to(getattr(torch, dtype))
    xd = x.double()
    m = xd.mean(1, keepdim=True)
    d = xd - m
    assert float(n * (d.abs().amax() + 1e-5 * xd.abs().amax()) ** 2) < 3e38
    r = 1.0 / torch.sqrt((d * d).mean(1, keepdim=True) + 1e-5)
    mean, rstd = torch.empty((2, rows, 1), device="cuda")
    y = rocket.rocket_layer_norm(x, w, b, mean=mean, rstd=rstd)
    h, off = d * r, 142 * U * float(xd.abs().amax()) * r
    ha, wide = h.abs(), 142 * (1 + off * off)
    want = h * w.double() + b.double()
    assert bool(((y.double() - want).abs() <= U * (142 * (1 + off) + wide * ha) * w.double() + (2 * U + half * 1.001) * want.abs()).all())
    assert bool(((rstd.double() - r).abs() <= U * wide * r).all())
    dx, dw, db = rocket.rocket_layer_norm_backward(x, dy, mean, rstd, w)
    gd = dy.double() * w.double()
    c1, c2 = gd.mean(1, keepdim=True), (gd * h).mean(1, keepdim=True)
    a1, a2 = gd.abs().mean(1, keepdim=True), (gd * h).abs().mean(1, keepdim=True)
    want = r * (gd - c1 - h * c2)
    tol = r * U * (146 * (a1 * (1 + ha) + a2 * (2 + ha)) + 8 * gd.abs() + wide * (gd.abs() + a1 + 3 * ha * a2)) + half * 1.001 * want.abs()
    assert bool(((dx.double() - want).abs() <= tol).all())
    assert bool(dw.isfinite().all()) and bool(db.isfinite().all())


@pytest.mark.parametrize("n", [1500, 20000, 30001])
def test_constant_rows_whose_mean_times_rstd_overflows(n):
    """x = m = 2^66 and r = 1 / sqrt(1e-42) = 1e21: h is 0 everywhere, also where a slot reaches beyond the row (there (0 - m) r would be
    -inf, and its product with 0 a NaN).  What is left is r (g - mean g); its sum adds at most 80 numbers one after the other."""
    import torch
    U = 2.0 ** -24
    g = torch.Generator(device="cuda")
    g.manual_seed(n)
    x = torch.full((3, n), 2.0 ** 66, device="cuda")
    w, dy = 0.5 + torch.rand(n, generator=g, device="cuda"), torch.randn((3, n), generator=g, device="cuda")
    mean, rstd = torch.empty((2, 3, 1), device="cuda")
    y = rocket.rocket_layer_norm(x, w, w, 1e-42, mean=mean, rstd=rstd)
    assert torch.equal(y, w.expand(3, n)) and bool((mean == 2.0 ** 66).all())
    dx, dw, db = rocket.rocket_layer_norm_backward(x, dy, mean, rstd, w)
    gd, r = dy.double() * w.double(), rstd.double()
    want = r * (gd - gd.mean(1, keepdim=True))
    assert bool(((dx.double() - want).abs() <= r * U * (84 * gd.abs().mean(1, keepdim=True) + 4 * gd.abs())).all())
    assert bool((dw == 0).all())
    assert bool(((db.double() - dy.double().sum(0)).abs() <= 4 * U * dy.double().abs().sum(0)).all())


@pytest.mark.parametrize("n", [65536 + 8192, 125000, 131072])
def test_sums_of_many_values_of_a_lane(n):
    """A row for each CU of so many 16-bit values that a lane holds up to 128.  Of three lanes two begin with 2^24 and one with -2^25 (but for
    every wavefront's last lane), all other values are 1: half a step, or less, of the sum that they are added to, lost each time, so that
    a sum of k numbers one after the other is off by k.  The mean of the distances has the error of such a sum of at most 80."""
    import torch
    rows, U = 256, 2.0 ** -24
    x = torch.ones((rows, n), dtype=torch.bfloat16, device="cuda")
    first = torch.tensor([2.0 ** 24, 2.0 ** 24, -2.0 ** 25] * 21 + [1.0], dtype=torch.bfloat16, device="cuda")
    x[:, 0:8192:8] = first.repeat(16)
    mean, rstd = torch.empty((2, rows, 1), device="cuda")
    rocket.rocket_layer_norm(x, mean=mean, rstd=rstd)
    d = x[0].double()
    m = float(d.mean())
    assert bool(((mean.double() - m).abs() <= U * abs(m) + 80 * U * float((d - m).abs().mean())).all())


SUMS = [(8191, 1, 7), (70001, 1, 3), (70001, 2, 30), (40009, 1, 65), (5003, 1025, 5), (9001, 3, 129), (20011, 1, 250), (20011, 1, 501), (8209, 1, 1000),
        (20011, 2, 1537), (4001, 1, 2050), (1201, 257, 2049), (401, 257, 4099), (677, 2, 10000), (3001, 1, 16384), (2003, 1, 20480), (5, 1, 20481), (3001, 1, 30001),
        (33001, 1, 20485), (7, 65535, 3), (400009, 1, 2048)]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows,planes,n", SUMS)
def test_sums_over_rows_miss_no_row_and_take_none_twice(rows, planes, n, dtype):
    """Gradients of -3 .. 3 and values of -1, 0 and 1 with a mean of 0, given an rstd of 1/2: every term of both sums is a multiple of 1/2 and
    every sum below 2^22, so that they are exact in whatever order and every single row counts."""
    import torch
    print("sums over rows", rows, planes, n, dtype, flush=True)
    t = getattr(torch, dtype)
    g = torch.Generator(device="cuda")
    g.manual_seed(rows + n)
    x = torch.zeros((rows, planes, n), dtype=t, device="cuda")
    half = n // 2
    dy = torch.empty_like(x)
    dw, db = torch.zeros((2, planes, n), dtype=torch.float64, device="cuda")
    step = max(1, (1 << 26) // (planes * n))
    for i in range(0, rows, step):
        some = min(step, rows - i)
        sign = (2 * torch.randint(0, 2, (some, planes, half), generator=g, device="cuda") - 1).to(t)
        x[i:i + some, :, :half], x[i:i + some, :, n - half:] = sign, -sign
        dy[i:i + some] = torch.randint(-3, 4, (some, planes, n), generator=g, device="cuda").to(t)
        d = dy[i:i + some].double()
        dw += (d * x[i:i + some].double()).sum(0) / 2
        db += d.sum(0)
    mean, rstd = torch.zeros((rows, planes), device="cuda"), torch.full((rows, planes), 0.5, device="cuda")
    w = torch.rand(planes * n, generator=g, device="cuda")
    _, gw, gb = rocket.rocket_layer_norm_backward(x.view(rows, -1), dy.view(rows, -1), mean, rstd, w, planes)
    assert torch.equal(gw.double().view(planes, n), dw) and torch.equal(gb.double().view(planes, n), db)


@pytest.mark.parametrize("rows,less,planes,n", [(677, 640, 2, 10000), (2100, 2048, 2, 500), (1500, 1080, 1, 30000), (300, 100, 1, 40000)])
def test_one_workspace_for_an_epoch(rows, less, planes, n):
    """the last batch, which is smaller, in the workspaces of the others, nothing beyond them is written"""
    import torch
    ws, wf = (torch.full((rocket.rocket_layer_norm_workspace_bytes(rows, planes, n, b) + 256,), 7, dtype=torch.uint8, device="cuda") for b in (True, False))
    for r in (rows, less):
        g = torch.Generator(device="cuda")
        g.manual_seed(r)
        x, dy = torch.randn((2, r, planes * n), generator=g, device="cuda")
        w = torch.rand(planes * n, generator=g, device="cuda")
        mean, rstd = torch.empty((2, r, planes), device="cuda")
        y = rocket.rocket_layer_norm(x, w, planes=planes, mean=mean, rstd=rstd, workspace=wf[:-256])
        assert torch.equal(y, rocket.rocket_layer_norm(x, w, planes=planes))
        got = rocket.rocket_layer_norm_backward(x, dy, mean, rstd, w, planes, workspace=ws[:-256])
        assert all(torch.equal(a, b) for a, b in zip(got, rocket.rocket_layer_norm_backward(x, dy, mean, rstd, w, planes)))
    assert bool((ws[-256:] == 7).all()) and bool((wf[-256:] == 7).all())


@pytest.mark.parametrize("rows,planes,n", [(7, 2, 300), (64, 1, 9000), (700, 2, 1537), (9, 1, 40000)])
def test_a_norm_that_is_not_trained(rows, planes, n):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(n)
    x, dy = torch.randn((2, rows, planes * n), generator=g, device="cuda")
    w = torch.rand(planes * n, generator=g, device="cuda")
    mean, rstd = torch.empty((2, rows, planes), device="cuda")
    rocket.rocket_layer_norm(x, w, planes=planes, mean=mean, rstd=rstd)
    back = lambda **k: rocket.rocket_layer_norm_backward(x, dy, mean, rstd, w, planes, **k)
    dx, dw, db = back()
    got = back(param_grads=False)
    assert torch.equal(got[0], dx) and got[1] is None and got[2] is None
    mine = torch.empty_like(db)
    got = back(param_grads=False, grad_bias=mine)       # one of the two
    assert torch.equal(got[0], dx) and got[1] is None and got[2] is mine and torch.equal(mine, db)


def test_more_long_rows_than_a_launch_has_groups_for():
    """33,001 rows in parts, in place; row 1,000 i + k is row k"""
    import torch
    rows, n, period = 33001, 65537, 1000
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    small = 3.0 + torch.randn((period, n), generator=g, device="cuda")
    w, b = torch.rand(n, generator=g, device="cuda"), torch.randn(n, generator=g, device="cuda")
    mean, rstd = torch.empty((2, period, 1), device="cuda")
    want = rocket.rocket_layer_norm(small, w, b, mean=mean, rstd=rstd)
    x = small.repeat(rows // period + 1, 1)[:rows]
    ms, rs = torch.empty((2, rows, 1), device="cuda")
    rocket.rocket_layer_norm(x, w, b, y=x, mean=ms, rstd=rs)
    for got, one in ((x, want), (ms, mean), (rs, rstd)):
        assert all(torch.equal(got[i:i + period], one[:rows - i]) for i in range(0, rows, period))


@pytest.mark.parametrize("rows,planes,n", [(5, 2, 3), (9, 3, 130), (6, 1, 1537), (3, 2, 9001), (2, 1, 70001)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_every_tensor_begins_anywhere(rows, planes, n, dtype):
    """one element behind a boundary, weights, results and sums too, the same bits as elsewhere; what lies around them stays"""
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(n)
    t = getattr(torch, dtype)
    x, dy = (torch.randn((rows, planes * n), generator=g, device="cuda").to(t) for _ in range(2))
    w, b = (torch.randn(planes * n, generator=g, device="cuda") for _ in range(2))
    mean, rstd = torch.empty((2, rows, planes), device="cuda")
    want = [rocket.rocket_layer_norm(x, w, b, planes=planes, mean=mean, rstd=rstd), mean, rstd]
    want += rocket.rocket_layer_norm_backward(x, dy, mean, rstd, w, planes)
    around = []

    def moved(like, fill=True):
        around.append(torch.full((like.numel() + 2,), 3.0, dtype=like.dtype, device="cuda"))
        inside = around[-1][1:-1].view(like.shape)
        return inside.copy_(like) if fill else inside

    x, dy, w, b = (moved(v) for v in (x, dy, w, b))
    y, m, r, dx, dw, db = got = [moved(v, False) for v in want]
    rocket.rocket_layer_norm(x, w, b, planes=planes, y=y, mean=m, rstd=r)
    rocket.rocket_layer_norm_backward(x, dy, m, r, w, planes, grad_x=dx, grad_weight=dw, grad_bias=db)
    assert all(torch.equal(u, v) for u, v in zip(got, want))
    assert all(bool((v[0] == 3.0) & (v[-1] == 3.0)) for v in around)


def test_the_longest_row():
    """2^30 - 3 values in 64 parts of 2,048 pieces, each joined with the ones before: a sum adds at most 48 + 5 * 2,048 + 40 < 10,400 numbers one
    after the other; mean and spread of the distances have such sums' errors, and there are a few roundings of h w + b"""
    import torch
    n, U, half = 2 ** 30 - 3, 2.0 ** -24, 2.0 ** -8
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    x = (5.0 + torch.randn(n, generator=g, device="cuda")).to(torch.bfloat16).view(1, n)
    w = torch.rand(n, generator=g, device="cuda")
    mean, rstd = torch.empty((2, 1, 1), device="cuda")
    y = rocket.rocket_layer_norm(x, w, mean=mean, rstd=rstd)
    step = 1 << 27
    m = sum(float(x[0, i:i + step].double().sum()) for i in range(0, n, step)) / n
    r = 1.0 / math.sqrt(sum(float((x[0, i:i + step].double() - m).square().sum()) for i in range(0, n, step)) / n + 1e-5)
    assert abs(float(mean) - m) <= U * m + 10400 * U / r and abs(float(rstd) - r) <= 10400 * U * r
    for i in range(0, n, step):
        h, ww = (x[0, i:i + step].double() - m) * r, w[i:i + step].double()
        assert bool(((y[0, i:i + step].double() - h * ww).abs() <= U * 10404 * ww * (1 + h.abs()) + (U + half * 1.001) * (h * ww).abs()).all())
    # the sums over a single row are dy h and dy themselves, but for the mean's rounding
    dy = torch.randint(-3, 4, (1, n), generator=g, device="cuda").to(torch.bfloat16)
    _, dw, db = rocket.rocket_layer_norm_backward(x, dy, mean, rstd, w, grad_x=y)
    rstd = float(rstd)
    for i in range(0, n, step):
        d, h = dy[0, i:i + step].double(), (x[0, i:i + step].double() - m) * rstd
        assert torch.equal(db[i:i + step].double(), d)
        assert bool(((dw[i:i + step].double() - d * h).abs() <= U * d.abs() * (8 * h.abs() + 10400)).all())
