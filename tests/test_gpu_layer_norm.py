"""Layer norm of feature planes (rocket_layer_norm, rocket_layer_norm_backward) against the formulas in fp64.  Needs an
MI355X.

Tolerances.  U = 2^-24 is half a step of fp32, `half(t)` of the result's type.  A sum of the kernels adds at most TERMS
numbers one after the other (64 values of a lane, 6 exchanges between lanes, 4 joins of wavefronts or parts of a row: 74), so
it is off by TERMS * U times the sum of the absolute values.  With h = (x - m) r:
  y   mean and spread are such sums, which moves h by TERMS * U * (1 + |h|); four more roundings of h, two of w h + b
  dx  = r (g - c1 - h c2), c1 and c2 such sums over |g| and |g h|
  dw  a sum over the rows, each term with the error of h
and one rounding to the result's type (f16 results below 2^-14 lie 2^-24 apart)."""
import numpy as np
import pytest

from paper_2301_08527_amd import rocket

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TERMS = 80
TYPES = ("float32", "bfloat16", "float16")


def _torch_type(name):
    import torch
    return getattr(torch, name)


def half(name):
    import torch
    return torch.finfo(_torch_type(name)).eps / 2


def tiny(name):
    return 2.0 ** -25 if name == "float16" else 2.0 ** -126


def make(rows, planes, n, dtype, seed, offset=8.0, unaligned=False):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randn((rows, planes, n), generator=g, device="cuda") * torch.exp(0.3 * torch.randn((rows, planes, 1), generator=g, device="cuda"))
    x = (x + offset).to(_torch_type(dtype)).reshape(rows, planes * n)
    dy = torch.randn((rows, planes * n), generator=g, device="cuda").to(_torch_type(dtype))
    if unaligned:       # one element past a boundary
        x, dy = (torch.cat([t.reshape(-1)[:1], t.reshape(-1)])[1:].view(rows, planes * n) for t in (x, dy))
        assert x.data_ptr() % 16 != 0
    w = 1.0 + 0.3 * torch.randn(planes * n, generator=g, device="cuda")
    b = 0.2 * torch.randn(planes * n, generator=g, device="cuda")
    return x, dy, w, b


def reference(x, w, b, planes, eps, dy=None):
    """fp64: h, r, y and, with dy, dx and the sums with the sums of absolute values that the tolerances need"""
    import torch
    rows = x.shape[0]
    x = x.double().view(rows, planes, -1)
    w = torch.ones_like(x[0]) if w is None else w.double().view(planes, -1)
    b = torch.zeros_like(x[0]) if b is None else b.double().view(planes, -1)
    m = x.mean(-1, keepdim=True)
    d = x - m
    r = 1.0 / torch.sqrt((d * d).mean(-1, keepdim=True) + eps)
    h = d * r
    out = dict(m=m, r=r, h=h, w=w, y=h * w + b)
    if dy is not None:
        dy = dy.double().view(rows, planes, -1)
        g = dy * w
        c1, c2 = g.mean(-1, keepdim=True), (g * h).mean(-1, keepdim=True)
        out.update(dy=dy, g=g, dx=r * (g - c1 - h * c2), dw=(dy * h).sum(0), db=dy.sum(0), abs1=g.abs().mean(-1, keepdim=True),
                   abs2=(g * h).abs().mean(-1, keepdim=True))
    return out


def check_forward(y, mean, rstd, ref, dtype, rows, planes):
    y = y.double().view(rows, planes, -1)
    h, w = ref["h"].abs(), ref["w"].abs()
    tol = U * ((TERMS + 4) * w * (1 + h) + 2 * ref["y"].abs()) + half(dtype) * ref["y"].abs() * 1.001 + tiny(dtype)
    off = (y - ref["y"]).abs()
    assert bool((off <= tol).all()), float((off / tol).max())
    if mean is not None:
        m, r = ref["m"][..., 0], ref["r"][..., 0]
        assert bool(((mean.double() - m).abs() <= U * m.abs() + TERMS * U / r).all())
        assert bool(((rstd.double() - r).abs() <= (TERMS + 4) * U * r).all())


def check_backward(dx, dw, db, ref, dtype, rows, planes):
    dx = dx.double().view(rows, planes, -1)
    h, r = ref["h"].abs(), ref["r"]
    # rstd and mean come rounded to 32 bits; of the mean's rounding e = mean h' is left with the error of a sum
    tol = r * U * ((TERMS + 8) * (ref["abs1"] * (1 + h) + ref["abs2"] * (2 + h)) + 8 * ref["g"].abs()) + half(dtype) * ref["dx"].abs() * 1.001 + tiny(dtype)
    off = (dx - ref["dx"]).abs()
    assert bool((off <= tol).all()), float((off / tol).max())
    sums = U * ((rows + 16) * (ref["dy"] * ref["h"]).abs().sum(0) + (TERMS + 4) * (ref["dy"].abs() * (1 + h)).sum(0))
    assert bool(((dw.double().view(planes, -1) - ref["dw"]).abs() <= sums + 2.0 ** -126).all())
    sums = U * (rows + 16) * ref["dy"].abs().sum(0)
    assert bool(((db.double().view(planes, -1) - ref["db"]).abs() <= sums + 2.0 ** -126).all())


def both(rows, planes, n, dtype, seed=0, eps=1e-5, offset=8.0, unaligned=False):
    import torch
    print("layer norm", rows, planes, n, dtype, unaligned, flush=True)
    x, dy, w, b = make(rows, planes, n, dtype, seed, offset, unaligned)
    mean, rstd = torch.full((2, rows, planes), float("nan"), device="cuda")
    y = rocket.rocket_layer_norm(x, w, b, eps, planes, mean=mean, rstd=rstd)
    ref = reference(x, w, b, planes, eps, dy)
    check_forward(y, mean, rstd, ref, dtype, rows, planes)
    ws = torch.full((rocket.rocket_layer_norm_workspace_bytes(rows, planes, n) // 4,), float("nan"), device="cuda")   # scratch is not read before it is written
    dx, dw, db = rocket.rocket_layer_norm_backward(x, dy, mean, rstd, w, planes, workspace=ws)
    check_backward(dx, dw, db, ref, dtype, rows, planes)


# every width at which a lane, a wavefront, a workgroup or a part of a row is just full, one short or one over
WIDTHS = sorted({1, 2, 3, 5, 7, 8, 9, 31, 33, 100, 500, 1000, 1537, 10000, 20001} |
                {w + d for w in (64, 128, 256, 512, 1024, 2048, 4096, 8192, 16384) for d in (-1, 0, 1)})


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", WIDTHS)
def test_widths(n, dtype):
    both(5, 2, n, dtype, seed=n)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [32768, 32769, 65537, 100000, 200001])
def test_rows_longer_than_a_workgroup_holds(n, dtype):
    both(3, 1, n, dtype, seed=n)


@pytest.mark.parametrize("rows,planes,n", [(1, 1, 1), (1, 1, 20000), (1, 3, 500), (2, 1, 3), (63, 1, 10), (257, 3, 37), (677, 2, 300), (1000, 1, 8),
                                           (4099, 1, 129), (8191, 3, 5), (70000, 1, 3), (3000, 1, 1000), (513, 1, 4100), (300, 2, 9001)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_rows(rows, planes, n, dtype):
    both(rows, planes, n, dtype, seed=rows + n)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("n", [100, 500, 700, 1000, 1537, 2001, 2500, 4000, 6001, 9000, 12001, 16384])
def test_many_rows_of_every_width(n, dtype):
    """two examples to a group of lanes, the last one alone; rows of whole cache lines beyond what the caches keep"""
    both(2051, 1, n, dtype, seed=n)
    both(1027, 2, n, dtype, seed=n + 1)


@pytest.mark.parametrize("dtype", ["float32", "float16"])
@pytest.mark.parametrize("n", [35000, 40961, 45057, 65535, 65536, 65537, 100001, 131072, 131073])
def test_a_long_row_for_each_cu(n, dtype):
    """rows that only then stay in registers"""
    import torch
    rows = 259
    x, _, w, b = make(rows, 1, n, dtype, n)
    mean, rstd = torch.empty((2, rows, 1), device="cuda")
    y = rocket.rocket_layer_norm(x, w, b, mean=mean, rstd=rstd)
    check_forward(y, mean, rstd, reference(x, w, b, 1, 1e-5), dtype, rows, 1)


def test_long_rows_beyond_the_caches():
    both(1501, 1, 40000, "float32", seed=4)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [33, 1001, 2047, 10001, 40001])
def test_rows_that_start_anywhere(n, dtype):
    both(4, 3, n, dtype, seed=n, unaligned=True)


@pytest.mark.parametrize("n", [50, 1000, 5000, 20000, 50000])
def test_mean_far_from_zero(n):
    """a mean of 10,000 spreads: its rounding to 32 bits alone would move every value of a row by 3e-4"""
    both(6, 1, n, "float32", seed=n, offset=1e4)


def test_constant_rows_and_one_value():
    import torch
    for n in (1, 40, 3000, 30000):
        x = torch.full((3, n), 7.3, device="cuda")
        w, b = torch.randn(n, device="cuda"), torch.randn(n, device="cuda")
        mean, rstd = torch.empty((2, 3, 1), device="cuda")
        y = rocket.rocket_layer_norm(x, w, b, 1e-5, mean=mean, rstd=rstd)
        # x - m is at most a rounding of the mean (U * 7.3, times 1/sqrt(eps) = 316)
        assert bool(((y - b).abs() <= 316.3 * U * 7.3 * w.abs() + U * b.abs() * 2).all())
        assert bool(((rstd - 1e5 ** 0.5).abs() <= 4 * U * 316.3).all())
        dy = torch.randn((3, n), device="cuda")
        dx, dw, db = rocket.rocket_layer_norm_backward(x, dy, mean, rstd, w)
        g = (dy * w).double()
        assert bool(((dx - 316.2278 * (g - g.mean(1, keepdim=True))).abs() <= 316.3 * 1e-5 * g.abs().max()).all())
        assert bool((dw.abs() <= 316.3 * 2 * U * 7.3 * dy.abs().sum(0)).all())


@pytest.mark.parametrize("n", [40, 1500, 12000, 40000])
def test_a_bad_row_leaves_the_others_alone(n):
    import torch
    x, dy, w, b = make(5, 1, n, "float32", n)
    mean, rstd = torch.empty((2, 5, 1), device="cuda")
    y = rocket.rocket_layer_norm(x, w, b, mean=mean, rstd=rstd)
    dx, _, _ = rocket.rocket_layer_norm_backward(x, dy, mean, rstd, w)
    for bad in (float("nan"), float("inf"), -float("inf")):
        xb = x.clone()
        xb[2, n // 3] = bad
        mb, rb = torch.empty((2, 5, 1), device="cuda")
        yb = rocket.rocket_layer_norm(xb, w, b, mean=mb, rstd=rb)
        dxb, dwb, _ = rocket.rocket_layer_norm_backward(xb, dy, mb, rb, w)
        good = [0, 1, 3, 4]
        assert torch.equal(yb[good], y[good]) and torch.equal(mb[good], mean[good]) and torch.equal(rb[good], rstd[good])
        assert torch.equal(dxb[good], dx[good])
        assert bool(yb[2].isnan().all()) and bool(dxb[2].isnan().all()) and bool(dwb.isnan().any())


@pytest.mark.parametrize("rows,planes,n", [(6, 2, 500), (40, 1, 3001), (9, 1, 20000), (2, 1, 70000), (3000, 1, 65)])
def test_in_place_without_weights_and_nothing_beyond_the_end(rows, planes, n):
    import torch
    for dtype in TYPES:
        print(rows, planes, n, dtype, flush=True)
        x, dy, w, b = make(rows, planes, n, dtype, 3)
        mean, rstd = torch.empty((2, rows, planes), device="cuda")
        want = rocket.rocket_layer_norm(x, w, b, planes=planes, mean=mean, rstd=rstd)
        guard = torch.full((rows * planes * n + 64,), 3.0, dtype=x.dtype, device="cuda")
        inside = guard[:-64].view(rows, planes * n)
        inside.copy_(x)
        rocket.rocket_layer_norm(inside, w, b, planes=planes, y=inside)
        assert torch.equal(inside, want) and bool((guard[-64:] == 3.0).all())
        want = rocket.rocket_layer_norm_backward(x, dy, mean, rstd, w, planes)
        inside.copy_(dy)
        sums = torch.full((2, planes * n + 64), 3.0, device="cuda")
        rocket.rocket_layer_norm_backward(x, inside, mean, rstd, w, planes, grad_x=inside, grad_weight=sums[0, :planes * n], grad_bias=sums[1, :planes * n])
        assert torch.equal(inside, want[0]) and bool((guard[-64:] == 3.0).all()) and bool((sums[:, planes * n:] == 3.0).all())
        assert torch.equal(sums[0, :planes * n], want[1]) and torch.equal(sums[1, :planes * n], want[2])
        for wt, bs in ((None, None), (w, None), (None, b)):
            ref = reference(x, wt, bs, planes, 1e-5, dy)
            check_forward(rocket.rocket_layer_norm(x, wt, bs, planes=planes), None, None, ref, dtype, rows, planes)
            if bs is None:
                check_backward(*rocket.rocket_layer_norm_backward(x, dy, mean, rstd, wt, planes), ref, dtype, rows, planes)


def test_backward_without_weight_gradients():
    import ctypes
    import torch
    lib = rocket.load_library()
    for rows, n in ((7, 300), (50, 9000), (3, 40000)):
        x, dy, w, _ = make(rows, 1, n, "float32", 5)
        mean, rstd = torch.empty((2, rows, 1), device="cuda")
        rocket.rocket_layer_norm(x, w, mean=mean, rstd=rstd)
        dx, dw, db = rocket.rocket_layer_norm_backward(x, dy, mean, rstd, w)
        ws = torch.empty(rocket.rocket_layer_norm_workspace_bytes(rows, 1, n), dtype=torch.uint8, device="cuda")
        stream = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
        for gw, gb in ((None, None), (torch.empty_like(w), None), (None, torch.empty_like(w))):
            got = torch.empty_like(dx)
            rc = lib.rocket_layer_norm_backward(x.data_ptr(), dy.data_ptr(), rocket.ROCKET_F32, rows, 1, n, w.data_ptr(), mean.data_ptr(), rstd.data_ptr(),
                                                got.data_ptr(), None if gw is None else gw.data_ptr(), None if gb is None else gb.data_ptr(),
                                                ws.data_ptr(), ws.numel(), stream)
            assert rc == rocket.ROCKET_OK, rocket.rocket_last_error()
            assert torch.equal(got, dx) and (gw is None or torch.equal(gw, dw)) and (gb is None or torch.equal(gb, db))


def test_gradients_against_differences():
    """central differences of the fp64 formula: step 1e-6, so errors of about 1e-9 beside those of the kernel"""
    import torch
    rows, planes, n, eps = 3, 2, 11, 1e-2
    x, dy, w, b = make(rows, planes, n, "float32", 17, offset=0.5)
    mean, rstd = torch.empty((2, rows, planes), device="cuda")
    rocket.rocket_layer_norm(x, w, b, eps, planes, mean=mean, rstd=rstd)
    dx, dw, db = (t.double().cpu().numpy().ravel() for t in rocket.rocket_layer_norm_backward(x, dy, mean, rstd, w, planes))
    x, dy, w, b = (t.double().cpu().numpy() for t in (x, dy, w, b))

    def loss(x, w, b):
        v = x.reshape(rows, planes, n)
        d = v - v.mean(-1, keepdims=True)
        y = d / np.sqrt((d * d).mean(-1, keepdims=True) + eps) * w.reshape(planes, n) + b.reshape(planes, n)
        return (y.reshape(rows, -1) * dy).sum()

    for which, grad in ((0, dx), (1, dw), (2, db)):
        args = [x, w, b]
        for i in range(grad.size):
            two = []
            for step in (1e-6, -1e-6):
                moved = args[which].copy()
                moved.ravel()[i] += step
                two.append(loss(*[moved if k == which else a for k, a in enumerate(args)]))
            assert abs((two[0] - two[1]) / 2e-6 - grad[i]) <= 1e-5


@pytest.mark.parametrize("rows,planes,n,dtype", [(16, 2, 500, "float32"), (300, 1, 1537, "bfloat16"), (64, 2, 10000, "float32"), (2, 1, 90001, "float16"),
                                                  (5000, 1, 256, "bfloat16")])
def test_same_bits_again_on_a_stream_and_in_a_graph(rows, planes, n, dtype):
    import torch
    x, dy, w, b = make(rows, planes, n, dtype, 23)
    mean, rstd = torch.empty((2, rows, planes), device="cuda")
    y = rocket.rocket_layer_norm(x, w, b, planes=planes, mean=mean, rstd=rstd)
    grads = rocket.rocket_layer_norm_backward(x, dy, mean, rstd, w, planes)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y2 = rocket.rocket_layer_norm(x, w, b, planes=planes, stream=side)
    grads2 = rocket.rocket_layer_norm_backward(x, dy, mean, rstd, w, planes, stream=side)
    side.synchronize()
    assert torch.equal(y, y2) and all(torch.equal(a, c) for a, c in zip(grads, grads2))
    xs, ys = x.clone(), torch.empty_like(x)
    ms, rs = torch.empty_like(mean), torch.empty_like(rstd)
    out = [torch.empty_like(t) for t in grads]
    ws = torch.empty(rocket.rocket_layer_norm_workspace_bytes(rows, planes, n), dtype=torch.uint8, device="cuda")
    wf = torch.empty(max(16, rocket.rocket_layer_norm_workspace_bytes(rows, planes, n, False)), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rocket.rocket_layer_norm(xs, w, b, planes=planes, y=ys, mean=ms, rstd=rs, workspace=wf)
        rocket.rocket_layer_norm_backward(xs, dy, ms, rs, w, planes, grad_x=out[0], grad_weight=out[1], grad_bias=out[2], workspace=ws)
    for k in range(3):
        xs.copy_(x if k != 1 else 2 * x + 1)
        graph.replay()
        torch.cuda.synchronize()
        m, r = torch.empty_like(mean), torch.empty_like(rstd)
        want = [rocket.rocket_layer_norm(xs, w, b, planes=planes, mean=m, rstd=r)] + list(rocket.rocket_layer_norm_backward(xs, dy, m, r, w, planes))
        assert all(torch.equal(a, c) for a, c in zip(want, [ys] + out))


def test_offsets_beyond_32_bits():
    """2.25e9 values: 1,000 rows again and again give the same rows again and again"""
    import torch
    rows, again, n = 1000, 1100, 2048
    x, dy, w, b = make(rows, 1, n, "bfloat16", 12)
    mean, rstd = torch.empty((2, rows, 1), device="cuda")
    y = rocket.rocket_layer_norm(x, w, b, mean=mean, rstd=rstd)
    ref = reference(x, w, b, 1, 1e-5, dy)
    xs, many, mean, rstd = x.repeat(again, 1), dy.repeat(again, 1), mean.repeat(again, 1), rstd.repeat(again, 1)
    assert xs.numel() > 1 << 31
    ys = rocket.rocket_layer_norm(xs, w, b)
    assert bool((ys.view(again, rows, n) == y).all())
    del ys
    dx, _, _ = rocket.rocket_layer_norm_backward(x, dy, mean[:rows].contiguous(), rstd[:rows].contiguous(), w)
    many, dw, db = rocket.rocket_layer_norm_backward(xs, many, mean, rstd, w, grad_x=many)
    assert bool((many.view(again, rows, n) == dx).all())
    # every sum is of at most 2,000 rows one after the other, the parts' sums are joined in fp64
    for got, want, terms in ((dw, ref["dw"], (ref["dy"] * ref["h"]).abs().sum(0)), (db, ref["db"], ref["dy"].abs().sum(0))):
        bound = again * U * (2000 * terms + (TERMS + 4) * (ref["dy"].abs() * (1 + ref["h"].abs())).sum(0))
        assert bool(((got.double().view(1, n) - again * want).abs() <= bound).all())


def test_more_rows_than_a_launch_holds():
    import torch
    rows = (1 << 28) + 5
    x = torch.arange(rows, device="cuda").remainder_(251).to(torch.bfloat16).view(rows, 1)
    w, b = torch.tensor([2.0], device="cuda"), torch.tensor([0.5], device="cuda")
    rocket.rocket_layer_norm(x, w, b, y=x)       # one value is its own mean
    assert bool((x == 0.5).all())


def test_refusals():
    import torch
    x, dy, w, b = make(4, 2, 30, "float32", 1)
    mean, rstd = torch.empty((2, 4, 2), device="cuda")

    def refused(code, f, *a, **k):
        with pytest.raises(rocket.RocketError) as e:
            f(*a, **k)
        assert e.value.code == code

    norm, back = rocket.rocket_layer_norm, rocket.rocket_layer_norm_backward
    refused(rocket.ROCKET_ESHAPE, norm, x, w, b, planes=7)
    refused(rocket.ROCKET_ESHAPE, norm, x, w, b, planes=0)
    refused(rocket.ROCKET_ESHAPE, norm, x[:0], w, b)
    refused(rocket.ROCKET_EINVAL, norm, x, w, b, eps=0.0)
    refused(rocket.ROCKET_EINVAL, norm, x, w, b, eps=float("nan"))
    refused(rocket.ROCKET_EINVAL, norm, x.double(), w, b)
    refused(rocket.ROCKET_EINVAL, norm, x.t(), w, b)
    refused(rocket.ROCKET_EINVAL, norm, x.cpu(), w, b)
    refused(rocket.ROCKET_EINVAL, norm, x, w[:-1], b)
    refused(rocket.ROCKET_EINVAL, norm, x, w.half(), b)
    refused(rocket.ROCKET_EINVAL, norm, x, w, b, planes=2, mean=mean)
    refused(rocket.ROCKET_EINVAL, norm, x, w, b, y=torch.empty((4, 59), device="cuda"))
    refused(rocket.ROCKET_EINVAL, back, x, dy.half(), mean, rstd, w, 2)
    refused(rocket.ROCKET_EINVAL, back, x, dy, mean[:3], rstd, w, 2)
    refused(rocket.ROCKET_EWORKSPACE, back, x, dy, mean, rstd, w, 2, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    refused(rocket.ROCKET_EWORKSPACE, back, x, dy, mean, rstd, w, 2,
            workspace=torch.empty(rocket.rocket_layer_norm_workspace_bytes(4, 2, 30) + 8, dtype=torch.uint8, device="cuda")[8:])
