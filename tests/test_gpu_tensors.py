"""Many tensors at once (rocket_grad_norm, rocket_grad_clip, rocket_sgd_tensors, rocket_sgd_update_clipped) against the
formulas in fp64.  Needs an MI355X.

Tolerances.  The norm is a sum of squares in fp64, each addition off by 2^-53 of the sum: N values, at most N * 2^-53
relative in the sum, half of it in the norm.  A scaled value is one product in fp64, rounded to 32 bits (2^-24) and to its
type (half a step); an updated one is one multiply-add in fp64 of an exact product, rounded to 32 bits."""
import math

import numpy as np
import pytest

from paper_2301_08527_amd import rocket

pytestmark = pytest.mark.gpu
TYPES = ("float32", "bfloat16", "float16")


def make(sizes, types, seed, scale=1.0, unaligned=False):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    out = []
    for n, t in zip(sizes, types):
        v = (scale * torch.randn(n + 1, generator=g, device="cuda")).to(getattr(torch, t))
        out.append(v[1:] if unaligned else v[1:].clone())
    return out


def exact_norm(grads):
    return math.sqrt(math.fsum(float(g.double().square().sum()) for g in grads))


def smallest(dtype):
    import torch
    return {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}[dtype]


def check_scaled(got, g, c):
    import torch
    want = g.double() * c
    tol = (torch.finfo(g.dtype).eps / 2 + 2.0 ** -24 + 1e-9) * want.abs() + smallest(g.dtype) / 2 * 1.001
    assert bool(((got.double() - want).abs() <= tol).all())


def check_norm(norm, grads, max_norm):
    n = sum(g.numel() for g in grads)
    want = exact_norm(grads)
    told = norm.cpu().numpy()
    assert abs(told[0] - want) <= (n + 8) * 2.0 ** -53 * want
    assert told[1] == (1.0 if told[0] <= max_norm else max_norm / told[0])
    return float(told[1])


LISTS = [([1], 1), ([7], 1), ([2047, 2048, 2049], 1), ([0, 5, 0], 1), ([1] * 500, 3), ([314, 100, 200, 200], 1), ([100003, 1, 8191, 8193, 65536], 3),
         ([3000001], 1), ([257 + 13 * i for i in range(200)], 3), ([0] * 150 + [77] * 150, 3), ([5000011, 3, 2500003], 3)]


@pytest.mark.parametrize("unaligned", [False, True])
@pytest.mark.parametrize("sizes,kinds", LISTS, ids=lambda v: str(len(v)) + "x" + str(v[-1]) if isinstance(v, list) else str(v))
def test_clip_and_update(sizes, kinds, unaligned):
    import torch
    for shift in range(3 if kinds == 1 else 1):
        types = [TYPES[(i * (kinds > 1) + shift) % 3] for i in range(len(sizes))]
        print(len(sizes), types[0], unaligned, flush=True)
        grads = make(sizes, types, len(sizes) + shift, unaligned=unaligned)
        full = exact_norm(grads)
        for max_norm in (0.37 * full, 2.0 * full + 1.0):
            ws = torch.full((rocket.rocket_grad_workspace_bytes(grads) // 8,), float("nan"), dtype=torch.float64, device="cuda")
            c = check_norm(rocket.rocket_grad_norm(grads, max_norm, workspace=ws), grads, max_norm)
            # into tensors of their own, which lie one behind the other: each is written to its end and no further
            flat = {t: torch.full((sum(n for n, u in zip(sizes, types) if u == t) + 9,), 3.0, dtype=getattr(torch, t), device="cuda") for t in TYPES}
            at, out = dict.fromkeys(TYPES, 0), []
            for n, t in zip(sizes, types):
                out.append(flat[t][at[t]:at[t] + n])
                at[t] += n
            ws.fill_(float("nan"))
            norm = rocket.rocket_grad_clip(grads, max_norm, out=out, workspace=ws)
            assert check_norm(norm, grads, max_norm) == c
            for g, o in zip(grads, out):
                check_scaled(o, g, c)
            assert all(bool((f[at[t]:] == 3.0).all()) for t, f in flat.items())
            mine = [g.clone() for g in grads]
            assert torch.equal(rocket.rocket_grad_clip(mine, max_norm), norm)
            assert all(torch.equal(m, o) for m, o in zip(mine, out))
            if c == 1.0:
                assert all(torch.equal(m, g) for m, g in zip(mine, grads))
            params = make(sizes, ["float32"] * len(sizes), 99, unaligned=unaligned)
            kept = [p.clone() for p in params]
            new = [torch.empty_like(p) for p in params]
            rocket.rocket_sgd_tensors(params, grads, 0.3, norm=norm, out=new)
            assert all(torch.equal(p, k) for p, k in zip(params, kept))
            for p, g, q in zip(params, grads, new):
                want = p.double() - 0.3 * c * g.double()
                assert bool(((q.double() - want).abs() <= 2.0 ** -24 * want.abs() * 1.001 + 1e-12 * g.double().abs()).all())
            rocket.rocket_sgd_tensors(params, grads, 0.3, norm=norm)
            assert all(torch.equal(p, q) for p, q in zip(params, new))


def test_offsets_beyond_32_bits():
    import torch
    base = make([1 << 20], ["bfloat16"], 3)[0]
    big = base.repeat(2100)
    assert big.numel() > 1 << 31
    one = exact_norm([base])
    norm = rocket.rocket_grad_clip([big], 0.5 * one)
    assert abs(float(norm[0]) / (one * math.sqrt(2100)) - 1) < 1e-9
    small = [base.clone()]
    c = float(norm[1])
    assert bool((big.view(2100, -1) == (small[0].double() * c).to(torch.float32).to(torch.bfloat16)).all())


def test_update_without_a_norm():
    import torch
    p, g = make([1000, 33], ["float32"] * 2, 1), make([1000, 33], ["bfloat16", "float32"], 2)
    want = [a.double() - 0.1 * b.double() for a, b in zip(p, g)]
    rocket.rocket_sgd_tensors(p, g, 0.1)
    assert all(bool(((a.double() - w).abs() <= 2.0 ** -24 * 1.001 * w.abs() + 1e-12).all()) for a, w in zip(p, want))


def test_no_overflow_no_loss_of_small_values():
    import torch
    big = [torch.full((1000,), 3e38, device="cuda"), torch.full((7,), -3e38, device="cuda")]
    norm = rocket.rocket_grad_clip(big, 1.0)
    assert abs(float(norm[0]) / (float(np.float32(3e38)) * math.sqrt(1007)) - 1) < 1e-12
    assert bool(((big[0].double() * math.sqrt(1007) - 1).abs() < 2.0 ** -23).all())      # the coefficient, 1e-40, has no digits in fp32
    small = [torch.full((4000,), 1e-44, device="cuda")]
    value = float(small[0][0].double())
    norm = rocket.rocket_grad_norm(small, 1e-50)
    assert abs(float(norm[0]) / (value * math.sqrt(4000)) - 1) < 1e-12 and float(norm[1]) < 1e-5
    zero = [torch.zeros(100, device="cuda"), torch.zeros(3, dtype=torch.float16, device="cuda")]
    assert rocket.rocket_grad_clip(zero, 1e-30).tolist() == [0.0, 1.0] and bool((zero[0] == 0).all())
    empty = [torch.empty(0, device="cuda")]
    assert rocket.rocket_grad_clip(empty, 1.0).tolist() == [0.0, 1.0]


@pytest.mark.parametrize("tensors", [16, 17, 165, 166, 220, 221, 330, 331, 662])
def test_lists_of_one_launch_and_one_more(tensors):
    """Tensors of all types, with empty ones among them and several units in some, as many as a launch's records hold and one more."""
    import torch
    sizes = [1 + 2917 * i % 9001 + (20011 if i % 29 == 3 else 0) for i in range(tensors)]
    for i in range(0, tensors, 11):
        sizes.insert(i, 0)
    grads = make(sizes, [TYPES[i % 3] for i in range(len(sizes))], tensors)
    params = make(sizes, ["float32"] * len(sizes), tensors + 1)
    max_norm = 0.37 * exact_norm(grads)
    out = [torch.full_like(g, 3.0) for g in grads]
    norm = rocket.rocket_grad_clip(grads, max_norm, out=out)
    c = check_norm(norm, grads, max_norm)
    new = [torch.full_like(p, 3.0) for p in params]
    rocket.rocket_sgd_tensors(params, grads, 0.25, norm=norm, out=new)
    for g, o, p, q in zip(grads, out, params, new):
        check_scaled(o, g, c)
        want = p.double() - 0.25 * c * g.double()
        # one rounding to 32 bits, and fp64's in the product and the difference
        tol = 2.0 ** -24 * want.abs() + 2.0 ** -51 * (p.double().abs() + g.double().abs()) + 2.0 ** -150
        assert bool(((q.double() - want).abs() <= tol).all())


@pytest.mark.parametrize("where", [0, 5000, 99999])
def test_infinities_and_nan(where):
    import torch
    for t in TYPES:
        g = make([100000, 10], [t, "float32"], 7)
        g[0][where] = float("inf")
        norm = rocket.rocket_grad_clip(g, 1.0)
        assert norm.tolist() == [math.inf, 0.0]
        assert bool(g[0][where].isnan()) and int(g[0].isnan().sum()) == 1 and bool((g[1] == 0).all())
        g[0][where] = float("nan")
        norm = rocket.rocket_grad_clip(g, 1.0)
        assert bool(norm.isnan().all()) and bool(g[0].isnan().all()) and bool(g[1].isnan().all())
        # never clips, whatever the norm
        g = make([1000], [t], 8)
        kept = g[0].clone()
        assert float(rocket.rocket_grad_clip(g, math.inf)[1]) == 1.0 and torch.equal(kept, g[0])


def test_same_bits_on_a_stream_and_in_a_graph():
    import torch
    sizes = [257 + 1301 * i for i in range(120)]
    types = [TYPES[i % 3] for i in range(120)]
    grads, params = make(sizes, types, 31), make(sizes, ["float32"] * 120, 32)
    lists = rocket.rocket_tensors(grads), rocket.rocket_tensors(params)
    new = [torch.empty_like(p) for p in params]
    norm = rocket.rocket_grad_norm(lists[0], 10.0)
    rocket.rocket_sgd_tensors(lists[1], lists[0], 0.5, norm=norm, out=new)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    norm2 = rocket.rocket_grad_norm(grads, 10.0, stream=side)
    new2 = [torch.empty_like(p) for p in params]
    side.wait_stream(torch.cuda.current_stream())
    rocket.rocket_sgd_tensors(params, grads, 0.5, norm=norm2, out=new2, stream=side)
    side.synchronize()
    assert torch.equal(norm, norm2) and all(torch.equal(a, b) for a, b in zip(new, new2))
    # two graphs with one workspace, replayed in turn
    ws = torch.empty(rocket.rocket_grad_workspace_bytes(lists[0]), dtype=torch.uint8, device="cuda")
    told = [torch.empty(2, dtype=torch.float64, device="cuda") for _ in range(2)]
    out = [[torch.empty_like(g) for g in grads] for _ in range(2)]
    graphs = []
    for k in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            rocket.rocket_grad_clip(grads, 10.0 * (k + 1), out=out[k], norm=told[k], workspace=ws)
            rocket.rocket_sgd_tensors(params, grads, 0.5, norm=told[k], out=new2)
        graphs.append(graph)
    for k in (0, 1, 0, 1):
        grads[3].mul_(1.5)
        graphs[k].replay()
        torch.cuda.synchronize()
        want = [torch.empty_like(g) for g in grads]
        norm = rocket.rocket_grad_clip(grads, 10.0 * (k + 1), out=want)
        rocket.rocket_sgd_tensors(params, grads, 0.5, norm=norm, out=new)
        assert torch.equal(norm, told[k]) and all(torch.equal(a, b) for a, b in zip(want, out[k])) and all(torch.equal(a, b) for a, b in zip(new, new2))


def test_kernels_update_with_the_coefficient():
    import torch
    a, b = (rocket.rocket_make_kernels(5, 300, 4, 900) for _ in range(2))
    gw, gb = make([a.total_weights, a.K], ["float32"] * 2, 3)
    norm = rocket.rocket_grad_norm([gw, gb], 1.0)
    assert float(norm[1]) < 1.0
    before = rocket.rocket_kernels_view_get(a)
    rocket.rocket_sgd_update_clipped(a, gw, gb, 0.5, norm, recentre=True)
    # the same update with the rate rounded as the kernel rounds it
    rocket.rocket_sgd_update(b, gw, gb, float(np.float32(np.float64(np.float32(0.5)) * float(norm[1]))), recentre=True)
    va, vb = rocket.rocket_kernels_view_get(a), rocket.rocket_kernels_view_get(b)
    assert np.array_equal(va["weights"], vb["weights"]) and np.array_equal(va["bias"], vb["bias"])
    assert not np.array_equal(va["bias"], before["bias"])
    one = torch.tensor([0.5, 1.0], dtype=torch.float64, device="cuda")
    rocket.rocket_sgd_update_clipped(a, gw, gb, 0.25, one)
    rocket.rocket_sgd_update(b, gw, gb, 0.25)
    va, vb = rocket.rocket_kernels_view_get(a), rocket.rocket_kernels_view_get(b)
    assert np.array_equal(va["weights"], vb["weights"]) and np.array_equal(va["bias"], vb["bias"])


def test_refusals():
    import torch

    def refused(code, f, *a, **k):
        with pytest.raises(rocket.RocketError) as e:
            f(*a, **k)
        assert e.value.code == code

    g = make([100, 7], ["float32"] * 2, 1)
    E = rocket.ROCKET_EINVAL
    refused(E, rocket.rocket_grad_norm, [])
    refused(E, rocket.rocket_grad_norm, [g[0].double()])
    refused(E, rocket.rocket_grad_norm, [g[0].cpu()])
    refused(E, rocket.rocket_grad_norm, [g[0][::2]])
    refused(E, rocket.rocket_grad_clip, g, 0.0)
    refused(E, rocket.rocket_grad_clip, g, -1.0)
    refused(E, rocket.rocket_grad_clip, g, float("nan"))
    refused(E, rocket.rocket_grad_clip, g, 1.0, norm=torch.empty(2, device="cuda"))
    refused(rocket.ROCKET_ESHAPE, rocket.rocket_grad_clip, g, 1.0, out=g[:1])
    refused(E, rocket.rocket_grad_clip, g, 1.0, out=g[::-1])
    refused(E, rocket.rocket_grad_clip, g, 1.0, out=[t.half() for t in g])
    refused(rocket.ROCKET_EWORKSPACE, rocket.rocket_grad_norm, g, workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))
    refused(E, rocket.rocket_sgd_tensors, [t.half() for t in g], g, 0.1)
    refused(E, rocket.rocket_sgd_tensors, g, g[::-1], 0.1)
    refused(E, rocket.rocket_sgd_tensors, g, g, float("inf"))
