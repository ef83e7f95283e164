"""Inference and training with a layer norm between features and head (rocket_infer_normed, rocket_train_step_normed)
against the library's single calls, the CPU oracle's features and gradients, and fp64.  Needs an MI355X."""
import numpy as np
import pytest

import oracle
from kernels_of import sampled
from paper_2301_08527_amd import rocket
from parity import check_backward

pytestmark = pytest.mark.gpu
LAM, SHIFT, EPS = 10.0, -3.0, 1e-5


def _gpu(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _problem(mask, B=6, C=3, L=700, K=96, u8=False, seed=0):
    rng = np.random.default_rng(seed + mask)
    h, kr = sampled(21, K, C, L)
    raw = rng.integers(0, 256, size=(B, C, L)).astype(np.uint8)
    x = oracle.znormalize_u8(raw) if u8 else rng.standard_normal((B, C, L)).astype(np.float32)
    F = bin(mask).count("1")
    model = dict(nw=(1 + 0.2 * rng.standard_normal(F * K)).astype(np.float32), nb=(0.1 * rng.standard_normal(F * K)).astype(np.float32),
                 coef=0.2 * rng.standard_normal(F * K), icpt=np.array([0.3]), y=rng.standard_normal(B).astype(np.float32))
    return h, kr, x, raw if u8 else x, F, {k: _gpu(v) for k, v in model.items()}


def _gradients(h, x, mask, F, m, max_norm):
    """the step's gradients by the library's single calls"""
    import torch
    transform, backward = ((rocket.rocket_transform_u8, rocket.rocket_soft_ppv_backward_u8) if x.dtype == torch.uint8
                           else (rocket.rocket_transform, rocket.rocket_soft_ppv_backward))
    feats = transform(h, x, mask, LAM, SHIFT)
    mean, rstd = torch.empty((2, x.shape[0], F), device="cuda")
    z = rocket.rocket_layer_norm(feats, m["nw"], m["nb"], EPS, F, mean=mean, rstd=rstd)
    pred = rocket.rocket_ridge_predict(z, m["coef"], m["icpt"])
    gz, loss = rocket.rocket_mse_grad(pred, m["y"], m["coef"])
    gf, gnw, gnb = rocket.rocket_layer_norm_backward(feats, gz, mean, rstd, m["nw"], F)
    gw, gb = backward(h, x, mask, gf, LAM, SHIFT, bool(mask & 1))
    norm = rocket.rocket_grad_norm([gw, gb, gnw, gnb], max_norm)
    return dict(feats=feats, z=z, pred=pred, loss=loss, gf=gf, gnw=gnw, gnb=gnb, gw=gw, gb=gb, norm=norm)


@pytest.mark.parametrize("mask,u8", [(4, False), (5, False), (7, True)])
def test_gradients_of_the_whole_step(mask, u8):
    """from the features on in fp64, the kernels' gradients by the oracle"""
    import torch
    h, kr, x, x_in, F, m = _problem(mask, u8=u8)
    print("normed gradients", mask, u8, flush=True)
    got = {k: v.double().cpu().numpy() for k, v in _gradients(h, _gpu(x_in), mask, F, m, 1.0).items()}
    B, K = x.shape[0], len(kr["length"])
    f = got["feats"].reshape(B, F, K)
    nw, nb, coef = (m[k].double().cpu().numpy() for k in ("nw", "nb", "coef"))
    d = f - f.mean(-1, keepdims=True)
    r = 1.0 / np.sqrt((d * d).mean(-1, keepdims=True) + EPS)
    hat = d * r
    z = (hat.reshape(B, -1) * nw + nb)
    # 64 roundings of a sum (see test_gpu_layer_norm.py) of values of a few units: 64 * 2^-24 * 8 = 3e-5
    np.testing.assert_allclose(got["z"], z, rtol=0, atol=3e-5)
    pred = z @ coef + 0.3
    # errors of z through the head: at most 3e-5 times the sum of |coef|
    slack = 3e-5 * np.abs(coef).sum()
    assert np.all(np.abs(got["pred"] - pred) <= slack)
    res = got["pred"] - m["y"].double().cpu().numpy()
    np.testing.assert_allclose(got["loss"], [(res * res).mean()], rtol=1e-12)
    gz = (2.0 / B) * res[:, None] * coef[None, :]
    scale = np.abs(gz).max()
    np.testing.assert_allclose(got["gnw"], (gz * hat.reshape(B, -1)).sum(0), rtol=0, atol=B * scale * 3e-5)
    np.testing.assert_allclose(got["gnb"], gz.sum(0), rtol=0, atol=B * scale * 1e-6)
    g = (gz * nw).reshape(B, F, K)
    gf = r * (g - g.mean(-1, keepdims=True) - hat * (g * hat).mean(-1, keepdims=True))
    np.testing.assert_allclose(got["gf"].reshape(B, F, K), gf, rtol=0, atol=float(r.max()) * scale * 1e-4)
    up = got["gf"].reshape(B, F, K)
    if not mask & 1:
        check_backward(x, kr, got["gw"], got["gb"], up[:, -1], None, LAM, SHIFT)
    else:       # kernels whose two largest outputs are too near to tell apart send the gradient to either
        o = oracle.transform(x, kr, lam=LAM)
        sel = np.nonzero(o["gap"].min(axis=0) > 1e-3)[0]
        assert len(sel) > K // 2
        check_backward(x, kr, got["gw"], got["gb"], up[:, -1], up[:, 0], LAM, SHIFT, sel=sel)
    total = np.sqrt(sum((got[k] ** 2).sum() for k in ("gw", "gb", "gnw", "gnb")))
    np.testing.assert_allclose(got["norm"], [total, min(1.0, 1.0 / total)], rtol=1e-11)


@pytest.mark.parametrize("mask,u8,recentre,max_norm", [(4, False, False, 0.05), (5, False, True, 0.05), (7, True, False, float("inf"))])
def test_step_is_its_single_calls(mask, u8, recentre, max_norm):
    import torch
    h, kr, x, x_in, F, m = _problem(mask, u8=u8)
    again, _ = sampled(21, h.K, h.C, h.L)
    xd = _gpu(x_in)
    want = _gradients(h, xd, mask, F, m, max_norm)
    if max_norm == 0.05:
        assert float(want["norm"][1]) < 1.0
    nw, nb = m["nw"].clone(), m["nb"].clone()
    loss, norm = rocket.rocket_train_step_normed(again, xd, mask, nw, nb, m["coef"], m["icpt"], m["y"], 0.25, max_norm, EPS, LAM, SHIFT, recentre)
    rocket.rocket_sgd_update_clipped(h, want["gw"], want["gb"], 0.25, want["norm"], recentre)
    rocket.rocket_sgd_tensors([m["nw"], m["nb"]], [want["gnw"], want["gnb"]], 0.25, norm=want["norm"])
    assert torch.equal(loss, want["loss"]) and torch.equal(norm, want["norm"])
    assert torch.equal(nw, m["nw"]) and torch.equal(nb, m["nb"]) and not torch.equal(nw, _problem(mask, u8=u8)[5]["nw"])
    a, b = rocket.rocket_kernels_view_get(h), rocket.rocket_kernels_view_get(again)
    assert np.array_equal(a["weights"], b["weights"]) and np.array_equal(a["bias"], b["bias"]) and not np.array_equal(a["bias"], kr["bias"])


@pytest.mark.parametrize("B,u8", [(1, True), (5, False)])
def test_inference_is_its_single_calls(B, u8):
    import torch
    for mask in (1, 3, 7):
        h, kr, x, x_in, F, m = _problem(mask, B=B, u8=u8)
        xd = _gpu(x_in)
        feats = (rocket.rocket_transform_u8 if u8 else rocket.rocket_transform)(h, xd, mask, LAM, SHIFT)
        for nw, nb in ((m["nw"], m["nb"]), (None, None)):
            want = rocket.rocket_layer_norm(feats, nw, nb, EPS, F)
            pred, got = rocket.rocket_infer_normed(h, xd, mask, nw, nb, m["coef"], m["icpt"], EPS, LAM, SHIFT)
            assert torch.equal(got, want) and torch.equal(pred, rocket.rocket_ridge_predict(want, m["coef"], m["icpt"]))


def test_steps_in_a_graph():
    """two steps captured together and replayed: the same parameters as four steps in turn"""
    import torch
    mask = 5
    a, _, _, x_in, F, m = _problem(mask)
    b = _problem(mask)[0]
    xd = _gpu(x_in)
    pa, pb = ([m["nw"].clone(), m["nb"].clone()] for _ in range(2))
    rocket.rocket_transform(b, xd, mask, LAM, SHIFT)       # uploads the parameters
    ws = torch.empty(rocket.rocket_train_normed_workspace_bytes(b, len(x_in), mask), dtype=torch.uint8, device="cuda")
    norm = torch.empty(2, dtype=torch.float64, device="cuda")

    def step(h, p, **k):
        return rocket.rocket_train_step_normed(h, xd, mask, p[0], p[1], m["coef"], m["icpt"], m["y"], 0.1, 0.5, EPS, LAM, SHIFT, **k)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        for _ in range(2):
            loss, _ = step(b, pb, norm=norm, workspace=ws)
    want = [step(a, pa) for _ in range(4)]
    for k in (1, 3):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(loss, want[k][0]) and torch.equal(norm, want[k][1])
    assert all(torch.equal(u, v) for u, v in zip(pa, pb))
    torch.cuda.synchronize()
    va, vb = rocket.rocket_kernels_view_get(a), rocket.rocket_kernels_view_get(b)
    assert np.array_equal(va["weights"], vb["weights"]) and np.array_equal(va["bias"], vb["bias"])


def test_refusals_leave_the_parameters():
    import torch
    h, kr, x, x_in, F, m = _problem(5)
    xd = _gpu(x_in)
    nw, nb = m["nw"].clone(), m["nb"].clone()

    def refused(*a, **k):
        with pytest.raises(rocket.RocketError):
            rocket.rocket_train_step_normed(*a, **k)

    args = (nw, nb, m["coef"], m["icpt"], m["y"])
    refused(h, xd, 3, *args, 0.1)
    refused(h, xd, 5, *args, float("nan"))
    refused(h, xd, 5, *args, 0.1, max_norm=0.0)
    refused(h, xd, 5, *args, 0.1, eps=0.0)
    refused(h, xd[:, :, :-1].contiguous(), 5, *args, 0.1)
    refused(h, xd, 5, nw[:-1], nb, *args[2:], 0.1)
    refused(h, xd, 5, None, nb, *args[2:], 0.1)
    refused(h, xd, 5, *args, 0.1, workspace=torch.empty(1 << 12, dtype=torch.uint8, device="cuda"))
    both = torch.ones(nw.numel() + 1, device="cuda")
    refused(h, xd, 5, both[:-1], both[1:], *args[2:], 0.1)
    assert torch.equal(nw, m["nw"]) and torch.equal(nb, m["nb"]) and bool((both == 1.0).all())
    view = rocket.rocket_kernels_view_get(h)
    assert np.array_equal(view["weights"], kr["weights"])
