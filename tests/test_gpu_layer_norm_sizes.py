"""The layer norm at sizes where its launches, its sums over rows and its ranges end (rocket_layer_norm, rocket_layer_norm_backward).
Needs an MI355X."""
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
