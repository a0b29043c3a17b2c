"""More rows, and more tiles, than the plain kernels have workgroups: they walk.

Tolerances.  e = 2^-24; a sum of C = 5 elements in any order is off by at most (C + 4) e of its magnitudes' sum."""
import pytest

pytestmark = pytest.mark.gpu

E = 2.0 ** -24


def _u():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from tests import feed_forward_util
    return feed_forward_util


def test_layer_norm_of_many_short_rows():
    import torch
    u, ig = _u(), _u().ig
    h, M, C, eps = u.handle(), (1 << 20) + 77, 5, 1e-5
    g = torch.Generator(device="cuda").manual_seed(3)
    x, dy = (torch.randn(M, C, device="cuda", generator=g) for _ in range(2))
    y, dx = (torch.full((M, C), float("nan"), device="cuda") for _ in range(2))
    mean, inv = (torch.full((M,), float("nan"), device="cuda") for _ in range(2))
    ds, db = (torch.full((C,), float("nan"), device="cuda") for _ in range(2))
    d = ig.TensorDescriptor().set(ig.IGC_DATA_FLOAT, M, C, 1, 1, (C, 1, 1, 1))
    ig.check(ig.layer_norm_forward(h, 1.0, d, x.data_ptr(), 0, 0, eps, 0.0, d, y.data_ptr(), mean.data_ptr(), inv.data_ptr()))
    size = ig.get_layer_norm_backward_workspace_size(h, d, d, d)
    ws = u.Workspace(size)
    ig.check(ig.layer_norm_backward(h, 1.0, d, x.data_ptr(), d, dy.data_ptr(), 0, mean.data_ptr(), inv.data_ptr(), ws.buf.data_ptr(), size, 0.0,
                                    None, 0, d, dx.data_ptr(), 0.0, ds.data_ptr(), db.data_ptr()))
    ws.check()
    wide = x.double()
    wm = wide.mean(1, keepdim=True)
    dev = wide - wm
    wi = 1 / (dev.square().mean(1, keepdim=True) + eps).sqrt()
    em = (C + 4) * E * wide.abs().mean(1, keepdim=True)
    ei = wi * (2 * (C + 8) * E + wi * wi * 2 * em * dev.abs().mean(1, keepdim=True) + wi * wi * em * em)
    assert bool(((mean.double() - wm[:, 0]).abs() <= em[:, 0] + 1e-300).all())
    assert bool(((inv.double() - wi[:, 0]).abs() <= (ei + 4 * E * wi)[:, 0]).all())
    assert bool(((y.double() - dev * wi).abs() <= em * wi + dev.abs() * (ei + 6 * E * wi) + 6 * E * (dev * wi).abs() + 1e-30).all())
    # the gradient from the mean and deviation that were kept
    hm, hi, q = mean.double()[:, None], inv.double()[:, None], dy.double()
    hh = (wide - hm) * hi
    want = hi * (q - q.mean(1, keepdim=True) - hh * (q * hh).mean(1, keepdim=True))
    mag = (wide - hm).abs() * hi + (hm * hi).abs() * 2
    tol = hi * ((C + 8) * E * q.abs().mean(1, keepdim=True) + (C + 16) * E * mag * (q.abs() * mag).mean(1, keepdim=True) + 8 * E * q.abs())
    assert bool(((dx.double() - want).abs() <= tol + 2 * E * want.abs() + 1e-30).all())
    assert bool(((ds.double() - (q * hh).sum(0)).abs() <= (M + 8) * E * (q.abs() * mag).sum(0)).all())
    assert bool(((db.double() - q.sum(0)).abs() <= (M + 8) * E * q.abs().sum(0)).all())


def test_product_of_many_rows():
    # one product per result: two roundings at most
    import torch
    u, ig = _u(), _u().ig
    h, M = u.handle(), (1 << 28) + 70
    x = torch.randn(M, device="cuda", generator=torch.Generator(device="cuda").manual_seed(4))
    y = torch.full((M + 64,), float("nan"), device="cuda")
    w = torch.tensor([1.7], device="cuda")
    d = ig.TensorDescriptor().set(ig.IGC_DATA_FLOAT, M, 1, 1, 1, (1, 1, 1, 1))
    ig.check(ig.linear_forward(h, 1.0, d, x.data_ptr(), u.filter_desc("f32", 1, 1), w.data_ptr(), 0, 0, 0, ig.IGC_ACTIVATION_IDENTITY, 0.0, None, 0, d,
                               0, y.data_ptr()))
    want = x * w
    assert bool(((y[:M] - want).abs() <= 4 * E * want.abs() + 1e-37).all())
    assert bool(torch.isnan(y[M:]).all())
