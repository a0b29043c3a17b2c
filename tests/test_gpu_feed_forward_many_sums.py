"""Gradients of parameters over very many rows: sums of small whole numbers, whose every partial sum float holds, so that a single row left out or taken
twice shows."""
import pytest

pytestmark = pytest.mark.gpu


def _u():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from tests import feed_forward_util
    return feed_forward_util


def _whole(torch, rows, cols, lo, hi, seed, dtype):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(lo, hi + 1, (rows, cols), device="cuda", generator=g).to(dtype)


@pytest.mark.parametrize("lend", [True, False], ids=["workspace", "alone"])
@pytest.mark.parametrize("C", [5, 64, 136, 1003])
@pytest.mark.parametrize("M", [(1 << 18) + 77, (1 << 20) + 77])
def test_layer_norm_gradient(M, C, lend):
    # x, dy and the mean are whole, 1 / deviation is 1 or 2: h = (x - mean) / deviation is whole, a product with dy below 2^4 times 2^20 rows below 2^24
    import torch
    u, ig = _u(), _u().ig
    if M * C > 1 << 28:
        M = (1 << 28) // C
    h = u.handle()
    x, dy = _whole(torch, M, C, -2, 2, 1, torch.float32), _whole(torch, M, C, -1, 1, 2, torch.float32)
    mean, inv = _whole(torch, M, 1, -1, 1, 3, torch.float32), _whole(torch, M, 1, 1, 2, 4, torch.float32)
    dx, ds, db = torch.empty(M, C, device="cuda"), torch.full((C,), float("nan"), device="cuda"), torch.full((C,), float("nan"), device="cuda")
    d = ig.TensorDescriptor().set(ig.IGC_DATA_FLOAT, M, C, 1, 1, (C, 1, 1, 1))
    ws = u.Workspace(ig.get_layer_norm_backward_workspace_size(h, d, d, d) if lend else 0)
    ig.check(ig.layer_norm_backward(h, 1.0, d, x.data_ptr(), d, dy.data_ptr(), 0, mean.data_ptr(), inv.data_ptr(), ws.buf.data_ptr(), ws.size, 0.0, None, 0,
                                    d, dx.data_ptr(), 0.0, ds.data_ptr(), db.data_ptr()))
    ws.check()
    hh = dy * (x - mean) * inv
    assert float(hh.abs().max()) <= 6 and 6 * M < 1 << 24
    want = hh.double().sum(0), dy.double().sum(0)
    assert float(want[0].abs().max()) > 0 and float(want[1].abs().max()) > 0
    assert torch.equal(ds.double(), want[0])
    assert torch.equal(db.double(), want[1])


@pytest.mark.parametrize("lend", ["all", "half", "none"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,C,K", [((1 << 18) + 5, 64, 64), ((1 << 20) + 3, 33, 40), (100003, 136, 250)])
def test_filter_gradient(M, C, K, dtype, lend):
    # (parts of whole numbers this small are the numbers themselves and 2^-133, which every sum here rounds away)
    import torch
    u, ig = _u(), _u().ig
    h = u.handle()
    x, dy = _whole(torch, M, C, -3, 3, 5, u.DTYPES[dtype]), _whole(torch, M, K, -2, 2, 6, u.DTYPES[dtype])
    assert 6 * M < 1 << 24
    desc = lambda t: ig.TensorDescriptor().set(u.DATA[dtype], t.shape[0], t.shape[1], 1, 1, (t.stride(0), 1, 1, 1))
    dw, db, wd = torch.full((K, C), float("nan"), device="cuda"), torch.full((K,), float("nan"), device="cuda"), u.filter_desc("f32", K, C)
    size = ig.get_linear_backward_filter_workspace_size(h, desc(x), desc(dy), wd)
    ws = u.Workspace({"all": size, "half": size // 32 * 16, "none": 0}[lend])
    ig.check(ig.linear_backward_filter(h, 1.0, desc(x), x.data_ptr(), desc(dy), dy.data_ptr(), ws.buf.data_ptr(), ws.size, 0.0, wd, dw.data_ptr(), db.data_ptr()))
    ws.check()
    assert torch.equal(dw.double(), dy.double().t().contiguous() @ x.double())
    assert torch.equal(db.double(), dy.double().sum(0))
