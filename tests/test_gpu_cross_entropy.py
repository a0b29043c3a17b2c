"""Cross entropy over a vocabulary and its gradients on the GPU, element by element against the formulas in 64 bits.

Tolerances.  e = 2^-24.  A logit: a sum of C products and the bias, (C + 4) e of the products' magnitudes (float: products in three bfloat16 parts leave out 2^-21 +
2^-30 of each), and e (|z| + |bias|).  exp(d) is off by 2 e |d| + 4 e of itself; a logarithm of a sum by the logits' errors at most, by the average of the exponentials'
and by its additions, no chain of which has more than 300; then half a step.  dz: its exponential's error and, of the logits' and logarithms', e^error - 1 of it; 4 e of the
terms; rounded to bfloat16 to the number next to it, or to either of two where its error reaches a border (at most 32 rows, and at the targets: in two parts, 2^-16).  A product of n terms with dz: dz's errors and (n + 8) e (float: and 2^-21 + 2^-30) of the terms, half a step
of the result, and of the sum over the pieces e for each piece."""
import pytest

pytestmark = pytest.mark.gpu

import torch

from oracle import cross_entropy_oracle as co

E = 2.0 ** -24
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
PART = {"f32": 2.0 ** -21 + 2.0 ** -30, "bf16": 0.0}


def _u():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from tests import feed_forward_util
    return feed_forward_util


def near(got, want, tol, what):
    assert got.shape == want.shape, what
    bad = ~((got.double() - want).abs() <= tol)
    if bool(bad.any()):
        i = tuple(int(v) for v in bad.nonzero()[0])
        raise AssertionError("%s: %d of %d off; %s: %.9g instead of %.9g, allowed %.3g" % (what, int(bad.sum()), bad.numel(), i, got[i], want[i], tol.expand(want.shape)[i]))


class Case:
    def __init__(self, M, C, V, dtype="bf16", layout=(0, 0), bias=False, seed=0, lost=0.2, size=2.0):
        u, ig = _u(), _u().ig
        self.g = torch.Generator(device="cuda").manual_seed(seed + M + 13 * C + 101 * V)
        rand = lambda *s: torch.randn(*s, generator=self.g, device="cuda")
        self.M, self.C, self.V, self.dtype, self.layout = M, C, V, dtype, layout
        self.X = u.Rows((M, C), dtype, *layout)
        self.X.view.copy_(rand(M, C))
        self.w = (rand(V, C) * size / C ** 0.5).to(u.DTYPES[dtype])
        self.bias = rand(V) if bias else None
        t = torch.randint(0, V, (M,), generator=self.g, device="cuda")
        gone = torch.rand(M, generator=self.g, device="cuda") < lost
        other = torch.tensor([-100, -1, V, 2 ** 31 - 1, -2 ** 31], device="cuda")[torch.randint(0, 5, (M,), generator=self.g, device="cuda")]
        self.t = torch.where(gone, other, t).to(torch.int32)
        self.wd, self.h = u.filter_desc(dtype, V, C), u.handle()

    def forward(self, keep=True, stream=None):
        u, ig = _u(), _u().ig
        size = ig.get_linear_cross_entropy_forward_workspace_size(self.h, self.X.desc, self.wd)
        ws = u.Workspace(size)
        loss, log_sum = (torch.full((self.M + 8,), float("nan"), device="cuda") for _ in range(2))
        ig.check(ig.linear_cross_entropy_forward(self.h, self.X.desc, self.X.ptr, self.wd, self.w.data_ptr(), u.ptr(self.bias), self.t.data_ptr(), ws.buf.data_ptr(), size,
                                                 loss.data_ptr(), log_sum.data_ptr() if keep else 0), "igcLinearCrossEntropyForward")
        ws.check()
        assert bool(loss[self.M:].isnan().all()) and bool(log_sum[self.M if keep else 0:].isnan().all())
        return loss[:self.M], log_sum[:self.M]

    def exact(self):
        x, w = self.X.view.double(), self.w.double()
        b = None if self.bias is None else self.bias.double()
        loss, log_sum, z = co.forward(x, w, b, self.t)
        size = x.abs() @ w.abs().t()
        tz = ((self.C + 4) * E + PART[self.dtype]) * size + E * (z.abs() + (0 if b is None else b.abs()))
        return loss, log_sum, z, tz

    def check_forward(self):
        loss, log_sum = self.forward()
        wl, ws, z, tz = self.exact()
        most = z.amax(1, keepdim=True)
        p = torch.exp(z - ws[:, None])
        ts = (p * torch.where(p > 0, tz + 2 * E * (z - most).abs(), 0.0)).sum(1) * 1.01 + 310 * E + 2 * E * (ws.abs() + most[:, 0].abs())
        at = torch.where((self.t >= 0) & (self.t < self.V), self.t, 0).long()[:, None]
        near(log_sum, ws, ts, "log_sum %s" % ((self.M, self.C, self.V, self.dtype, self.layout),))
        near(loss, wl, ts + tz.gather(1, at)[:, 0] + 2 * E * wl.abs(), "loss %s" % ((self.M, self.C, self.V, self.dtype, self.layout),))
        assert bool((loss[(self.t < 0) | (self.t >= self.V)] == 0).all())

    def backward(self, dx="bf16", dw="bf16", dbias=True, alpha=1.0, beta=0.0, pbeta=0.0, ones=False):
        """{name: (got, old)}; and the inputs logSum and dloss."""
        u, ig = _u(), _u().ig
        rand = lambda *s: torch.randn(*s, generator=self.g, device="cuda")
        _, log_sum, _, _ = self.exact()
        self.log_sum, self.dloss = log_sum.float(), None if ones else rand(self.M)
        self.dloss_given = torch.where((self.t >= 0) & (self.t < self.V), self.dloss, float("nan")) if not ones else None     # (not read into anything elsewhere)
        old = lambda n, rows, t, f: (0.01 * rand(rows, n)).to(u.DTYPES[t]) if f else torch.full((rows, n), float("nan"), device="cuda").to(u.DTYPES[t])
        out = {}
        DX = DW = DB = None
        if dx:
            DX = u.Rows((self.M, self.C), dx, *self.layout)
            DX.view.copy_(old(self.C, self.M, dx, beta))
            out["dx"] = DX.view.clone()
        if dw:
            DW = torch.full((self.V * self.C + 64,), u.GUARD, dtype=u.DTYPES[dw], device="cuda")
            DW[:self.V * self.C] = old(self.C, self.V, dw, pbeta).view(-1)
            out["dw"] = DW[:self.V * self.C].view(self.V, self.C).clone()
        if dbias:
            DB = torch.full((self.V + 64,), u.GUARD, device="cuda")
            DB[:self.V] = old(self.V, 1, "f32", pbeta)[0]
            out["dbias"] = DB[:self.V].clone()
        dwd = u.filter_desc(dw, self.V, self.C) if dw else None
        size = ig.get_linear_cross_entropy_backward_workspace_size(self.h, self.X.desc, self.wd, DX.desc if dx else None, dwd)
        ws = u.Workspace(size)
        ig.check(ig.linear_cross_entropy_backward(self.h, alpha, self.X.desc, self.X.ptr, self.wd, self.w.data_ptr(), u.ptr(self.bias), self.t.data_ptr(),
                                                  self.log_sum.data_ptr(), u.ptr(self.dloss_given), ws.buf.data_ptr(), size, beta, DX.desc if dx else None, u.ptr(DX), pbeta,
                                                  dwd, u.ptr(DW), u.ptr(DB)), "igcLinearCrossEntropyBackward")
        ws.check()
        if dw:
            assert bool((DW[self.V * self.C:] == u.GUARD).all())
        if dbias:
            assert bool((DB[self.V:] == u.GUARD).all())
        got = {}
        if dx:
            got["dx"] = (torch.from_numpy(DX.numpy()).cuda(), out["dx"].double())
        if dw:
            got["dw"] = (DW[:self.V * self.C].view(self.V, self.C).double(), out["dw"].double())
        if dbias:
            got["dbias"] = (DB[:self.V].double(), out["dbias"].double())
        return got

    def check_backward(self, dx="bf16", dw="bf16", dbias=True, alpha=1.0, beta=0.0, pbeta=0.0, ones=False, pieces=1, entries=slice(None)):
        """entries: of the vocabulary, where dw is looked at"""
        got = self.backward(dx, dw, dbias, alpha, beta, pbeta, ones)
        _, _, z, tz = self.exact()
        s = self.log_sum.double()
        d = torch.ones(self.M, dtype=torch.float64, device="cuda") if ones else self.dloss.double()
        dz = alpha * co.slopes(z, s, self.t, d)
        there = ((self.t >= 0) & (self.t < self.V))[:, None]
        size = torch.where(there, abs(alpha) * d.abs()[:, None] * torch.exp(z - s[:, None]), 0.0)
        tdz = size * (torch.expm1(tz) + 2 * E * (z - s[:, None]).abs() + 8 * E) + 8 * E * dz.abs()
        tsum = tdz.sum(0) + (self.M + 8) * E * dz.abs().sum(0)
        # dz as the products take it: from the lowest to the highest number that it may have been rounded to
        fine = (torch.arange(self.V, device="cuda")[None, :] == self.t[:, None]) | (self.M <= 32) | (self.dtype == "f32")
        parts = tdz + (0.0 if self.dtype == "f32" else 2.0 ** -16) * (dz.abs() + tdz)
        low, high = (torch.where(fine, dz + f, (dz + q).float().to(torch.bfloat16).double()) for q, f in ((-tdz, -parts), (tdz, parts)))
        dbz, dz, tdz = dz.sum(0), (low + high) / 2, (high - low) / 2
        x, w = self.X.view.double(), self.w.double()
        what = str((self.M, self.C, self.V, self.dtype, self.layout, dx, dw, alpha, beta, pbeta))

        def check(name, want, tol, scale, out):
            have, old = got[name]
            if scale:
                want = want + scale * old
                tol = tol + 4 * E * (scale * old).abs()
            near(have, want, tol + HALF[out] * (want.abs() + tol) + 1e-37, name + " " + what)

        if dbias:
            check("dbias", dbz, tsum, pbeta, "f32")
        if dx:
            sizes = (dz.abs() + tdz) @ w.abs()
            check("dx", dz @ w, tdz @ w.abs() + ((self.V + 8 + 2 * pieces) * E + PART[self.dtype]) * sizes, beta, dx)
        if dw:
            dz, tdz = dz[:, entries], tdz[:, entries]
            sizes = (dz.abs() + tdz).t() @ x.abs()
            got["dw"] = tuple(v[entries] for v in got["dw"])
            check("dw", dz.t() @ x, tdz.t() @ x.abs() + ((self.M + 8) * E + PART[self.dtype]) * sizes, pbeta, dw)


LAYOUTS = [(0, 0), (3, 1), (8, 8), (1, 0)]
SIZES = [(1, 1, 1), (1, 8, 2), (3, 5, 7), (1, 64, 1000), (2, 100, 257), (5, 33, 2049), (16, 128, 300), (63, 77, 511), (64, 256, 2048), (65, 200, 4100), (130, 64, 5003), (257, 130, 129),
         (300, 512, 1030)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", LAYOUTS, ids=str)
def test_loss(layout, dtype):
    for i, (M, C, V) in enumerate(SIZES):
        print("loss", dtype, layout, M, C, V, flush=True)
        Case(M, C, V, dtype, layout, bias=i % 2 == 0).check_forward()


@pytest.mark.parametrize("types", [("bf16", "bf16", "bf16"), ("bf16", "f32", "f32"), ("bf16", "f32", "bf16"), ("f32", "f32", "f32")], ids="-".join)
@pytest.mark.parametrize("layout", LAYOUTS, ids=str)
def test_gradients(layout, types):
    dtype, dx, dw = types
    for i, (M, C, V) in enumerate(SIZES):
        print("loss gradients", types, layout, M, C, V, flush=True)
        c = Case(M, C, V, dtype, layout, bias=i % 2 == 1)
        c.check_backward(dx, dw, dbias=i % 3 != 0, alpha=1.0 if i % 4 else 0.5, beta=(0.0, 1.0, -2.0)[i % 3], pbeta=(0.0, 0.0, 1.0, 0.5)[i % 4], ones=i % 5 == 4)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_one_gradient_at_a_time(dtype):
    c = Case(70, 96, 300, dtype, bias=True)
    for ask in ((dtype, None, False), (None, dtype, False), (None, None, True), (None, dtype, True), (dtype, None, True)):
        c.check_backward(*ask)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_several_pieces(dtype):
    """More logits than are made at a time: rows and entries that divide into pieces, or not."""
    for M, C, V in ((2048, 64, 40000), (5000, 72, 20011)):
        c = Case(M, C, V, dtype, (8, 8) if M > 4096 else (0, 0), bias=True)
        c.check_forward()
        c.check_backward(dtype, dtype, True, beta=1.0, pieces=4)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_tiles(dtype):
    Case(1100, 520, 6000, dtype).check_forward()
    Case(1100, 520, 6000, dtype).check_backward(dtype, dtype)
    Case(4, 1024, 70000, dtype).check_forward()
    Case(4, 1024, 70000, dtype).check_backward(dtype, dtype)


@pytest.mark.parametrize("types", [("bf16", "bf16", "bf16"), ("bf16", "f32", "f32"), ("f32", "f32", "f32")], ids="-".join)
def test_few_tokens(types):
    """One and two pieces of sixteen tokens, short and long rows, vocabularies of few and of many entries; thirty-three tokens."""
    dtype, dx, dw = types
    for i, (M, C, V) in enumerate([(1, 4100, 700), (9, 136, 40000), (17, 96, 9000), (32, 130, 515), (20, 1027, 20011), (16, 2048, 8192), (3, 129, 8193), (30, 80, 40001), (33, 96, 9000)]):
        print("few tokens", types, M, C, V, flush=True)
        c = Case(M, C, V, dtype, LAYOUTS[i % 4], bias=i % 2 == 0)
        c.check_forward()
        c.check_backward(dx, dw, beta=(0.0, 1.0)[i % 2], pbeta=(0.0, 1.0, -0.5)[i % 3], alpha=1.0 if i % 3 else 2.0)
    # nearly all of a row's gradient is its target's: two parts hold it to 2^-16
    if dtype == "bf16":
        c = Case(1, 64, 50, "bf16", lost=0.0)
        got = c.backward("f32", "f32", dbias=False)
        dz = co.slopes(c.exact()[2], c.log_sum.double(), c.t, c.dloss.double())
        for name, want in (("dx", dz @ c.w.double()), ("dw", dz.t() @ c.X.view.double())):
            assert float((got[name][0] - want).norm() / want.norm()) < 2.0 ** -15, name


def test_large_logits_and_entries_taken_out():
    """Logits up to a thousand; entries with a bias of minus infinity; a row whose target is such an entry."""
    for dtype in ("bf16", "f32"):
        c = Case(40, 64, 700, dtype, bias=True, size=200.0, lost=0.0)
        c.check_forward()
        c = Case(40, 64, 700, dtype, bias=True, lost=0.0)
        c.bias[::3] = float("-inf")
        c.t[:] = (c.t // 3 * 3 + 1) % 699
        c.t[5] = 3
        loss, log_sum = c.forward()
        wl, ws, _, _ = c.exact()
        assert torch.isinf(loss[5]) and loss[5] > 0
        rest = torch.arange(40, device="cuda") != 5
        assert bool(((loss - wl).abs()[rest] < 1e-4).all()) and bool(((log_sum - ws).abs() < 1e-4).all())
        got = c.backward(dtype, dtype)
        dz = co.slopes(c.exact()[2], c.log_sum.double(), c.t, c.dloss.double())
        near(got["dbias"][0], dz.sum(0), torch.full((700,), 1e-4, dtype=torch.float64, device="cuda"), "dbias")
        assert bool(torch.isfinite(got["dw"][0]).all()) and bool(torch.isfinite(got["dx"][0]).all())
        c.bias[:] = float("-inf")
        loss, log_sum = c.forward()
        assert bool(loss.isnan().all()) and bool((log_sum == float("-inf")).all())


def test_rows_keep_to_themselves():
    """Undefined and infinite features, and what lies between the rows."""
    for dtype in ("bf16", "f32"):
        for M, V in ((50, 900), (300, 3000)):
            c = Case(M, 72, V, dtype, (3, 1), lost=0.0)
            keep = c.X.view.clone()
            c.X.buf.fill_(float("nan"))
            c.X.view.copy_(keep)
            whole = c.exact()
            c.X.view[3, 10] = float("nan")
            c.X.view[7, 11] = float("inf")
            loss, log_sum = c.forward()
            bad = torch.zeros(M, dtype=torch.bool, device="cuda")
            bad[3] = bad[7] = True
            assert bool(loss[bad].isnan().all()) and bool(log_sum[3].isnan())
            assert bool(((loss - whole[0]).abs()[~bad] < 2e-4).all()) and bool(((log_sum - whole[1]).abs()[~bad] < 2e-4).all())
            c.t[3] = c.t[7] = -1                       # (such a row's dx is then that of no target)
            c.X.view.copy_(keep)
            got = c.backward(dtype, dtype)
            assert bool((got["dx"][0][bad] == 0).all())


def test_against_differences():
    """The gradients of a float loss as differences of losses in 64 bits."""
    c = Case(6, 10, 23, "f32", bias=True)
    got = c.backward("f32", "f32")
    x, w, b = c.X.view.double(), c.w.double(), c.bias.double()
    d = torch.where((c.t >= 0) & (c.t < 23), c.dloss.double(), 0.0)
    total = lambda: float((d * co.forward(x, w, b, c.t)[0]).sum())
    for name, p in (("dx", x), ("dw", w), ("dbias", b)):
        flat, want = p.view(-1), got[name][0].reshape(-1)
        for i in range(0, flat.numel(), 7):
            step, keep = 1e-5, float(flat[i])
            flat[i] = keep + step
            up = total()
            flat[i] = keep - step
            down = total()
            flat[i] = keep
            assert abs((up - down) / (2 * step) - float(want[i])) < 1e-5, (name, i)


def test_whole_images_as_rows():
    """Channels-last images: every position is a row."""
    u, ig = _u(), _u().ig
    N, C, H, W, V = 2, 24, 5, 3, 50
    x = torch.randn(N, H, W, C, device="cuda")
    xd = ig.TensorDescriptor().set(ig.IGC_DATA_FLOAT, N, C, H, W, (H * W * C, 1, W * C, C))
    w, t = torch.randn(V, C, device="cuda"), torch.randint(0, V, (N * H * W,), device="cuda", dtype=torch.int32)
    wd, h = u.filter_desc("f32", V, C), u.handle()
    size = ig.get_linear_cross_entropy_forward_workspace_size(h, xd, wd)
    ws, loss = u.Workspace(size), torch.empty(N * H * W, device="cuda")
    ig.check(ig.linear_cross_entropy_forward(h, xd, x.data_ptr(), wd, w.data_ptr(), 0, t.data_ptr(), ws.buf.data_ptr(), size, loss.data_ptr(), 0))
    assert float((loss - co.forward(x.view(-1, C).double(), w.double(), None, t)[0]).abs().max()) < 1e-4


@pytest.mark.parametrize("M", [5, 200])
def test_in_a_graph_and_on_another_stream(M):
    """Loss and gradients captured, replayed over changed inputs with eager calls between, bit for bit those of the eager calls."""
    u, ig = _u(), _u().ig
    c = Case(M, 128, 1000, "bf16", bias=True)
    sizes = [ig.get_linear_cross_entropy_forward_workspace_size(c.h, c.X.desc, c.wd), ig.get_linear_cross_entropy_backward_workspace_size(c.h, c.X.desc, c.wd, c.X.desc, c.wd)]

    def outputs():
        return [torch.zeros(M, device="cuda"), torch.zeros(M, device="cuda"), torch.zeros(M, 128, dtype=torch.bfloat16, device="cuda"),
                torch.zeros(1000, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(1000, device="cuda"), torch.empty(max(sizes), dtype=torch.uint8, device="cuda")]

    def call(o):
        h = ig.Handle()
        h.set_stream(torch.cuda.current_stream().cuda_stream)
        loss, log_sum, dx, dw, db, ws = o
        ig.check(ig.linear_cross_entropy_forward(h, c.X.desc, c.X.ptr, c.wd, c.w.data_ptr(), c.bias.data_ptr(), c.t.data_ptr(), ws.data_ptr(), sizes[0], loss.data_ptr(),
                                                 log_sum.data_ptr()))
        dxd = ig.TensorDescriptor().set(ig.IGC_DATA_BFLOAT16, M, 128, 1, 1, (128, 1, 1, 1))
        ig.check(ig.linear_cross_entropy_backward(h, 0.5, c.X.desc, c.X.ptr, c.wd, c.w.data_ptr(), c.bias.data_ptr(), c.t.data_ptr(), log_sum.data_ptr(), 0, ws.data_ptr(), sizes[1],
                                                  0.0, dxd, dx.data_ptr(), 0.0, c.wd, dw.data_ptr(), db.data_ptr()))

    a, b = outputs(), outputs()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        call(a)
    for i in range(4):
        c.X.view.copy_(torch.randn(M, 128, device="cuda"))
        c.t.copy_(torch.randint(-1, 1000, (M,), device="cuda"))
        graph.replay()
        call(b)
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(a[:5], b[:5])), i
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    d = outputs()
    torch.cuda.synchronize()
    with torch.cuda.stream(other):
        call(d)
    other.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(d[:5], b[:5]))


def test_vocabulary_beyond_32_bits():
    """w of 2.2e9 elements, 4.4 GB: its last entries lie behind 2^32 bytes, those of dw too."""
    for M in (3, 40):
        print("far vocabulary", M, flush=True)
        case = Case(M, 8200, 270001, "bf16", seed=31)
        case.t[0] = case.V - 1
        case.check_forward()
        entries = torch.cat([torch.arange(300), torch.arange(262000, 262300), torch.arange(case.V - 300, case.V)]).cuda()
        case.check_backward(pieces=8, entries=entries)
        del case
        torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_beyond_32_bits(dtype):
    """Rows of x and dx 2^25 elements apart."""
    u, ig = _u(), _u().ig
    for M in (70, 130):
        print("far rows", dtype, M, flush=True)
        case = Case(M, 72, 500, dtype)
        apart = 2 ** 25

        class Far(u.Rows):
            def __init__(self, shape, dtype, *layout):
                self.buf = torch.empty(M * apart, dtype=u.DTYPES[dtype], device="cuda").view(M, apart)
                self.buf[:, 72:80] = u.GUARD
                self.view = self.buf[:, :72]
                self.desc = ig.TensorDescriptor().set({"f32": ig.IGC_DATA_FLOAT, "bf16": ig.IGC_DATA_BFLOAT16}[dtype], M, 72, 1, 1, (apart, 1, 1, 1))

            def numpy(self):
                assert bool((self.buf[:, 72:80] == u.GUARD).all())
                return self.view.double().cpu().numpy()

        far = Far(None, dtype)
        far.view.copy_(case.X.view)
        case.X = far
        case.check_forward()
        keep, u.Rows = u.Rows, Far
        try:
            case.check_backward(dx=dtype, dw=dtype)
        finally:
            u.Rows = keep
        del case, far
        torch.cuda.empty_cache()


@pytest.mark.parametrize("types", [("bf16", "bf16", "bf16"), ("bf16", "f32", "f32")], ids="-".join)
def test_targets_that_repeat(types):
    """All rows of one target, of two, of neighbours; across pieces, in ranges of the reduction, in copies."""
    for M, C, V, layout in ((33, 64, 100, (0, 0)), (600, 70, 50, (1, 1)), (1500, 2100, 300, (8, 8)), (3000, 40, 130, (0, 0)), (2000, 64, 140001, (0, 0))):
        for how in ("one", "two", "neighbours", "last"):
            print("targets that repeat", types, M, C, V, layout, how, flush=True)
            case = Case(M, C, V, types[0], layout, bias=True, lost=0.0)
            m = torch.arange(M, device="cuda")
            case.t = {"one": 0 * m + V // 2, "two": m % 2 * (V - 1), "neighbours": m % V, "last": V - 1 - m // 700}[how].to(torch.int32)
            case.t[M // 3] = -100
            case.check_backward(types[1], types[2], alpha=1.0 / M, beta=0.5 if how == "two" else 0.0, pbeta=0.5 if how == "two" else 0.0, pieces=4)
            del case
    torch.cuda.empty_cache()
