"""Low-rank adapters and their gradient, the norm of many gradients with
clipping, and the verification of drafted tokens (paper_1903_05133_amd/operators.py)
on the GPU against plain implementations in 64 bits.

Tolerances count roundings, u = 2^-24: a float32 sum of n terms in any order is
off by at most n u of the sum of their magnitudes, each product and each result
by half a step of its type."""

import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = [torch.float32, torch.bfloat16, torch.float16]
INF, NAN = math.inf, math.nan


@pytest.fixture(scope="module")
def ops(gpu_lib):
    from paper_1903_05133_amd import operators
    return operators


@pytest.fixture(autouse=True)
def float32_by_default():
    was = torch.get_default_dtype()
    torch.set_default_dtype(torch.float32)
    yield
    torch.set_default_dtype(was)


def say(*a):
    print("[gpu case]", *a, flush=True)


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def half_step(t):
    return torch.finfo(t).eps / 2


def least(t):
    """Half the step of the subnormals."""
    return torch.finfo(t).smallest_normal * torch.finfo(t).eps / 2


# ------------------------------------------------------------------ adapters
class Adapters:
    """Inputs on the CPU, and the definition in 64 bits with its error bounds."""

    def __init__(self, rows, n, rank, k, cols, dtype, seed, ids=None, scaled=True):
        g = gen(seed)
        self.n, self.rank, self.k, self.cols = n, rank, k, cols
        self.x = (torch.randn(rows, k, generator=g) * torch.exp(torch.randn(rows, 1, generator=g))).to(dtype)
        self.down = (torch.randn(n, rank, k, generator=g) / math.sqrt(k)).to(dtype)
        self.up = torch.randn(n, rank, cols, generator=g).to(dtype)
        self.scales = (torch.rand(n, generator=g) * 4 - 2) if scaled else None
        self.ids = torch.randint(-1, n, (rows,), generator=g) if ids is None else ids
        self.dy = torch.randn(rows, cols, generator=g).to(dtype)
        self.base = torch.randn(rows, cols, generator=g)
        self.xbase = torch.randn(rows, k, generator=g)

    def scale(self, a):
        return 1.0 if self.scales is None else float(self.scales[a])

    def rows_of(self, a):
        return (self.ids == a).nonzero()[:, 0]

    def forward(self, base):
        """(y, its bound without the last rounding, h, its bound)"""
        y = torch.zeros(len(self.x), self.cols, dtype=torch.float64) if base is None else base.double().clone()
        h, th = (torch.zeros(len(self.x), self.rank, dtype=torch.float64) for _ in range(2))
        tol = torch.zeros_like(y)
        for a in range(self.n):
            r = self.rows_of(a)
            x, d, u, s = self.x[r].double(), self.down[a].double(), self.up[a].double(), self.scale(a)
            h[r] = x @ d.t()
            th[r] = (self.k + 8) * U * (x.abs() @ d.abs().t())
            y[r] += s * (h[r] @ u)
            tol[r] = abs(s) * ((th[r] + (self.rank + 8) * U * h[r].abs()) @ u.abs()) + 2 * U * y[r].abs()
        return y, tol, h, th

    def backward(self, base, h=None):
        """(dx, bound), (ddown, bound), (dup, bound)"""
        dx = torch.zeros(len(self.x), self.k, dtype=torch.float64) if base is None else base.double().clone()
        tx = torch.zeros_like(dx)
        dd, td = (torch.zeros(self.n, self.rank, self.k, dtype=torch.float64) for _ in range(2))
        du, tu = (torch.zeros(self.n, self.rank, self.cols, dtype=torch.float64) for _ in range(2))
        for a in range(self.n):
            r = self.rows_of(a)
            m = len(r)
            x, dy, d, u, s = (*(t.double() for t in (self.x[r], self.dy[r], self.down[a], self.up[a])), self.scale(a))
            dh = dy @ u.t()
            tdh = (self.cols + 8) * U * (dy.abs() @ u.abs().t())
            hh = x @ d.t() if h is None else h[r].double()
            th = (self.k + 8) * U * (x.abs() @ d.abs().t()) if h is None else torch.zeros_like(hh)
            dx[r] += s * (dh @ d)
            tx[r] = abs(s) * ((tdh + (self.rank + 8) * U * dh.abs()) @ d.abs()) + 2 * U * dx[r].abs()
            dd[a], td[a] = s * (dh.t() @ x), abs(s) * ((tdh + (m + 8) * U * dh.abs()).t() @ x.abs())
            du[a], tu[a] = s * (hh.t() @ dy), abs(s) * ((th + (m + 8) * U * hh.abs()).t() @ dy.abs())
        return (dx, tx), (dd, td), (du, tu)


def near(got, want, tol, what):
    """Within the bound and the last rounding, everywhere."""
    d = half_step(got.dtype)
    limit = tol * (1 + 2 * d) + d * want.abs() * (1 + d) + least(got.dtype) + 1e-40
    off = (got.cpu().double() - want).abs()
    assert torch.isfinite(want).all() and not torch.isnan(off).any(), what
    assert torch.all(off <= limit), (what, float((off / limit).max()))


def on_gpu(*t):
    return [None if x is None else x.cuda() for x in t]


SHAPES = [(1, 1, 1, 1, 1), (1, 4, 16, 4096, 4096), (2, 2, 8, 33, 7), (5, 3, 4, 16, 129), (17, 2, 17, 100, 515), (64, 40, 16, 257, 130),
          (64, 1, 128, 300, 513), (65, 3, 5, 64, 1000), (130, 200, 9, 70, 60), (257, 2, 33, 1001, 37), (777, 5, 24, 1000, 300),
          (1025, 1, 64, 300, 260), (2500, 3, 65, 130, 200), (4100, 7, 127, 65, 90)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n,rank,k,cols", SHAPES)
def test_adapter_product(rows, n, rank, k, cols, dtype, ops):
    say("adapters", rows, n, rank, k, cols, dtype)
    c = Adapters(rows, n, rank, k, cols, dtype, rows + rank + k, scaled=rank % 2 == 0)
    x, ids, down, up, scales = on_gpu(c.x, c.ids, c.down, c.up, c.scales)
    for out in {dtype, torch.float32}:
        base = c.base.to(out)
        y, tol, h, th = c.forward(base)
        got, hidden = ops.adapter_product(x, ids, down, up, scales, base=base.cuda(), hidden=True)
        assert got.dtype == out and got.shape == (rows, cols) and hidden.dtype == torch.float32
        near(got, y, tol, "y")
        near(hidden, h, th, "hidden")
        assert torch.equal(got.cpu()[c.ids < 0], base[c.ids < 0])
        # the same bits from ids of 32 bits, in place, and in rows of wider buffers at odd places
        wide, xwide = torch.full((rows, cols + 5), 3.0, dtype=out, device="cuda"), torch.full((rows, k + 3), NAN, dtype=dtype, device="cuda")
        xwide[:, 1:k + 1] = x
        wide[:, 3:cols + 3] = base.cuda()
        view = wide[:, 3:cols + 3]
        assert ops.adapter_product(xwide[:, 1:k + 1], ids.int(), down, up, scales, base=view, out=view).data_ptr() == view.data_ptr()
        assert torch.equal(view, got) and torch.all(wide[:, :3] == 3.0) and torch.all(wide[:, cols + 3:] == 3.0)
    y, tol, _, _ = c.forward(None)
    got = ops.adapter_product(x, ids, down, up, scales)
    assert got.dtype == dtype
    near(got, y, tol, "without a base")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n,rank,k,cols", SHAPES)
def test_adapter_product_grad(rows, n, rank, k, cols, dtype, ops):
    say("adapters grad", rows, n, rank, k, cols, dtype)
    c = Adapters(rows, n, rank, k, cols, dtype, rows + rank + k + 1, scaled=rank % 2 == 1)
    dy, x, ids, down, up, scales = on_gpu(c.dy, c.x, c.ids, c.down, c.up, c.scales)
    base = c.xbase.to(dtype)
    want = c.backward(base)
    r = ops.adapter_product_grad(dy, x, ids, down, up, scales, base=base.cuda())
    assert r.dx.dtype == dtype and r.down.dtype == r.up.dtype == torch.float32
    for got, (w, tol), what in zip(r, want, ("dx", "ddown", "dup")):
        near(got, w, tol, what)
    for a in range(n):
        if not (c.ids == a).any():
            assert not r.down[a].any() and not r.up[a].any()
    # hidden values of the forward, 16-bit gradients, dx in place, each of the results alone
    hidden = ops.adapter_product(x, ids, down, up, scales, hidden=True)[1]
    here = base.cuda()
    t = ops.adapter_product_grad(dy, x, ids.int(), down, up, scales, hidden=hidden, base=here, out=here, grad_dtype=torch.bfloat16)
    assert t.dx.data_ptr() == here.data_ptr() and torch.equal(here, r.dx) and torch.equal(t.down, r.down.bfloat16())
    (w, tol), = c.backward(base, hidden.cpu())[2:]
    near(t.up, w, tol, "dup of hidden values")
    only = ops.adapter_product_grad(dy, x, ids, down, up, scales, weights=False)
    near(only.dx, *c.backward(None)[0], "dx alone")
    assert only.down is None and only.up is None
    only = ops.adapter_product_grad(dy, x, ids, down, up, scales, dx=False)
    assert only.dx is None and torch.equal(only.down, r.down) and torch.equal(only.up, r.up)


def test_adapter_grad_formula_against_differences():
    """The formulas of Adapters.backward against central differences of Adapters.forward in 64 bits."""
    c = Adapters(9, 2, 3, 5, 4, torch.float32, 3)
    loss = lambda: float((c.forward(None)[0] * c.dy.double()).sum())  # noqa: E731
    (dx, _), (dd, _), (du, _) = c.backward(None)
    for name, grad in (("x", dx), ("down", dd), ("up", du)):
        t = getattr(c, name).double()
        setattr(c, name, t)
        for i in range(t.numel()):
            at = t.view(-1)[i].item()
            t.view(-1)[i] = at + 1e-5
            up = loss()
            t.view(-1)[i] = at - 1e-5
            low = loss()
            t.view(-1)[i] = at
            # second differences vanish (the loss is bilinear): rounding of two sums of 36 terms around 10
            assert abs((up - low) / 2e-5 - grad.view(-1)[i].item()) <= 1e-7


@pytest.mark.parametrize("rows", [7, 64, 200])
def test_adapter_rows_apart(rows, ops):
    """Rows without an adapter keep base whatever they hold; ids past the end give NaN and add nothing; a NaN stays in
    its row and its adapter."""
    c = Adapters(rows, 3, 6, 40, 50, torch.bfloat16, 5, ids=torch.arange(rows) % 5 - 1)  # -1, 0, 1, 2, 3
    none, wrong = c.ids == -1, c.ids == 3
    c.x[none] = NAN
    c.dy[none] = INF
    c.x[wrong] = INF
    bad = int((c.ids == 1).nonzero()[0])
    c.x[bad, 7] = NAN
    base = c.base.bfloat16()
    x, ids, down, up, scales, dy = on_gpu(c.x, c.ids, c.down, c.up, c.scales, c.dy)
    y, h = (t.cpu() for t in ops.adapter_product(x, ids, down, up, scales, base=base.cuda(), hidden=True))
    nan = torch.isnan(y)
    assert torch.equal(y[none], base[none]) and not h[none].any()
    assert nan[wrong].all() and torch.isnan(h[wrong]).all() and nan[bad].all()
    others = ~none & ~wrong
    others[bad] = False
    assert not nan[others].any()
    r = ops.adapter_product_grad(dy, x, ids, down, up, scales, base=c.xbase.bfloat16().cuda())
    dx = r.dx.cpu()
    assert torch.equal(dx[none], c.xbase.bfloat16()[none]) and torch.isnan(dx[wrong]).all() and torch.isfinite(dx[others]).all()
    assert torch.isfinite(r.down[[0, 2]]).all() and torch.isfinite(r.up[[0, 2]]).all()
    assert torch.isnan(r.down[1, :, 7]).all() and torch.isnan(r.up[1]).all()
    clean = Adapters(rows, 3, 6, 40, 50, torch.bfloat16, 5, ids=torch.where(wrong, -1, c.ids))
    want = clean.backward(None)
    for a in (0, 2):
        near(r.down[a], want[1][0][a], want[1][1][a], "ddown")
        near(r.up[a], want[2][0][a], want[2][1][a], "dup")


def test_adapters_without_rows_and_refusals(ops):
    c = Adapters(4, 2, 3, 8, 6, torch.float32, 1)
    x, ids, down, up, dy = on_gpu(c.x, c.ids, c.down, c.up, c.dy)
    assert ops.adapter_product(x[:0], ids[:0], down, up).shape == (0, 6)
    r = ops.adapter_product_grad(dy[:0], x[:0], ids[:0], down, up)
    assert r.dx.shape == (0, 8) and not r.down.any() and not r.up.any()
    none = torch.full_like(ids, -1)
    assert not ops.adapter_product(x, none, down, up).any()
    r = ops.adapter_product_grad(dy, x, none, down, up)
    assert not r.dx.any() and not r.down.any() and not r.up.any()
    # more dimensions
    y = ops.adapter_product(x.view(2, 2, 8), ids.view(2, 2), down, up, hidden=True)
    assert y[0].shape == (2, 2, 6) and y[1].shape == (2, 2, 3)
    assert torch.equal(y[0].view(4, 6), ops.adapter_product(x, ids, down, up))
    buf = torch.zeros(4, 20, device="cuda")
    for bad in (lambda: ops.adapter_product(x.half(), ids, down, up), lambda: ops.adapter_product(x[:, :7], ids, down, up),
                lambda: ops.adapter_product(x, ids[:3], down, up), lambda: ops.adapter_product(x, ids.float(), down, up),
                lambda: ops.adapter_product(x, ids, down[:1], up), lambda: ops.adapter_product(x, ids, down, up.transpose(1, 2)),
                lambda: ops.adapter_product(x, ids, down, up, scales=torch.ones(3, device="cuda")),
                lambda: ops.adapter_product(x, ids, down, up, base=x), lambda: ops.adapter_product(x, ids, down, up, dtype=torch.float64),
                lambda: ops.adapter_product(x, ids, down.cpu(), up.cpu()), lambda: ops.adapter_product(x.cpu(), ids, down, up),
                lambda: ops.adapter_product_grad(dy, x, ids, down, up, dx=False, weights=False),
                lambda: ops.adapter_product_grad(dy, x, ids, down, up, hidden=torch.zeros(4, 2, device="cuda")),
                lambda: ops.adapter_product_grad(dy, x, ids, down, up, dx=False, base=x),
                lambda: ops.adapter_product_grad(dy.half(), x, ids, down, up),
                lambda: ops.adapter_product(x, ids, torch.zeros(1, 129, 8, device="cuda"), torch.zeros(1, 129, 6, device="cuda"))):
        with pytest.raises(ValueError):
            bad()
    buf[:, :8] = x
    for bad in (lambda: ops.adapter_product(buf[:, :8], ids, down, up, out=buf[:, 4:10]),
                lambda: ops.adapter_product(x, ids, down, up, base=buf[:, 1:7], out=buf[:, 2:8]),
                lambda: ops.adapter_product_grad(dy, buf[:, :8], ids, down, up, out=buf[:, 1:9])):
        with pytest.raises(ops.native.HierAvgError, match="overlap"):
            bad()
    # beside each other in one buffer: not refused
    ops.adapter_product(buf[:, :8], ids, down, up, out=buf[:, 8:14])
    assert torch.equal(buf[:, 8:14], ops.adapter_product(x, ids, down, up))


def test_many_adapters(ops):
    """As many adapters as there may be, most without rows, and rows of the last."""
    n = 8192
    ids = torch.tensor([n - 1, 0, n - 1, 5000] * 40)
    c = Adapters(160, n, 2, 3, 4, torch.float32, 2, ids=ids)
    x, i, down, up, scales, dy = on_gpu(c.x, c.ids, c.down, c.up, c.scales, c.dy)
    used = [0, 5000, n - 1]
    y = ops.adapter_product(x, i, down, up, scales).cpu().double()
    r = ops.adapter_product_grad(dy, x, i, down, up, scales)
    for a in used:
        rows = c.rows_of(a)
        w = c.scale(a) * (c.x[rows].double() @ c.down[a].double().t()) @ c.up[a].double()
        assert (y[rows] - w).norm() <= 1e-6 * w.norm()  # 5 roundings of sums of 3 and 2 terms
        w = c.scale(a) * (c.dy[rows].double() @ c.up[a].double().t()).t() @ c.x[rows].double()
        assert (r.down[a].cpu().double() - w).norm() <= 1e-5 * w.norm()  # sums of 4 and 80 terms
    rest = torch.ones(n, dtype=torch.bool)
    rest[used] = False
    assert not r.down.cpu()[rest].any() and not r.up.cpu()[rest].any()


def test_adapters_offsets_past_32_bits(ops):
    """Rows more than 2^31 elements apart, and adapters past 2^32 elements."""
    c = Adapters(3, 2, 4, 40, 24, torch.bfloat16, 9, ids=torch.tensor([1, 0, 1]))
    x, ids, down, up, scales, dy = on_gpu(c.x, c.ids, c.down, c.up, c.scales, c.dy)
    stride = (1 << 31) + 8
    buf = torch.zeros(2 * stride + 64, dtype=torch.bfloat16, device="cuda")
    far = buf.as_strided((3, 40), (stride, 1))
    far.copy_(x)
    out = buf[40:].as_strided((3, 24), (stride, 1))
    want = ops.adapter_product(x, ids, down, up, scales)
    ops.adapter_product(far, ids, down, up, scales, out=out)
    assert torch.equal(out, want)
    r = ops.adapter_product_grad(dy, x, ids, down, up, scales)
    t = ops.adapter_product_grad(out.copy_(dy), far, ids, down, up, scales)
    assert torch.equal(t.dx, r.dx) and torch.equal(t.down, r.down) and torch.equal(t.up, r.up)
    del buf, far, out
    n, rank, k = 8192, 128, 4100
    big = torch.zeros(n, rank, k, dtype=torch.bfloat16, device="cuda")
    big[-1, :4, :40] = down[1]
    small = torch.zeros(n, rank, 1, dtype=torch.bfloat16, device="cuda")
    small[-1, :4, 0] = 1
    xw = torch.zeros(3, k, dtype=torch.bfloat16, device="cuda")
    xw[:, :40] = x
    y = ops.adapter_product(xw, torch.full((3,), n - 1, device="cuda"), big, small, dtype=torch.float32)
    w = (c.x.double() @ c.down[1].double().t()).sum(1)
    bound = (c.x.double().abs() @ c.down[1].double().abs().t()).sum(1) * (44 + 8) * U
    assert torch.all((y.cpu().double()[:, 0] - w).abs() <= bound)


# ------------------------------------------------------------------ norms and clipping
def plain_norms(tensors, most):
    sums = [0.0 if t is None else float(t.double().square().sum()) for t in tensors]
    norm = math.sqrt(math.fsum(sums))
    return [math.sqrt(s) for s in sums], norm, 1.0 if norm <= most else most / norm


def close(got, want, roundings=3):
    # eight squares at a time in float32: of their sum off by 4 u at most (three additions one after the other and one
    # that joins), of its root by 2 u; the rest of the sum in 64 bits, 1e-9 at most here; the result's rounding
    return abs(got - want) <= (roundings * U + 1e-9) * abs(want) + 1e-45


SETS = [[1], [5, 0, 3], [300, 300000, 37], [16384, 16385, 16383, 1], [7] * 300, [2_000_003, 5, 1 << 20], [9_000_001],
        [70_000_001, 3]]


@pytest.mark.parametrize("dtype", TYPES + ["mixed"])
@pytest.mark.parametrize("sizes", SETS, ids=lambda s: f"{len(s)}x{max(s)}")
def test_grad_norm_and_clipping(sizes, dtype, ops):
    say("norm", sizes[:5], dtype)
    g = torch.Generator(device="cuda").manual_seed(len(sizes) + max(sizes))
    kinds = [TYPES[i % 3] if dtype == "mixed" else dtype for i in range(len(sizes))]
    # at odd places of a buffer
    made = [torch.randn(n + 1, device="cuda", generator=g).to(t)[1:] for n, t in zip(sizes, kinds)]
    norms, norm, _ = plain_norms(made, INF)
    for most in (None, 0.5 * norm, 2.0 * norm, 0.0):
        want = 1.0 if most is None or norm <= most else most / norm
        r = ops.grad_norm(made, most)
        assert r.norm.shape == () and r.norms.shape == (len(sizes),)
        assert close(r.norm.item(), norm) and close(r.factor.item(), want)
        assert all(close(a, b) for a, b in zip(r.norms.tolist(), norms))
        again = ops.grad_norm(made, most)
        assert all(torch.equal(a, b) for a, b in zip(r, again))
        if most is None:
            continue
        out = [torch.full_like(t, 7.0) for t in made]
        kept = [t.clone() for t in made]
        c = ops.clip_grads(made, most, out=out)
        assert all(torch.equal(a, b) for a, b in zip(c, r)) and all(torch.equal(a, b) for a, b in zip(made, kept))
        for t, o in zip(made, out):
            assert torch.equal(o, (t.float() * r.factor).to(t.dtype))
        ops.clip_grads(kept, most)
        assert all(torch.equal(a, b) for a, b in zip(kept, out))


def test_grad_norm_of_extremes(ops):
    """Squares past float32's range on both sides, NaN, infinities, absent and empty gradients."""
    for v in (3e38, 1e-38, 1e-45, 2.0 ** -140):
        t = torch.full((1000,), v, device="cuda")
        want = math.sqrt(1000) * float(t[0].double())
        assert close(ops.grad_norm([t]).norm.item(), want) if want < 3.4e38 else ops.grad_norm([t]).norm.item() == INF
    big = torch.full((1000,), 3e38, device="cuda")
    r = ops.grad_norm([big, None, big[:0]], 1.0)
    assert r.norm.item() == INF and close(r.factor.item(), 1.0 / (math.sqrt(1000) * float(big[0].double())))
    assert r.norms.tolist()[1:] == [0.0, 0.0]
    for bad, norm, factor in ((NAN, NAN, NAN), (INF, INF, 0.0), (-INF, INF, 0.0)):
        t = torch.ones(70000, device="cuda")
        t[66000] = bad
        r = ops.grad_norm([t, torch.ones(4, device="cuda")], 1.0)
        got = [r.norm.item(), r.factor.item(), r.norms[0].item(), r.norms[1].item()]
        assert all(a == b or (math.isnan(a) and math.isnan(b)) for a, b in zip(got, (norm, factor, norm, 2.0))), got
    zero = ops.grad_norm([torch.zeros(5, device="cuda")], 0.0)
    assert zero.norm.item() == 0.0 and zero.factor.item() == 1.0


def test_clipping_refusals(ops):
    a, b = torch.ones(10, device="cuda"), torch.ones(10, device="cuda")
    for bad in (lambda: ops.grad_norm([]), lambda: ops.grad_norm([None]), lambda: ops.grad_norm([a.double()]),
                lambda: ops.grad_norm([a[::2]]), lambda: ops.grad_norm([a, b.cpu()]), lambda: ops.grad_norm([a], -1.0),
                lambda: ops.grad_norm([a], NAN), lambda: ops.clip_grads([a], 1.0, out=[]), lambda: ops.clip_grads([a], 1.0, out=[b.half()]),
                lambda: ops.clip_grads([a], 1.0, out=[None]), lambda: ops.clip_grads([a], 1.0, out=[b[:9]])):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: ops.clip_grads([a[:9]], 1.0, out=[a[1:]]), lambda: ops.clip_grads([a, a], 1.0),
                lambda: ops.clip_grads([a, b], 1.0, out=[b, a]), lambda: ops.clip_grads([a, b], 1.0, out=[b, b])):
        with pytest.raises(ops.native.HierAvgError, match="overlap"):
            bad()
    assert torch.all(a == 1) and torch.all(b == 1)
    version = a._version
    ops.clip_grads([a, None], 1.0)
    assert a._version > version and close(ops.grad_norm([a]).norm.item(), 1.0, 6)


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_takes_the_factor(bits, ops):
    """A step on gradients times the factor is the step on the products; a factor of 1 is the plain step."""
    def made():
        g = gen(4)
        p = [torch.randn(n, generator=g).cuda() for n in (300, 5000, 1)]
        return p, ops.AdamW(p, state_bits=bits, lr=1e-2, seed=1)
    (p, a), (q, b), (o, c), (w, d) = made(), made(), made(), made()
    for i in range(3):
        grads = [torch.randn(t.shape, generator=gen(10 * i + k)).cuda() for k, t in enumerate(p)]
        r = ops.grad_norm(grads, 0.25)
        assert 0.0 < r.factor.item() < 0.1
        a.step(grads, factor=r.factor)
        b.step([t * r.factor for t in grads])
        c.step(grads, factor=torch.ones(1, device="cuda"))
        d.step(grads)
    for x, y in (*zip(p, q), *zip(o, w)):
        assert torch.equal(x, y)
    assert torch.equal(a.m.view(torch.uint8), b.m.view(torch.uint8)) and torch.equal(a.v, b.v)
    assert torch.equal(c.m.view(torch.uint8), d.m.view(torch.uint8)) and torch.equal(c.v, d.v)
    for bad in (torch.ones(2, device="cuda"), torch.ones(1), torch.ones(1, device="cuda").half()):
        with pytest.raises(ValueError):
            a.step(grads, factor=bad)


# ------------------------------------------------------------------ verification of drafts
def distribution(row, t):
    """In 64 bits; None without one."""
    row = row.double()
    most = row.max()
    if torch.isnan(row).any() or most == INF or most == -INF:
        return None
    if t > 0 and t < INF:
        e = ((row - most) / t).exp()
        return e / e.sum()
    p = torch.zeros_like(row)
    p[int((row == most).nonzero()[0])] = 1.0
    return p


def plain_verify(logits, drafts, uniforms, given, lengths, temperature):
    """The definition, and which sequences 64 bits decide: no two sides of a
    comparison, and no running sum and its mark, within 1e-12 of each other (sums of up
    to 2^18 terms are off by 2^18 2^-53 = 3e-11 of a term's mean at most, 1e-16 of
    the whole for each), and a difference p - q of 1e-9 at least (each of its terms is off by 2^-52)."""
    tokens, accepted, logps, clear = [], [], [], []
    for b in range(logits.shape[0]):
        n = logits.shape[1] - 1
        n = n if lengths is None else min(max(int(lengths[b]), 0), n)
        t = 1.0 if temperature is None else float(temperature[b])
        warm = t > 0 and t < INF
        out, lp, i, w, edge = [], [], 0, None, 1.0
        while True:
            p = distribution(logits[b, i], t)
            if i == n:
                w = p
                break
            j = int(drafts[b, i])
            q = None
            if warm and given is not None:
                q = distribution(given[b, i], t)
            else:
                q = torch.zeros(logits.shape[2], dtype=torch.float64)
                if 0 <= j < len(q):
                    q[j] = 1.0
            inside = 0 <= j < logits.shape[2]
            if p is not None and q is not None and inside:
                lhs, rhs = float(uniforms[b, i]) * float(q[j]), float(p[j])
                if lhs > 0 and rhs > 0:
                    edge = min(edge, abs(lhs / rhs - 1))
                if lhs < rhs:
                    out.append(j)
                    lp.append(math.log(rhs))
                    i += 1
                    continue
            if p is None or (q is None):
                w = None
            else:
                w = (p - q).clamp(min=0.0)
                edge = edge if float(w.sum()) > 1e-9 else 0.0
                w = w if float(w.sum()) > 0 else p
            break
        accepted.append(i)
        if w is None:
            out.append(-1)
            lp.append(0.0)
        else:
            c = w.cumsum(0)
            u = float(uniforms[b, -1]) * float(c[-1])
            j = int((c > u).nonzero()[0]) if u < c[-1] else int((w > 0).nonzero()[-1])
            if warm:
                edge = min(edge, float((c / c[-1] - float(uniforms[b, -1])).abs().min()) if len(c) > 1 else 1.0)
            out.append(j)
            lp.append(math.log(float(p[j])))
        out += [-1] * (logits.shape[1] - len(out))
        lp += [0.0] * (logits.shape[1] - len(lp))
        tokens.append(out)
        logps.append(lp)
        clear.append(edge > 1e-12)
    return tokens, accepted, logps, clear


def check_verify(r, want, classes):
    tokens, accepted, logps, clear = want
    assert all(clear), "the case has no reference"
    assert r.accepted.tolist() == accepted and r.tokens.tolist() == tokens, (r.accepted.tolist(), accepted)
    # log z: a float32 sum, off by (classes / 256 + 110) u at most, and the logarithm's and the result's roundings
    got = r.logp.cpu().double()
    lp = torch.tensor(logps, dtype=torch.float64)
    assert torch.all((got - lp).abs() <= (classes / 256 + 114) * U + 2 * U * lp.abs())


def verify_case(B, G, V, dtype, qtype, seed, pad=0, near_by=0.7):
    g = gen(seed)
    both = 4 * torch.randn(B, max(G, 1), V + pad, generator=g)
    x = 4 * torch.randn(B, G + 1, V + pad, generator=g)
    x[:, :G] = both[:, :G] + near_by * torch.randn(B, G, V + pad, generator=g)
    x, q = x.to(dtype)[:, :, :V], both.to(qtype)[:, :G, :V]
    t = torch.tensor([0.0, 0.7, 1.0, 1.5])[torch.randint(0, 4, (B,), generator=g)]
    noise = -torch.log(-torch.log(torch.rand(B, G, V, generator=g).clamp(1e-12, 1 - 1e-7)))
    drafts = (q.float() + t[:, None, None] * noise).argmax(2)
    return x, q, drafts, torch.rand(B, G + 1, generator=g), torch.randint(0, G + 1, (B,), generator=g, dtype=torch.int32), t


VERIFY = [(1, 0, 1, 0), (1, 1, 1, 0), (3, 2, 2, 1), (40, 5, 10, 0), (9, 1, 64, 0), (7, 3, 1000, 5), (2, 8, 2048, 0), (3, 4, 2049, 0), (5, 4, 4097, 3),
          (1, 4, 32000, 0), (6, 2, 50001, 7), (1, 64, 300, 0), (300, 2, 70, 0), (2, 2, 131072, 0), (1, 1, 140001, 0)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,G,V,pad", VERIFY)
def test_verify_drafts(B, G, V, pad, dtype, ops):
    say("verify", B, G, V, pad, dtype)
    qtype = TYPES[(TYPES.index(dtype) + (V % 2)) % 3]
    x, q, drafts, u, lengths, t = verify_case(B, G, V, dtype, qtype, B + G + V, pad)
    xg, qg, dg, ug, lg, tg = on_gpu(x, q, drafts, u, lengths, t)
    # views keep their wide rows
    if pad:
        xg = torch.full((B, G + 1, V + pad), NAN, dtype=dtype, device="cuda")
        xg[:, :, :V] = x.cuda()
        xg = xg[:, :, :V]
    for given in (q, None):
        for ln in (lengths, None):
            for temp in (t, None):
                r = ops.verify_drafts(xg, dg, ug, draft_logits=None if given is None else qg, lengths=None if ln is None else lg,
                                      temperature=None if temp is None else tg)
                check_verify(r, plain_verify(x, drafts, u, given, ln, temp), V)
                r2 = ops.verify_drafts(xg, dg.int(), ug, draft_logits=None if given is None else qg, lengths=None if ln is None else lg,
                                       temperature=None if temp is None else tg)
                assert all(torch.equal(a, b) for a, b in zip(r, r2))


def test_verify_all_accepted_and_draws(ops):
    """Drafts of the target's own distribution are all accepted; draws of the bonus row follow it at every uniform number."""
    V, B = 5000, 256
    x, _, _, _, _, _ = verify_case(1, 3, V, torch.float32, torch.float32, 3)
    xs = x.expand(B, 4, V).contiguous()
    drafts = torch.randint(0, V, (B, 3), generator=gen(1))
    u = torch.rand(B, 4, generator=gen(2))
    u[:, 3] = torch.arange(B) / B
    u[-1, 3] = 1 - 2.0 ** -24
    r = ops.verify_drafts(xs.cuda(), drafts.cuda(), u.cuda(), draft_logits=xs[:, :3].contiguous().cuda())
    assert r.accepted.tolist() == [3] * B and torch.equal(r.tokens[:, :3].cpu().long(), drafts)
    c = distribution(x[0, 3], 1.0).cumsum(0)
    for b in range(B):
        assert r.tokens[b, 3].item() == int((c > float(u[b, 3]) * float(c[-1])).nonzero()[0])


def test_verify_at_the_border(ops):
    """Uniform numbers next to p / q: float32 sums cannot settle these, sums in 64 bits do."""
    V = 20000
    x, q, drafts, u, _, _ = verify_case(1, 1, V, torch.float32, torch.float32, 8)
    p, d = distribution(x[0, 0], 1.0), distribution(q[0, 0], 1.0)
    ratio = p / d
    some = ((ratio > 0.2) & (ratio < 0.95)).nonzero()[:40, 0]
    edges = torch.stack([(ratio[some].float().view(torch.int32) + k).view(torch.float32) for k in (-2, -1, 0, 1, 2)], 1)
    B = edges.numel()
    uu = torch.full((B, 2), 0.4)
    uu[:, 0] = edges.reshape(-1)
    ids = some.repeat_interleave(5)[:, None]
    xs, qs = x.expand(B, 2, V).contiguous(), q.expand(B, 1, V).contiguous()
    r = ops.verify_drafts(xs.cuda(), ids.cuda(), uu.cuda(), draft_logits=qs.cuda())
    want = (uu[:, 0].double() * d[ids[:, 0]] < p[ids[:, 0]]).int()
    assert 0 < want.sum() < B and torch.equal(r.accepted.cpu(), want)


def test_verify_special_rows(ops):
    """Masked rows, rows without a distribution, drafts that are no class or impossible, temperatures that are none."""
    V = 3000
    x, q, _, _, _, _ = verify_case(12, 2, V, torch.float32, torch.float32, 5)
    drafts = torch.tensor([[3, 4]]).repeat(12, 1)
    u = torch.full((12, 3), 0.5)
    t = torch.ones(12)
    x[:, :, 3] = 30.0  # accepted, then ...
    q[:, :, 3] = 30.0
    x[0, 1] = NAN                       # no distribution of the target
    x[1, 1, 7] = INF
    x[2, 1] = -INF
    q[3, 1, 5] = NAN                    # none of the draft model
    drafts[4, 1] = V                    # no class
    drafts[5, 1] = -5
    q[6, 1, 4] = -INF                   # impossible for the draft model: u 0 < p
    x[7, 1, 4] = -INF                   # impossible for the target
    x[8, 1] = -INF                      # one class is left
    x[8, 1, 77] = torch.finfo(torch.float32).min
    t[9], t[10], t[11] = NAN, INF, -1.0  # stand for 0
    x[9:, 1, 4] = 50.0
    r = ops.verify_drafts(x.cuda(), drafts.cuda(), u.cuda(), draft_logits=q.cuda(), temperature=t.cuda())
    check_verify(r, plain_verify(x, drafts, u, q, None, t), V)
    assert r.tokens[:4, 1].tolist() == [-1] * 4 and r.accepted[8].item() == 1 and r.tokens[8, 1].item() == 77
    assert r.accepted[9:].tolist() != [0, 0, 0]
    r = ops.verify_drafts(x.cuda(), drafts.cuda(), u.cuda(), temperature=t.cuda())
    check_verify(r, plain_verify(x, drafts, u, None, None, t), V)
    for low in (1e-45, 1e-30, 1e-3, 3e38):  # the largest class, or nearly all alike
        tt = torch.full((12,), low)
        r = ops.verify_drafts(x.cuda(), drafts.cuda(), u.cuda(), draft_logits=q.cuda(), temperature=tt.cuda())
        tokens, _, _, clear = plain_verify(x, drafts, u, q, None, tt)
        # at 3e38 all classes are alike to 1e-37: p - q and the half of 3000 equal terms are below what 64 bits hold,
        # below 1 p - q is 0 exactly where it is less than 1e-9 (both whole on one class)
        for got, want, yes in zip(r.tokens.tolist(), tokens, clear):
            assert got == want or (low > 1 and not yes)


def test_verify_lengths_outside_and_no_sequences(ops):
    x, q, drafts, u, _, _ = verify_case(4, 2, 50, torch.bfloat16, torch.bfloat16, 6)
    ln = torch.tensor([-3, 0, 2, 9], dtype=torch.int32)
    r = ops.verify_drafts(x.cuda(), drafts.cuda(), u.cuda(), draft_logits=q.cuda(), lengths=ln.cuda())
    check_verify(r, plain_verify(x, drafts, u, q, ln, None), 50)
    r = ops.verify_drafts(x[:0].cuda(), drafts[:0].cuda(), u[:0].cuda(), draft_logits=q[:0].cuda())
    assert r.tokens.shape == (0, 3) and r.accepted.shape == (0,)


def test_verify_many_sequences(ops):
    """More sequences than one set of launches takes."""
    B, V = 5000, 12
    x, q, drafts, u, lengths, t = verify_case(B, 2, V, torch.float16, torch.float16, 7)
    r = ops.verify_drafts(x.cuda(), drafts.cuda(), u.cuda(), draft_logits=q.cuda(), lengths=lengths.cuda(), temperature=t.cuda())
    check_verify(r, plain_verify(x, drafts, u, q, lengths, t), V)


def test_verify_offsets_past_32_bits(ops):
    stride = (1 << 30) + 3
    buf = torch.zeros(5 * stride + 100, dtype=torch.bfloat16, device="cuda")
    x, q, drafts, u, _, _ = verify_case(2, 1, 100, torch.bfloat16, torch.bfloat16, 11)
    far = buf.as_strided((2, 2, 100), (2 * stride, stride, 1))
    far.copy_(x)
    qfar = buf[200:].as_strided((2, 1, 100), (4 * stride, 4 * stride, 1))
    qfar.copy_(q)
    a = ops.verify_drafts(far, drafts.cuda(), u.cuda(), draft_logits=qfar)
    b = ops.verify_drafts(x.cuda(), drafts.cuda(), u.cuda(), draft_logits=q.cuda())
    assert all(torch.equal(s, t) for s, t in zip(a, b))


def test_verify_refusals(ops):
    x, q, drafts, u, ln, t = on_gpu(*verify_case(2, 2, 9, torch.float32, torch.float32, 1))
    for bad in (lambda: ops.verify_drafts(x[0], drafts, u), lambda: ops.verify_drafts(x, drafts[:, :1], u),
                lambda: ops.verify_drafts(x, drafts, u[:, :2]), lambda: ops.verify_drafts(x, drafts, u.double()),
                lambda: ops.verify_drafts(x, drafts.float(), u), lambda: ops.verify_drafts(x.double(), drafts, u),
                lambda: ops.verify_drafts(x, drafts, u, draft_logits=x), lambda: ops.verify_drafts(x, drafts, u, draft_logits=q.double()),
                lambda: ops.verify_drafts(x, drafts, u, lengths=ln.long()), lambda: ops.verify_drafts(x, drafts, u, temperature=t[:1]),
                lambda: ops.verify_drafts(x, drafts, u.cpu()), lambda: ops.verify_drafts(x.transpose(0, 1), drafts, u),
                lambda: ops.verify_drafts(torch.zeros(1, 66, 4, device="cuda"), torch.zeros(1, 65, dtype=torch.int32, device="cuda"),
                                          torch.zeros(1, 66, device="cuda"))):
        with pytest.raises(ValueError):
            bad()


def test_verify_draw_at_zero(ops):
    """A uniform number of 0 draws the first class that has any probability, here 2^-1074 before two large ones."""
    x = torch.full((2, 1, 6000), -INF)
    x[0, 0, 17], x[0, 0, 4000], x[0, 0, 5000] = -744.5, 0.0, 0.0
    x[1, 0, 4000] = 3.0
    r = ops.verify_drafts(x.cuda(), torch.zeros(2, 0, dtype=torch.int32, device="cuda"), torch.zeros(2, 1, device="cuda"))
    assert r.tokens[:, 0].tolist() == [17, 4000] and r.accepted.tolist() == [0, 0]


# ------------------------------------------------------------------ ranges of adapters
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("big,small", [(2.0 ** 14, 2.0 ** -14), (2.0 ** -14, 2.0 ** 3), (2.0 ** 12, 1.0)])
def test_adapter_hidden_values_past_16_bits(big, small, dtype, ops):
    """Hidden values far beyond the range of f16 on both sides, rows of very different size beside each other."""
    c = Adapters(130, 3, 20, 260, 140, dtype, 21)
    c.x = (c.x.float() * big * torch.where(torch.arange(130) % 3 == 0, 1.0, 2.0 ** -9)[:, None]).clamp(-6e4, 6e4).to(dtype)
    c.dy = (c.dy.float() * big).clamp(-6e4, 6e4).to(dtype)
    c.down, c.up = (c.down.float() * 16).to(dtype), (c.up.float() * small).to(dtype)
    x, ids, down, up, scales, dy = on_gpu(c.x, c.ids, c.down, c.up, c.scales, c.dy)
    y, tol, h, th = c.forward(None)
    got, hidden = ops.adapter_product(x, ids, down, up, scales, dtype=torch.float32, hidden=True)
    near(hidden, h, th, "hidden")
    near(got, y, tol, "y")
    r = ops.adapter_product_grad(dy, x, ids, down, up, scales, out=torch.empty(130, 260, device="cuda"))
    for g, (w, t), what in zip(r, c.backward(None), ("dx", "ddown", "dup")):
        near(g, w, t, what)


# ------------------------------------------------------------------ together, streams, graphs
class AdaptedLayer:
    """A layer with many classes whose weights are fixed in 8 bits, with adapters
    beside them: a training step of the adapters (float32 with bf16 working copies),
    clipped, and the verification of drafts from the adapted logits."""

    def __init__(self, ops, N, C, K, n, rank, seed=0):
        g = gen(seed)
        self.ops, self.N, self.C, self.n, self.rank = ops, N, C, n, rank
        self.w = ops.quantize_blocks((torch.randn(C, K, generator=g) / math.sqrt(K)).cuda(), tiles=True, columns=True)
        self.x = torch.randn(N, K, generator=g).bfloat16().cuda()
        self.ids = (torch.arange(N) * n // N - (torch.arange(N) % 11 == 0).long() * n).cuda()
        y = torch.randint(0, C, (N,), generator=g)
        y[::7] = -1
        self.y = y.cuda()
        self.g = torch.full((N,), -1.0 / N, device="cuda")
        self.down = (torch.randn(n, rank, K, generator=g) / math.sqrt(K)).cuda()
        self.up = (torch.randn(n, rank, C, generator=g) * 0.1).cuda()
        self.copies = [self.down.bfloat16(), self.up.bfloat16()]
        self.scales = (torch.rand(n, generator=g) + 0.5).cuda()
        self.opt = ops.AdamW([self.down, self.up], copies=self.copies, grad_dtype=torch.float32, lr=1e-2)
        self.drafts = torch.randint(0, C, (N // 4, 3), generator=g).cuda()
        self.given = torch.randn(N // 4, 3, C, generator=g).cuda()
        self.u = torch.rand(N // 4, 4, generator=g).cuda()

    def logits(self):
        o = self.ops
        xq, _ = o.quantize_blocks(self.x)
        base = o.block_product(xq, self.w[0])
        return o.adapter_product(self.x, self.ids, *self.copies, scales=self.scales, base=base, out=base, hidden=True)

    def step(self):
        o = self.ops
        logits, hidden = self.logits()
        r = o.log_probs(logits, self.y)
        d = o.log_probs_grad(logits, self.y, r.lse, self.g)
        dq, _ = o.quantize_blocks(d)
        dx = o.block_product(dq, self.w[1])
        a = o.adapter_product_grad(d, self.x, self.ids, *self.copies, scales=self.scales, hidden=hidden, base=dx, out=dx)
        n = o.grad_norm([a.down, a.up], 1e-3)
        self.opt.step([a.down, a.up], factor=n.factor)
        v = o.verify_drafts(logits.view(self.N // 4, 4, self.C), self.drafts, self.u, draft_logits=self.given)
        return [logits, hidden, r.logp, d, *a, *n, *v]

    def state(self):
        return [self.down, self.up, *self.copies, self.opt.m, self.opt.v]


@pytest.mark.parametrize("N,C,K,n,rank", [(64, 1000, 300, 3, 8), (132, 515, 129, 5, 33)])
def test_training_step_of_adapters(N, C, K, n, rank, ops):
    """The chain's gradient against autograd in 64 bits of the same loss at the same values."""
    say("adapted layer", N, C, K, n, rank)
    layer = AdaptedLayer(ops, N, C, K, n, rank)
    down, up = (t.double().cpu().requires_grad_(True) for t in layer.copies)
    was = [t.clone() for t in (layer.down, layer.up)]
    logits, hidden, logp, d, dx, dd, du, norm, factor, norms, tokens, accepted, lp = layer.step()
    x, ids, s = layer.x.double().cpu().requires_grad_(True), layer.ids.cpu(), layer.scales.double().cpu()
    xq = ops.quantize_blocks(layer.x)[0].values(torch.float64).cpu()
    w = layer.w[0].values(torch.float64).cpu()
    on = ids >= 0
    a = ids.clamp(min=0)
    h = torch.bmm(down[a], x[:, :, None])[:, :, 0]
    extra = s[a, None] * torch.bmm(h[:, None], up[a])[:, 0] * on[:, None]
    base = (xq @ w.t()).bfloat16().double()  # the shared projection is rounded before the adapters are added
    full = base + extra
    # the logits: the base's rounding may fall the other way (2^-8 of it), and their own
    assert torch.all((logits.cpu().double() - full).abs() <= 2.0 ** -8 * (base.abs() + full.abs()) + 1e-4)
    # the gradient in the logits as it was returned, through the adapters
    dl = d.cpu().double()
    extra.backward(dl)
    dxw = ops.block_product(ops.quantize_blocks(d)[0], layer.w[1]).cpu().double()
    assert (dx.cpu().double() - (x.grad + dxw)).norm() <= 2.0 ** -8 * (x.grad + dxw).norm()
    for got, t in ((dd, down), (du, up)):
        assert (got.cpu().double() - t.grad).norm() <= 1e-5 * t.grad.norm()  # sums of up to C float32 terms, (C + N) u
    want = math.sqrt(float(dd.double().square().sum() + du.double().square().sum()))
    assert close(norm.item(), want) and close(factor.item(), min(1.0, 1e-3 / want), 4)
    # and a step that a plain one on the scaled gradients repeats to the bit
    twin = [t.clone() for t in was]
    opt = ops.AdamW(twin, lr=1e-2)
    opt.step([dd * factor, du * factor])
    assert torch.equal(twin[0], layer.down) and torch.equal(twin[1], layer.up)
    assert torch.equal(layer.copies[0], layer.down.bfloat16())
    r = plain_verify(logits.cpu().view(N // 4, 4, C), layer.drafts.cpu(), layer.u.cpu(), layer.given.cpu(), None, None)
    assert tokens.tolist() == r[0] and accepted.tolist() == r[1]


def test_adapted_layers_in_graphs(ops):
    """Two captured steps of two layers, replayed in turn with eager work between them, against eager steps of twins."""
    sizes = [(40, 600, 200, 3, 8), (136, 300, 70, 2, 40)]
    layers = [AdaptedLayer(ops, *z, seed=i) for i, z in enumerate(sizes)]
    twins = [AdaptedLayer(ops, *z, seed=i) for i, z in enumerate(sizes)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for a in layers:
            a.step()
    torch.cuda.current_stream().wait_stream(side)
    for b in twins:
        b.step()
    graphs, outs = [], []
    for a in layers:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(a.step())
        graphs.append(g)
    for i in range(4):
        for k in (0, 1):
            if i == 2:  # other rows' adapters, drafts and numbers in the captured memory
                for t in (layers[k], twins[k]):
                    t.ids.copy_(t.ids.flip(0))
                    t.u.copy_(1 - 2.0 ** -24 - t.u)
                    t.drafts.copy_((t.drafts + 1) % t.C)
            graphs[k].replay()
            want = twins[k].step()
            torch.cuda.synchronize()
            for x, y in zip(outs[k], want):
                assert torch.equal(x, y), (i, k)
            for x, y in zip(layers[k].state(), twins[k].state()):
                assert torch.equal(x, y), (i, k)
        ops.grad_norm([torch.ones(100000, device="cuda")])  # other eager work
        ops.adapter_product(layers[0].x, layers[0].ids, *layers[0].copies)
    assert layers[0].opt.steps == twins[0].opt.steps == 5


def test_streams_at_once(ops):
    """Calls on two streams at the same time, one of them named by the argument."""
    layers = [AdaptedLayer(ops, 128, 3000, 256, 4, 16, seed=s) for s in (1, 2)]

    def calls(a, **kw):
        y, h = ops.adapter_product(a.x, a.ids, *a.copies, scales=a.scales, hidden=True, **kw)
        g = ops.adapter_product_grad(y, a.x, a.ids, *a.copies, hidden=h, **kw)
        out = [torch.empty_like(g.down), torch.empty_like(g.up)]
        n = ops.clip_grads([g.down, g.up], 1e-2, out=out, **kw)
        v = ops.verify_drafts(y.view(32, 4, 3000), a.drafts, a.u, draft_logits=a.given, **kw)
        return [y, h, *g, *out, *n, *v]

    want = [calls(a) for a in layers]
    streams = [torch.cuda.Stream() for _ in layers]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(4):
        with torch.cuda.stream(streams[0]):
            got[0].append(calls(layers[0]))
        with torch.cuda.stream(streams[1]):
            pass
        got[1].append(calls(layers[1], stream=streams[1] if _ % 2 else streams[1].cuda_stream))
    torch.cuda.synchronize()
    for k in (0, 1):
        for r in got[k]:
            for a, b in zip(r, want[k]):
                assert torch.equal(a, b)


def test_written_tensors_count_as_modified(ops):
    c = Adapters(5, 2, 3, 8, 6, torch.float32, 1)
    x, ids, down, up, dy = on_gpu(c.x, c.ids, c.down, c.up, c.dy)
    out, dx = torch.zeros(5, 6, device="cuda"), torch.zeros(5, 8, device="cuda")
    was = out._version, dx._version
    ops.adapter_product(x, ids, down, up, out=out)
    ops.adapter_product_grad(dy, x, ids, down, up, out=dx)
    assert out._version > was[0] and dx._version > was[1]
    p = torch.ones(4, requires_grad=True, device="cuda")
    assert not ops.grad_norm([p]).norm.requires_grad


def test_repeated_calls_give_equal_bits(ops):
    c = Adapters(3000, 6, 40, 700, 500, torch.bfloat16, 4)
    x, ids, down, up, scales, dy = on_gpu(c.x, c.ids, c.down, c.up, c.scales, c.dy)
    first = None
    for _ in range(3):
        y, h = ops.adapter_product(x, ids, down, up, scales, hidden=True)
        r = [y, h, *ops.adapter_product_grad(dy, x, ids, down, up, scales)]
        first = first or r
        assert all(torch.equal(a, b) for a, b in zip(r, first))


@pytest.mark.parametrize("dtype", TYPES)
def test_adapters_of_every_length(dtype, ops):
    """Axes from one element on, around every border of a lane's load, a step and a workgroup's columns."""
    lengths = [*range(1, 19), 23, 24, 25, 31, 33, 63, 64, 65, 127, 128, 129, 191, 255, 257, 511, 512, 513, 519, 520]
    for i, k in enumerate(lengths):
        cols = lengths[-1 - i]
        for rows in (3, 70):
            c = Adapters(rows, 2, 1 + (7 * i) % 40, k, cols, dtype, i)
            dy, x, ids, down, up, scales = on_gpu(c.dy, c.x, c.ids, c.down, c.up, c.scales)
            # the last rows of their memory: nothing may be read behind them
            base = c.base.to(dtype)
            y, tol, h, th = c.forward(base)
            got, hidden = ops.adapter_product(x, ids, down, up, scales, base=base.cuda(), hidden=True)
            near(got, y, tol, ("y", rows, k, cols))
            near(hidden, h, th, ("hidden", rows, k, cols))
            r = ops.adapter_product_grad(dy, x, ids, down, up, scales, base=c.xbase.to(dtype).cuda())
            for g, (w, t), what in zip(r, c.backward(c.xbase.to(dtype)), ("dx", "ddown", "dup")):
                near(g, w, t, (what, rows, k, cols))


def test_adapter_results_of_other_types(ops):
    """Beside float32 operands a base and a result of 16 bits; beside 16 bits no other 16 bits."""
    c = Adapters(70, 3, 5, 40, 300, torch.float32, 6)
    x, ids, down, up, scales = on_gpu(c.x, c.ids, c.down, c.up, c.scales)
    for t in TYPES:
        base = c.base.to(t)
        y, tol, _, _ = c.forward(base)
        got = ops.adapter_product(x, ids, down, up, scales, base=base.cuda())
        assert got.dtype == t
        near(got, y, tol, t)
    with pytest.raises(ValueError):
        ops.adapter_product(x.half(), ids, down.half(), up.half(), dtype=torch.bfloat16)


@pytest.mark.parametrize("V", [300, 5000])
def test_verify_of_equal_distributions(V, ops):
    """A draft that is no class, on rows that are equal: p - q is 0 for every class, and the token is drawn from p."""
    B = 64
    x, _, _, _, _, t = verify_case(B, 1, V, torch.bfloat16, torch.bfloat16, 3)
    u = torch.rand(B, 2, generator=gen(5))
    drafts = torch.full((B, 1), V)
    for temp in (None, torch.full((B,), 0.7)):
        r = ops.verify_drafts(x.cuda(), drafts.cuda(), u.cuda(), draft_logits=x[:, :1].contiguous().cuda(),
                              temperature=None if temp is None else temp.cuda())
        assert r.accepted.tolist() == [0] * B
        for b in range(B):
            c = distribution(x[b, 0], 1.0 if temp is None else float(temp[b])).cumsum(0)
            assert r.tokens[b, 0].item() == int((c > float(u[b, 1]) * float(c[-1])).nonzero()[0])
