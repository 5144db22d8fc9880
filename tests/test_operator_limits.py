"""The tensor operators where their arithmetic is at a limit: sums whose terms
cancel, logits of large magnitude, second moments below the normal range, and
what a state leaves out.  u = 2^-24 is half a step of float32."""

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


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


# ------------------------------------------------------------------ 8-bit blocks
# Every form of the product: few rows on either side, split and not, 128 x 128
# tiles, split and not, 256 x 256 tiles, with contractions of every rest of 4 blocks.
SUMS = [(1, 100, 128), (1, 40, 9000), (16, 50, 500), (20, 300, 1100), (700, 32, 386), (64, 64, 4000), (130, 129, 258),
        (129, 200, 1026), (300, 515, 640), (2304, 2304, 100), (2304, 2050, 254), (2304, 2050, 514), (2100, 4097, 640), (2049, 2304, 770), (2304, 2304, 1030)]


@pytest.mark.parametrize("m,n,k", SUMS)
def test_block_product_of_terms_that_cancel(m, n, k, ops):
    """Two products of 448 x 448 that cancel in every block beside integers up to
    9: every partial sum is a whole number below 2^24, which float32 holds, so
    the result is the exact sum, rounded once to the output's type."""
    say("products that cancel", m, n, k)
    x = torch.randint(-3, 4, (m, k), generator=gen(k)).float()
    w = torch.randint(-3, 4, (n, k), generator=gen(k + 1)).float()
    x[:, 0::128] = 448
    x[:, 1::128] = 448
    w[:, 0::128] = 448
    w[:, 1::128] = -448
    a, _ = ops.quantize_blocks(x.cuda())
    want = (x.cuda().double() @ w.cuda().double().t()).float()  # whole numbers: exact in both
    for tiles in (False, True):
        b, _ = ops.quantize_blocks(w.cuda(), tiles=tiles)
        for dtype in (torch.bfloat16, torch.float16):
            got = ops.block_product(a, b, dtype)
            assert torch.equal(got, want.to(dtype))


@pytest.mark.parametrize("m,n,k", [(2, 40, 130), (100, 130, 300), (2304, 2304, 514)])
def test_block_product_at_every_scale(m, n, k, ops):
    """Scale bytes 0 to 254 against their inverses, ones for codes: k exactly
    (2^-127 is below the normal range).  Byte 255 is NaN."""
    say("scales", m, n, k)

    def ones(rows, byte):
        pitch, blocks, spitch = ops.block_shape(rows, k)
        codes = torch.zeros(rows, pitch, dtype=torch.uint8, device="cuda")
        codes[:, :k] = 0x38
        scales = torch.full((blocks, spitch), byte, dtype=torch.uint8, device="cuda")
        return ops.BlockTensor(codes.view(torch.float8_e4m3fn), scales, rows, k)

    want = torch.full((m, n), float(k), device="cuda").to(torch.float16)
    for byte in (0, 1, 2, 3, 60, 127, 200, 253, 254):
        assert torch.equal(ops.block_product(ones(m, byte), ones(n, 254 - byte), torch.float16), want), byte
    assert torch.all(torch.isnan(ops.block_product(ones(m, 255), ones(n, 127))))
    assert torch.all(torch.isnan(ops.block_product(ones(m, 127), ones(n, 255))))


# ------------------------------------------------------------------ AdamW
@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_second_moments_below_the_normal_range(bits, ops):
    """Gradients whose squares, at 1 - beta2, fall below 2^-126, and an eps far
    below their roots: the step follows the formula on the documented float32
    moments (which numpy, like the GPU, keeps below the normal range)."""
    h = dict(lr=0.25, beta1=0.9, beta2=0.999, eps=2.0 ** -100, weight_decay=0.0)
    f = np.float32
    e = np.arange(-74, -49).repeat(128)  # squares from 2^-148 to 2^-100, a block each
    g = (np.ldexp(1 + np.random.default_rng(1).random(e.size), e) * np.where(np.arange(e.size) % 3, 1, -1)).astype(f)
    g[::128] = 0
    p = torch.zeros(g.size, device="cuda")
    opt = ops.AdamW([p], state_bits=bits, **h)
    m, v, w = np.zeros(g.size, f), np.zeros(g.size, f), np.zeros(g.size)
    for t in range(1, 3 if bits == 32 else 2):
        say("adamw below the normal range", bits, t)
        opt.step([torch.from_numpy(g).cuda()])
        m = f(h["beta1"]) * m + f(1 - h["beta1"]) * g
        v = f(h["beta2"]) * v + f(1 - h["beta2"]) * (g * g)
        assert m.dtype == f and v.dtype == f and (t > 1 or np.any((v > 0) & (v < 2.0 ** -126)))
        d = h["lr"] * (m.astype(float) / (1 - h["beta1"] ** t)) / (
            np.sqrt(v.astype(float) / (1 - h["beta2"] ** t)) + h["eps"])
        # the two factors (rounded), root, product and sum, reciprocal, two
        # products: 9 roundings of d, of which the hardware's root and reciprocal
        # are within a step (2 u) each; then w's own
        tol = 11 * U * np.abs(d) * t + U * t * np.abs(w - d)
        w = w - d
        got = p.cpu().double().numpy()
        assert np.all(np.abs(got - w) <= tol), (t, float(np.max(np.abs(got - w) / np.maximum(tol, 1e-300))))
        if bits == 32:
            assert np.array_equal(opt.m.cpu().numpy(), m) and np.array_equal(opt.v.cpu().numpy(), v)
        assert np.all(got[::128] == 0)


# ------------------------------------------------------------------ the gradient of log probabilities
def far_rows(n, dtype):
    """Rows whose log of the sum of exponentials is large against 1, so that
    float32 holds few of its digits; their values are whole steps of the type."""
    d = torch.randn(n, generator=gen(n)).double() * 3
    top = torch.finfo(dtype).max
    at = [v for v in (70.0, -300.0, 20000.0, -60000.0, 1e6, 1e7, -1e7, 1e30) if abs(v) < top]
    rows = [(v + d * max(1.0, abs(v) * torch.finfo(dtype).eps)).to(dtype) for v in at]
    rows.append(torch.full((n,), torch.finfo(dtype).min, dtype=dtype))
    rows.append(torch.full((n,), top, dtype=dtype))
    one = torch.full((n,), torch.finfo(dtype).min, dtype=dtype)
    one[n // 2] = 500.0
    rows.append(one)
    masked = (5000.0 + 4 * d).to(dtype)
    masked[::3] = -float("inf")
    masked[1 % n] = 5000.0
    rows.append(masked)
    rows.append((d * 0.5).to(dtype))  # an ordinary row between them
    return torch.stack(rows)


def grad_by_differences(x, y, g, h):
    """The formula in 64 bits, log p = (x - m) - log Z, and a bound of the same in float32."""
    v = x.double()
    d = v - v.amax(1, keepdim=True)
    logz = d.exp().sum(1, keepdim=True).log()
    logs = d - logz
    p = logs.exp()
    ent = -torch.where(p > 0, p * logs, torch.zeros_like(p)).sum(1, keepdim=True)
    hot = torch.arange(x.shape[1])[None] == y[:, None]
    g = torch.where(y < 0, torch.zeros_like(g), g).double()[:, None]
    h = h.double()[:, None]
    slope = torch.where(p > 0, p * (logs + ent), torch.zeros_like(p))
    # Z: at most n / 64 + 40 additions one after the other, exp of each; log p:
    # the roundings of x - m and of the difference, log Z's error; exp: 1.25 |l| + 2.
    # An ordinary row's log p comes from lse: |lse| u more, at most 64 of them.
    sums = (x.shape[1] / 64 + 60) * U
    size = torch.where(p > 0, logs.abs(), torch.zeros_like(p))
    dl = sums + U * (4 * (1 + logz) + 4 * size + 64)
    dent = 2 * sums + 4 * U + 2 * (sums + 4 * U) * (2 * logz + 1)
    tol = g.abs() * (p * dl + 4 * U * (hot + p)) + h.abs() * p * (dl * (1 + size + ent) + dent + 5 * U * (size + ent))
    tol = tol + 3 * U * (g.abs() * (hot + p) + h.abs() * slope.abs())
    # A p below 2^-126 counts as 0 (exp2 has no results below the normal range):
    # what it would add is lost, at most 2^-126 of |g| + |h| |log p + H|.
    low = torch.where((p > 0) & (p < 2.0 ** -126), g.abs() + h.abs() * (size + ent), torch.zeros_like(p)) * 2.0 ** -126
    return g * (hot.double() - p) - h * slope, tol + low


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("n", [1, 2, 10, 1000, 5000, 131075])
def test_log_probs_grad_of_large_logits(n, dtype, ops):
    say("gradient of large logits", n, dtype)
    x = far_rows(n, dtype)
    rows = x.shape[0]
    y = torch.arange(rows) * 7 % n
    y[3] = -1
    g, h = torch.linspace(0.5, 1.5, rows), torch.linspace(-1, 0.5, rows)
    wide = torch.full((rows, n + 3), 7.0, dtype=dtype)
    wide[:, :n] = x
    xg, yg = wide.cuda()[:, :n], y.cuda()
    f = ops.log_probs(xg, yg)
    eps = torch.finfo(dtype)
    for gg, hh in ((g, None), (g, h), (torch.zeros(rows), h)):
        want, tol = grad_by_differences(x, y, gg, torch.zeros(rows) if hh is None else hh)
        tol = 1.01 * tol + eps.eps / 2 * (want.abs() + tol) + eps.smallest_normal * eps.eps / 2
        args = (yg, f.lse, gg.cuda())
        kw = {} if hh is None else dict(entropy=f.entropy, g_entropy=hh.cuda())
        got = ops.log_probs_grad(xg, *args, **kw)
        far = (got.cpu().double() - want).abs() / tol
        assert torch.all(far <= 1), (far.amax(1), f.lse)
        buf = wide.cuda()  # in place of the logits
        ops.log_probs_grad(buf[:, :n], *args, out=buf[:, :n], **kw)
        assert torch.equal(buf[:, :n], got) and torch.all(buf[:, n:] == 7.0)


def test_log_probs_grad_takes_another_lse_as_it_is(ops):
    """Part of a longer row: its lse is not that of these classes.  The formula
    at what is given, off by the roundings of x - lse and of exp."""
    x = (torch.randint(-64, 64, (4, 300), generator=gen(4)).float() / 16 + torch.tensor([[0.0], [1000.0], [-4000.0], [65536.0]]))
    y = torch.tensor([3, -1, 299, 0])
    lse = torch.logsumexp(x.double(), 1).float() + 2.0
    g = torch.tensor([1.0, 2.0, -0.5, 0.25])
    got = ops.log_probs_grad(x.cuda(), y.cuda(), lse.cuda(), g.cuda()).cpu().double()
    logs = x.double() - lse.double()[:, None]
    p = logs.exp()
    hot = torch.arange(300)[None] == y[:, None]
    w = torch.where(y < 0, torch.zeros_like(g), g).double()[:, None]
    tol = w.abs() * (p * U * (4 * logs.abs() + 4) + 3 * U * (hot + p))
    assert torch.all((got - w * (hot.double() - p)).abs() <= 1.01 * tol)


def test_log_probs_grad_of_float32_to_its_digits(ops):
    """Differences x - lse that float32 holds exactly: what is left is exp, its
    exp2 within a step (2 u), the factor for the rest and their product within u
    each, and the rounding of the result."""
    l = torch.arange(-85 * 64, 20 * 64 + 1).float() / 64
    lse = torch.tensor([20.0, -3.5])
    x = l + lse[:, None]
    g = torch.tensor([1.0, -2.0])  # powers of two: their products are exact
    y = torch.tensor([0, l.numel() - 1])
    got = ops.log_probs_grad(x.cuda(), y.cuda(), lse.cuda(), g.cuda()).cpu().double()
    p = l.double().exp()
    want = -g.double()[:, None] * p
    others = torch.ones(2, l.numel(), dtype=torch.bool)
    others[0, 0] = others[1, -1] = False
    off = ((got - want).abs() / want.abs())[others]
    assert torch.all(off <= 5 * U), float(off.max() / U)


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_state_keeps_the_step_size(bits, ops):
    """A run whose step size was changed goes on from its state bit for bit."""
    g = [torch.randn(1000, generator=gen(k)).cuda() for k in range(3)]
    p = [torch.ones(1000, device="cuda")]
    a = ops.AdamW(p, lr=0.1, state_bits=bits, seed=2)
    a.step([g[0]])
    a.set_lr(3e-4)
    a.step([g[1]])
    assert a.lr == 3e-4
    q = [p[0].clone()]
    b = ops.AdamW(q, lr=0.1, state_bits=bits, seed=2)
    assert b.lr == 0.1
    st = a.state()
    b.load_state(st)
    assert b.lr == 3e-4 and b.steps == 2
    a.step([g[2]])
    b.step([g[2]])
    assert torch.equal(p[0], q[0])
    c = ops.AdamW([p[0].clone()], lr=0.1, state_bits=bits, seed=2)  # a state from before it held the step size
    c.load_state({k: v for k, v in st.items() if k != "lr"})
    assert c.lr == 0.1


# ------------------------------------------------------------------ autograd's record of writes
def test_tensors_written_in_place_count_as_modified(ops):
    """A backward pass over a value that a call has replaced raises, as after
    torch's own operations; over one that the call left alone it runs."""
    def saved(t):
        return (t * t).sum()

    p = [torch.ones(300, device="cuda", requires_grad=True) for _ in range(2)]
    copies = [torch.ones(300, dtype=torch.bfloat16, device="cuda", requires_grad=True), None]
    opt = ops.AdamW(p, copies=copies)
    left = saved(p[0]), saved(copies[0])
    opt.step([None, torch.ones(300, device="cuda")])
    for y in left:
        y.backward()
    gone = [saved(p[0]), saved(p[1]), saved(copies[0])]
    opt.step([torch.ones(300, device="cuda")] * 2)
    for y in gone:
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.backward()
    before = [t._version for t in p]
    with pytest.raises(ValueError):
        opt.step([torch.ones(300, device="cuda"), torch.ones(3, device="cuda")])
    assert [t._version for t in p] == before  # refused: nothing was written

    w = torch.randn(4, 10, device="cuda", requires_grad=True)
    logits = w * 2
    y = saved(logits)
    f = ops.log_probs(logits, torch.zeros(4, dtype=torch.int64, device="cuda"))
    ops.log_probs_grad(logits, torch.zeros(4, dtype=torch.int64, device="cuda"), f.lse, f.lse, out=logits)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()
    a, _ = ops.quantize_blocks(torch.randn(4, 10, device="cuda"))
    out = (torch.ones(4, 4, dtype=torch.bfloat16, device="cuda", requires_grad=True) * 1)
    y = saved(out)
    ops.block_product(a, a, out=out)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()


# ------------------------------------------------------------------ captures
def test_adamw_that_ends_during_a_capture(ops):
    """An object that goes out of use while a graph is captured leaves the
    capture whole; its tables are freed afterwards."""
    p, q = [torch.ones(300, device="cuda")], [torch.ones(300, device="cuda")]
    g = torch.ones(300, device="cuda")
    old, opt = ops.AdamW(q), ops.AdamW(p)
    old.step([g])
    opt.step([g])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        opt.step([g])
        del old
    assert len(ops._ended) == 1
    for k in range(3):
        graph.replay()
        assert opt.steps == k + 2
    other = ops.AdamW(q)
    assert not ops._ended
    other.close()
    other.close()
    r = [torch.ones(300, device="cuda")]
    ref = ops.AdamW(r)
    for _ in range(4):
        ref.step([g])
    assert torch.equal(p[0], r[0])


def test_adamw_refuses_parameters_with_other_memory(ops):
    """A parameter or copy whose memory was replaced after the object was made:
    its old memory may be anyone's by then."""
    g = torch.ones(300, device="cuda")
    for which in range(2):
        p = [torch.ones(300, device="cuda") for _ in range(2)]
        c = [torch.ones(300, dtype=torch.bfloat16, device="cuda"), None]
        opt = ops.AdamW(p, copies=c)
        opt.step([g, g])
        old = (p[0], c[0])[which]
        kept = old.data
        old.data = old.data.clone()
        before = [t.clone() for t in (p[0], p[1], c[0], kept, opt.m)]
        with pytest.raises(ValueError, match="parameter 0"):
            opt.step([g, g])
        assert all(torch.equal(a, b) for a, b in zip(before, (p[0], p[1], c[0], kept, opt.m))) and opt.steps == 1
        opt.step([None, g])  # not stepped, not looked at
        old.data = kept
        opt.step([g, g])
        assert opt.steps == 3
