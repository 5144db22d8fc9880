"""The tensor operators (paper_1903_05133_amd/operators.py) on the GPU against
plain implementations in 64 bits.

Tolerances count roundings: u = 2^-24 for a float32 operation, half a step of
the output's type for the last one.  Sums of n positive float32 terms in any
order of at most n / 64 + 32 sequential additions per chain (the rest is a
tree) are off by at most (n / 64 + 32) u of their value, exp and log by 4 u,
and a difference x - lse carries u (|x| + |lse|)."""

import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import rng

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
    """Inputs are made in float32 whatever default an earlier test left."""
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


# ------------------------------------------------------------------ log_probs
def ordered_top(x, k):
    """Indices of the k largest of a row: NaN first, ties to the lowest index."""
    v = [(0 if math.isnan(a) else 1, -a if not math.isnan(a) else 0.0, j) for j, a in enumerate(x.tolist())]
    return [j for _, _, j in sorted(v)[:k]]


def logits_case(rows, classes, dtype, pad, seed, scale=3.0):
    g = gen(seed)
    x = (torch.randn(rows, classes + pad, generator=g) * scale).to(dtype)
    y = torch.randint(-1, classes, (rows,), generator=g)
    return x, y


def check_log_probs(r, x, labels, top):
    """r: what the operator returned; x, labels on the CPU."""
    y = x.double()
    n = x.shape[1]
    most = y.amax(1)
    good = torch.isfinite(most)
    d = y - most[:, None]  # not x - lse: 64 bits do not hold the lowest float plus log n
    logz = d.exp().sum(1).log()
    lse, logs = most + logz, d - logz[:, None]
    p = logs.exp()
    ent = -(torch.where(p > 0, p * logs, torch.zeros_like(p))).sum(1)
    sum_err = (n / 64 + 40) * U
    # m + log z: the sum's error, log's and the addition's roundings
    tol = sum_err + 4 * U * (1 + lse.abs())
    # (x - m) - log z: the same, with roundings of each difference
    ptol = sum_err + 4 * U * (1 + logz.abs())
    got = r.lse.cpu().double()
    assert torch.equal(good, torch.isfinite(got)), (good, got)
    assert torch.all(torch.isnan(got[~good]))
    assert torch.all((got - lse).abs()[good] <= tol[good])
    if r.entropy is not None:
        # log z - s / z: both sums' errors, each relative to its own value
        z = logz
        etol = 2 * sum_err + 4 * U + 2 * (sum_err + 4 * U) * (z + (z - ent).abs() + 1)
        e = r.entropy.cpu().double()
        assert torch.all((e - ent).abs()[good] <= etol[good])
        assert torch.all(torch.isnan(e[~good]))
    if r.logp is not None:
        lp = r.logp.cpu().double()
        for i, t in enumerate(labels.tolist()):
            if t < 0:
                assert lp[i] == 0
            elif t >= n or not good[i]:
                assert math.isnan(lp[i])
            elif x[i, t] == -INF:
                assert lp[i] == -INF
            else:
                assert abs(lp[i] - logs[i, t]) <= ptol[i] + U * (abs(d[i, t]) + abs(logs[i, t]))
    if top:
        ids, tl = r.top_ids.cpu(), r.top_logp.cpu().double()
        for i in range(x.shape[0]):
            want = ordered_top(x[i].float(), top)
            assert ids[i].tolist() == want, (i, ids[i].tolist(), want)
            for k, j in enumerate(want):
                if not good[i]:
                    assert math.isnan(tl[i, k])
                elif x[i, j] == -INF:
                    assert tl[i, k] == -INF
                else:
                    assert abs(tl[i, k] - logs[i, j]) <= ptol[i] + U * (abs(d[i, j]) + abs(logs[i, j]))


SHAPES = [(1, 1, 1, 0), (3, 2, 2, 1), (1000, 10, 3, 0), (5, 16, 16, 0), (7, 17, 5, 3), (4, 64, 64, 0), (3, 65, 64, 5),
          (33, 257, 1, 0), (9, 1000, 5, 0), (8, 1000, 9, 1), (6, 1024, 64, 0), (7, 65, 64, 0), (5, 100, 33, 2), (3, 8192, 32, 0), (5, 1025, 20, 0), (4, 2047, 7, 1), (3, 4097, 3, 0), (3, 12289, 20, 1), (2, 8193, 64, 0),
          (2, 8193, 20, 0), (2, 16385, 64, 9), (2, 32769, 20, 0), (1, 50001, 1, 3), (1, 131072, 64, 0),
          (520, 4100, 2, 0), (300, 9001, 20, 0)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,classes,top,pad", SHAPES)
def test_log_probs(rows, classes, top, pad, dtype, ops):
    say("log_probs", rows, classes, top, pad, dtype)
    x, y = logits_case(rows, classes, dtype, pad, seed=rows + classes)
    xg = x.cuda()[:, :classes]
    r = ops.log_probs(xg, y.cuda(), top=top)
    check_log_probs(r, x[:, :classes], y, top)
    r2 = ops.log_probs(xg, y.cuda().int(), top=top)  # labels of 32 bits, and the same bits again
    for a, b in zip(r, r2):
        assert a is None or torch.equal(a, b)


def special_rows(n, dtype, seed=0):
    """Rows where the order, the sums or the mask can go wrong."""
    g = gen(seed)
    low = torch.finfo(dtype).min
    base = torch.randn(n, generator=g)
    rows = {}
    rows["constant"] = torch.full((n,), 0.5)
    rows["ascending"] = torch.arange(n).float() / max(1, n // 8)
    rows["descending"] = -torch.arange(n).float() / max(1, n // 8)
    rows["empty"] = torch.full((n,), -INF)
    one = torch.full((n,), -INF)
    one[n * 2 // 3] = -7.0
    rows["one_left"] = one
    few = torch.full((n,), -INF)
    few[torch.randperm(n, generator=g)[:3]] = base[:3] if n >= 3 else base[:n]
    rows["few_left"] = few
    nan = base.clone()
    nan[n // 2] = NAN
    nan[n - 1] = NAN
    rows["nan"] = nan
    both = base.clone()
    both[0] = INF
    both[n // 3] = NAN
    rows["inf_and_nan"] = both
    inf = base.clone()
    inf[n // 2] = INF
    rows["inf"] = inf
    lowest = base.clone()
    lowest[torch.rand(n, generator=g) < 0.5] = low
    rows["lowest"] = lowest
    rows["all_lowest"] = torch.full((n,), low)
    zeros = torch.zeros(n)
    zeros[::2] = -0.0
    rows["zeros"] = zeros
    rows["last_is_largest"] = torch.where(torch.arange(n) == n - 1, torch.tensor(30.0), base)
    rows["ties"] = torch.randint(-2, 3, (n,), generator=g).float()
    rows["large"] = base * 1000 + 20000
    rows["only_nan"] = torch.full((n,), NAN)
    half = torch.where(torch.arange(n) < n // 2, torch.tensor(-INF), base)
    rows["first_half_masked"] = half
    return rows


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [1, 3, 10, 100, 1000, 5000, 40000, 131072])
def test_log_probs_special_rows(n, dtype, ops):
    say("special rows", n, dtype)
    rows = special_rows(n, dtype)
    x = torch.stack(list(rows.values())).to(dtype)
    y = torch.arange(len(rows)) % n
    for top in sorted({0, 1, min(n, 8), min(n, 64)}):
        check_log_probs(ops.log_probs(x.cuda(), y.cuda(), top=top), x, y, top)
    # labels that are not: below 0 and past the end
    y = torch.where(torch.arange(len(rows)) % 2 == 0, torch.tensor(-1), torch.tensor(n))
    check_log_probs(ops.log_probs(x.cuda(), y.cuda()), x, y, 0)
    # many rows: the form that takes a row in one workgroup
    reps = 700 // len(rows) + 1
    if n <= 5000:
        xx = x.repeat(reps, 1)
        yy = torch.arange(xx.shape[0]) % n
        r = ops.log_probs(xx.cuda(), yy.cuda(), top=min(n, 8))
        check_log_probs(ops.LogProbs(*(t[:len(rows)] for t in r)), x, yy[:len(rows)], min(n, 8))
        for t in r[1:]:  # every repetition the same, but for logp, whose labels differ
            t = t.reshape(reps, len(rows), -1)
            assert torch.all((t == t[:1]) | (torch.isnan(t) & torch.isnan(t[:1])))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,top", [(9001, 20), (20000, 33), (140001, 64)])
def test_log_probs_lists_made_again(n, top, dtype, ops):
    """More classes at the first bound than a list holds: rows that begin masked or rise, some of them with a NaN."""
    say("lists made again", n, top, dtype)
    base = torch.randn(n, generator=gen(5))
    at = torch.arange(n)
    x = torch.stack([torch.where(at < n * 9 // 10, torch.tensor(-INF), base),
                     torch.where(at < n * 9 // 10, torch.tensor(torch.finfo(dtype).min), base),
                     base.sort().values, torch.where(at < n - top, torch.tensor(-INF), base),
                     torch.where(at < n - top + 1, torch.tensor(-INF), base),
                     torch.where(at == n - 2, torch.tensor(NAN), torch.where(at < n // 2, torch.tensor(-INF), base))]).to(dtype)
    x = torch.cat([x] * 350) if n < 10000 else x  # 2100 rows: one part each
    y = torch.arange(x.shape[0]) % n
    check_log_probs(ops.log_probs(x.cuda(), y.cuda(), top=top), x, y, top)


def test_log_probs_without_labels_or_entropy(ops):
    x, _ = logits_case(5, 300, torch.float32, 0, 1)
    r = ops.log_probs(x.cuda(), top=4, entropy=False)
    assert r.logp is None and r.entropy is None
    check_log_probs(r, x, None, 4)
    r = ops.log_probs(x.cuda()[:0], torch.zeros(0, dtype=torch.int64, device="cuda"), top=2)
    assert r.logp.shape == (0,) and r.top_ids.shape == (0, 2)
    x3 = x[:4].view(2, 2, 300).cuda()
    r = ops.log_probs(x3, torch.zeros(2, 2, dtype=torch.int64, device="cuda"), top=3)
    assert r.lse.shape == (2, 2) and r.top_ids.shape == (2, 2, 3)


def grad_reference(x, labels, g, h):
    """The formula in 64 bits, and the magnitude its roundings are relative to."""
    y = x.double()
    most = y.amax(1, keepdim=True)
    logs = y - most
    logz = logs.exp().sum(1, keepdim=True).log()
    lse, logs = most + logz, logs - logz
    p = logs.exp()
    plogp = torch.where(p > 0, p * logs, torch.zeros_like(p))
    ent = -plogp.sum(1, keepdim=True)
    hot = torch.zeros_like(p)
    for i, t in enumerate(labels.tolist()):
        if t >= 0:
            hot[i, t] = 1
    g = torch.where(labels < 0, torch.zeros_like(g), g).double()[:, None]
    h = h.double()[:, None]
    slope = torch.where(p > 0, p * (logs + ent), torch.zeros_like(p))
    sums = (x.shape[1] / 64 + 60) * U
    # l = x - lse is off by its roundings and by lse's error, absolutely: a
    # small l (p near 1) too.  p = exp(l) is off by as much relatively.
    dl = sums + 4 * U * (1 + lse.abs() + torch.where(p > 0, y.abs(), torch.zeros_like(p)))
    # entropy as check_log_probs bounds it
    dent = 2 * sums + 4 * U + 2 * (sums + 4 * U) * (logz + (logz - ent).abs() + 1)
    logs0 = torch.where(p > 0, logs.abs(), torch.zeros_like(p))
    # g ([j = t] - p): p's error and three roundings.  h p (l + H): the errors of
    # l and H times p, p's error times |l + H|, four roundings of each factor.
    tol = g.abs() * (p * dl + 3 * U * (hot + p)) + h.abs() * p * (dl + dent + dl * (logs0 + ent) + 4 * U * (logs0 + ent))
    tol = tol + 2 * U * (g.abs() * (hot + p) + h.abs() * slope.abs())  # the last sum
    return g * (hot - p) - h * slope, tol


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,classes,pad", [(1, 1, 0), (3, 2, 1), (40, 10, 0), (7, 17, 3), (9, 1000, 0), (5, 1025, 1),
                                              (3, 4099, 5), (2, 50001, 7), (600, 130, 0)])
def test_log_probs_grad(rows, classes, pad, dtype, ops):
    say("log_probs_grad", rows, classes, pad, dtype)
    x, y = logits_case(rows, classes, dtype, pad, seed=classes)
    g, h = torch.randn(rows, generator=gen(5)), torch.randn(rows, generator=gen(6))
    xv, buf = x[:, :classes], x.cuda()
    xg, yg = buf[:, :classes], y.cuda()
    f = ops.log_probs(xg, yg)
    zero = torch.zeros(rows)
    for gg, hh in ((g, None), (None, h), (g, h)):
        want, tol = grad_reference(xv, y, zero if gg is None else gg, zero if hh is None else hh)
        got = ops.log_probs_grad(xg, yg if gg is not None else None, f.lse, None if gg is None else gg.cuda(),
                                 entropy=None if hh is None else f.entropy, g_entropy=None if hh is None else hh.cuda())
        assert got.dtype == dtype and got.shape == xg.shape
        tol = tol * 1.01 + half_step(dtype) * want.abs() + torch.finfo(dtype).smallest_normal * half_step(dtype)
        assert torch.all((got.cpu().double() - want).abs() <= tol)
    # in place of the logits; the buffer's padding stays
    before = buf.clone()
    out = ops.log_probs_grad(xg, yg, f.lse, g.cuda(), entropy=f.entropy, g_entropy=h.cuda(), out=xg)
    assert out is xg and torch.equal(xg, got) and torch.equal(buf[:, classes:], before[:, classes:])


def test_log_probs_grad_formula_against_differences():
    """The formula itself: central differences of the 64-bit forward."""
    x = torch.randn(3, 7, generator=gen(1), dtype=torch.float64)
    y = torch.tensor([2, -1, 6])
    g, h = torch.tensor([0.7, 5.0, -0.3]), torch.tensor([0.2, -0.4, 0.0])

    def loss(x):
        logs = torch.log_softmax(x, 1)
        ent = -(logs.exp() * logs).sum(1)
        lp = torch.stack([logs[i, t] if t >= 0 else logs.new_zeros(()) for i, t in enumerate(y.tolist())])
        return (g.double() * lp + h.double() * ent).sum()

    want, _ = grad_reference(x, y, g, h)
    e = 1e-6
    for i in range(3):
        for j in range(7):
            d = torch.zeros_like(x)
            d[i, j] = e
            # the truncation is e^2 / 6 times a third derivative below 10, the rounding 2^-52 / e
            assert abs((loss(x + d) - loss(x - d)) / (2 * e) - want[i, j]) < 1e-8


@pytest.mark.parametrize("dtype", TYPES)
def test_log_probs_grad_special_rows(dtype, ops):
    n = 3000
    rows = special_rows(n, dtype)
    x = torch.stack(list(rows.values())).to(dtype)
    names = list(rows)
    y = torch.arange(len(rows)) % n
    xg, yg = x.cuda(), y.cuda()
    f = ops.log_probs(xg, yg)
    good = torch.isfinite(torch.logsumexp(x.double(), 1))
    g, h = torch.full((len(rows),), 0.5), torch.full((len(rows),), 0.25)
    got = ops.log_probs_grad(xg, yg, f.lse, g.cuda(), entropy=f.entropy, g_entropy=h.cuda()).cpu().double()
    want, tol = grad_reference(x, y, g, h)
    tol = tol * 1.01 + half_step(dtype) * want.abs() + torch.finfo(dtype).smallest_normal * half_step(dtype)
    for i, name in enumerate(names):
        if good[i]:
            assert torch.all((got[i] - want[i]).abs() <= tol[i]), name
        else:
            assert torch.all(torch.isnan(got[i])), name
    # no weight: zeros, whatever the row holds; no label and no entropy weight: zeros
    zero = torch.zeros(len(rows), device="cuda")
    assert torch.all(ops.log_probs_grad(xg, yg, f.lse, zero, entropy=f.entropy, g_entropy=zero) == 0)
    assert torch.all(ops.log_probs_grad(xg, torch.full_like(yg, -1), f.lse, g.cuda()) == 0)
    # a label past the end: NaN
    assert torch.all(torch.isnan(ops.log_probs_grad(xg, torch.full_like(yg, n), f.lse, g.cuda())))


def test_log_probs_offsets_past_32_bits(ops):
    """Two rows 2^31 + 3 elements apart."""
    stride, n = (1 << 31) + 3, 1000
    buf = torch.empty(stride + n, dtype=torch.bfloat16, device="cuda")
    x, y = logits_case(2, n, torch.bfloat16, 0, 3)
    v = buf.as_strided((2, n), (stride, 1))
    v.copy_(x)
    r = ops.log_probs(v, y.cuda(), top=5)
    check_log_probs(r, x, y, 5)
    g = torch.ones(2, device="cuda")
    out = ops.log_probs_grad(v, y.cuda(), r.lse, g)
    dense = ops.log_probs_grad(x.cuda(), y.cuda(), r.lse, g)
    assert torch.equal(out, dense)
    ops.log_probs_grad(v, y.cuda(), r.lse, g, out=v)
    assert torch.equal(v, dense)


@pytest.mark.parametrize("classes", [3, 1100])
def test_log_probs_many_rows(classes, ops):
    """More rows than a grid's second dimension takes: those around the border."""
    rows = 70000
    x = torch.randn(rows, classes, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    y = torch.arange(rows, device="cuda") % (classes + 1) - 1
    g, h = torch.linspace(-1, 1, rows, device="cuda"), torch.linspace(1, -1, rows, device="cuda")
    r = ops.log_probs(x, y, top=2)
    d = ops.log_probs_grad(x, y, r.lse, g, entropy=r.entropy, g_entropy=h)
    for a in (0, 65530, rows - 8):
        part = slice(a, a + 8)
        check_log_probs(ops.LogProbs(*(t[part] for t in r)), x[part].cpu(), y[part].cpu(), 2)
        want, tol = grad_reference(x[part].cpu(), y[part].cpu(), g[part].cpu(), h[part].cpu())
        assert torch.all((d[part].cpu().double() - want).abs() <= 1.01 * tol + U * want.abs())


@pytest.mark.parametrize("classes,top", [(65, 9), (20, 1)])
def test_log_probs_rows_past_a_grid(classes, top, ops):
    """More rows than one launch has workgroups: those around the border and at the ends."""
    rows = 2 ** 24 + 5
    x = torch.randn(rows, classes, dtype=torch.float16, device="cuda",
                    generator=torch.Generator(device="cuda").manual_seed(2))
    y = (torch.arange(rows, device="cuda") % classes).int()
    r = ops.log_probs(x, y, top=top)
    for a in (0, 2 ** 24 - 8, rows - 8):
        part = slice(a, a + 8)
        check_log_probs(ops.LogProbs(*(t[part] for t in r)), x[part].cpu(), y[part].cpu(), top)
    assert bool(torch.isfinite(r.logp).all()) and int(r.top_ids.min()) == 0 and int(r.top_ids.max()) == classes - 1


def test_log_probs_refusals(ops):
    x = torch.zeros(4, 8, device="cuda")
    y = torch.zeros(4, dtype=torch.int64, device="cuda")
    for bad in (lambda: ops.log_probs(x, y, top=9), lambda: ops.log_probs(x, y, top=-1),
                lambda: ops.log_probs(x.t(), y), lambda: ops.log_probs(x.double(), y),
                lambda: ops.log_probs(x, y[:3]), lambda: ops.log_probs(x, y.float()),
                lambda: ops.log_probs(x, y.cpu()), lambda: ops.log_probs(x.cpu(), y.cpu()),
                lambda: ops.log_probs(x[:1].expand(4, 8), y), lambda: ops.log_probs(torch.zeros(2, 0, device="cuda")),
                lambda: ops.log_probs(torch.zeros(1, 200, device="cuda"), top=65),
                lambda: ops.log_probs_grad(x, y, torch.zeros(4, device="cuda"), None),
                lambda: ops.log_probs_grad(x, None, torch.zeros(4, device="cuda"), torch.zeros(4, device="cuda")),
                lambda: ops.log_probs_grad(x, y, torch.zeros(3, device="cuda"), torch.zeros(4, device="cuda")),
                lambda: ops.log_probs_grad(x, y, torch.zeros(4, device="cuda"), torch.zeros(4, device="cuda"),
                                           out=torch.zeros(4, 9, device="cuda")),
                lambda: ops.log_probs_grad(x, y, torch.zeros(4, device="cuda"), torch.zeros(4, device="cuda"),
                                           g_entropy=torch.zeros(4, device="cuda"))):
        with pytest.raises(ValueError):
            bad()


# ------------------------------------------------------------------ AdamW
TAG = 0x68762E6164616D77  # "hv.adamw"
F32 = np.float32


def pow2(e):
    return np.ldexp(np.float64(1), np.asarray(e).astype(np.int64))


def block_exponent(a, top):
    """Least e in [-127, 127] with max |a| <= top * 2^e."""
    amax = float(np.max(np.abs(a)))
    if amax == 0:
        return 0
    e = -127
    while e < 127 and amax > top * 2.0 ** e:
        e += 1
    return e


def v_value(c):
    c = c.astype(np.int64)
    e, f = c >> 4, c & 15
    return np.where(e == 0, f * 2.0 ** -18, (16 + f) * 2.0 ** (e - 19.0))


def round_random(y, u, mantissa, least):
    """y >= 0 (float32) on a grid with `mantissa` bits and least normal exponent, up where the fraction + u passes one."""
    y = y.astype(np.float32)
    e = np.maximum(np.floor(np.log2(np.maximum(y, F32(2.0 ** -140)).astype(np.float64))), least) - mantissa
    n = np.floor((y / pow2(e)).astype(np.float32) + u.astype(np.float32))
    return n.astype(np.float64) * pow2(e)


def random_bits(seed, t, n):
    key = rng.h_scalar(rng.h_scalar(seed, TAG), t)
    h = rng.h(key, np.arange(-(-n // 2), dtype=np.uint64))
    r = np.empty(2 * len(h), dtype=np.uint64)
    r[0::2], r[1::2] = h & np.uint64(0xFFFFFFFF), h >> np.uint64(32)
    return r[:n]


class Plain:
    """The documented step on the CPU, element by element: float32 where the
    document says so, 64 bits elsewhere."""

    def __init__(self, sizes, hyper, bits, seed=0):
        self.h, self.bits, self.seed, self.t = hyper, bits, seed, 0
        self.sizes, self.starts = sizes, []
        total = 0
        for n in sizes:
            self.starts.append(total)
            total += -(-n // 128) * 128
        self.total = total
        if bits == 32:
            self.m, self.v = np.zeros(total), np.zeros(total)
            self.dm, self.dv = np.zeros(total), np.zeros(total)  # bounds of their rounding
        else:
            self.m, self.v = np.zeros(total, F32), np.zeros(total, F32)
            self.mc, self.vc = np.zeros(total), np.zeros(total)  # values of the codes
            self.ms, self.vs = (np.full(total // 128, 127, np.uint8) for _ in range(2))

    def step(self, params, grads):
        """params (float64 arrays) after a step on grads (float32 arrays or None), and bounds of the roundings."""
        self.t += 1
        h, t = self.h, self.t
        b1, b2 = h["beta1"], h["beta2"]
        bits = random_bits(self.seed, t, self.total) if self.bits == 8 else None
        out = []
        for p, g, s, n in zip(params, grads, self.starts, self.sizes):
            if g is None:
                out.append((p, np.zeros(n)))
                continue
            a = slice(s, s + n)
            if self.bits == 32:
                m, v = b1 * self.m[a] + (1 - b1) * g.astype(np.float64), b2 * self.v[a] + (1 - b2) * g.astype(np.float64) ** 2
                # constants, products and the sum: 3 roundings of each term
                self.dm[a] = b1 * self.dm[a] + 3.01 * U * (abs(b1 * self.m[a]) + abs((1 - b1) * g.astype(np.float64)))
                self.dv[a] = b2 * self.dv[a] + 4.01 * U * v
                self.m[a], self.v[a] = m, v
                dm, dv = self.dm[a], self.dv[a]
            else:
                m = F32(b1) * self.m[a] + F32(1 - b1) * g
                v = F32(b2) * self.v[a] + F32(1 - b2) * (g * g)
                assert m.dtype == F32 and v.dtype == F32
                dm, dv = 2 * U * abs(F32(b1) * self.m[a].astype(np.float64)), 2 * U * v.astype(np.float64)
                self.quantize(s, n, m, v, bits)
            m, v = m.astype(np.float64), v.astype(np.float64)
            c1, c2 = 1 - b1 ** t, 1 - b2 ** t
            den = np.sqrt(v / c2) + h["eps"]
            d = h["lr"] * m / c1 / den
            w = p * (1 - h["lr"] * h["weight_decay"]) - d
            # factors, sqrt, sum, quotient, product: 10 roundings of d, and the decay's and the difference's of p
            tol = h["lr"] * dm / c1 / den + abs(d) * (0.5 * dv / np.maximum(v, 1e-300) + 10 * U) + 3 * U * abs(p)
            out.append((w, tol))
        return out

    def quantize(self, s, n, m, v, bits):
        for i in range(0, n, 128):
            j = min(n, i + 128)
            b = (s + i) // 128
            for x, scales, codes, vals, top, mant, least, shift in (
                    (m[i:j], self.ms, self.mc, self.m, 448.0, 3, -6, 0),
                    (v[i:j], self.vs, self.vc, self.v, 1.9375, 4, -14, 16)):
                if not np.all(np.isfinite(x)):
                    scales[b] = 255
                    codes[s + i:s + j] = 0
                    vals[s + i:s + j] = np.nan
                    continue
                e = block_exponent(x, top)
                u = ((bits[s + i:s + j] >> np.uint64(shift)) & np.uint64(0xFFFF)).astype(np.float32) / F32(65536)
                q = round_random((np.abs(x).astype(np.float64) / pow2(e)).astype(F32), u, mant, least)
                if shift:
                    q = np.where((x > 0) & (q == 0), 2.0 ** -18, q)
                q = np.copysign(q, x)
                scales[b] = e + 127
                codes[s + i:s + j] = q
                vals[s + i:s + j] = (q * pow2(e)).astype(F32)


SIZES = [1, 127, 128, 129, 0, 2047, 2048, 2049, 5000, 3]
HYPER = dict(lr=1e-2, beta1=0.9, beta2=0.95, eps=1e-6, weight_decay=0.1)


def adamw_tensors(sizes, ptype, gtype, seed, offset=0):
    """Parameters as views that start `offset` elements into their buffers."""
    g = gen(seed)
    params = [torch.randn(n + offset, generator=g).to(ptype).cuda()[offset:] for n in sizes]
    grads = [[(torch.randn(n + offset, generator=g) * 10.0 ** (i - 2)).to(gtype).cuda()[offset:] for n in sizes]
             for i in range(4)]
    return params, grads


def check_states(opt, ref):
    if ref.bits == 32:
        m, v = opt.m.cpu().double().numpy(), opt.v.cpu().double().numpy()
        assert np.all(abs(m - ref.m) <= ref.dm) and np.all(abs(v - ref.v) <= ref.dv)
        return
    assert np.array_equal(opt.m_scales.cpu().numpy(), ref.ms)
    assert np.array_equal(opt.v_scales.cpu().numpy(), ref.vs)
    assert np.array_equal(opt.m.cpu().double().numpy(), ref.mc)
    assert np.array_equal(v_value(opt.v.cpu().numpy()), ref.vc)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("ptype,gtype,ctype,offset", [
    (torch.float32, torch.float32, None, 0), (torch.float32, torch.bfloat16, torch.bfloat16, 1),
    (torch.bfloat16, torch.bfloat16, None, 3), (torch.float16, torch.float16, None, 1),
    (torch.float32, torch.float16, torch.float16, 0), (torch.bfloat16, torch.float32, torch.float32, 2)])
def test_adamw_steps(bits, ptype, gtype, ctype, offset, ops):
    say("adamw", bits, ptype, gtype, ctype, offset)
    params, grads = adamw_tensors(SIZES, ptype, gtype, 7, offset)
    copies = None if ctype is None else [torch.zeros(n + offset, dtype=ctype, device="cuda")[offset:] for n in SIZES]
    opt = ops.AdamW(params, state_bits=bits, copies=copies, grad_dtype=gtype, seed=99, **HYPER)
    ref = Plain(SIZES, HYPER, bits, seed=99)
    for step, gs in enumerate(grads):
        if step == 2:
            gs = [g if k % 3 else None for k, g in enumerate(gs)]  # no gradient: the tensor stays
        before = [p.cpu().double().numpy() for p in params]
        opt.step(gs)
        want = ref.step(before, [None if g is None else g.cpu().float().numpy() for g in gs])
        for k, (p, (w, tol)) in enumerate(zip(params, want)):
            got = p.cpu().double().numpy()
            if gs[k] is None:
                assert np.array_equal(got, before[k])
                continue
            tiny = torch.finfo(ptype).smallest_normal * half_step(ptype)
            assert np.all(abs(got - w) <= tol * 1.01 + half_step(ptype) * (abs(w) + tol) + tiny), (step, k)
            if copies is not None and ptype == torch.float32:
                assert torch.equal(copies[k], p.to(ctype))
            elif copies is not None:
                assert np.all(abs(copies[k].cpu().double().numpy() - w) <= tol * 1.01 + U * (abs(w) + tol))
        check_states(opt, ref)
    assert opt.steps == 4


def test_adamw_many_tensors_and_resume(ops):
    """More tensors than one launch takes; a run resumed from a state goes on bit for bit; lr changes."""
    sizes = [(37 * k) % 300 + 1 for k in range(700)]
    params, grads = adamw_tensors(sizes, torch.float32, torch.float32, 11)
    for bits in (32, 8):
        a = [p.clone() for p in params]
        o1 = ops.AdamW(a, state_bits=bits, seed=5, **HYPER)
        o1.step(grads[0])
        o1.step(grads[1])
        b = [p.clone() for p in a]
        o2 = ops.AdamW(b, state_bits=bits, seed=5, **HYPER)
        o2.load_state(o1.state())
        for o in (o1, o2):
            o.set_lr(3e-3)
            o.step(grads[2])
        assert o1.steps == o2.steps == 3
        for x, y in zip(a, b):
            assert torch.equal(x, y)
        assert torch.equal(o1.v, o2.v) and torch.equal(o1.m.view(torch.uint8), o2.m.view(torch.uint8))
        ref = Plain(sizes, HYPER, bits, seed=5)
        w = [p.cpu().double().numpy() for p in params]
        tol = [0.0] * len(w)
        for k in range(3):
            if k == 2:
                ref.h = dict(HYPER, lr=3e-3)
            got = ref.step(w, [g.cpu().numpy() for g in grads[k]])
            w, tol = [x for x, _ in got], [e + t + U * abs(x) for (x, t), e in zip(got, tol)]
        for x, y, t in zip(a, w, tol):
            assert np.all(abs(x.cpu().double().numpy() - y) <= 1.01 * t)


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_non_finite_gradients(bits, ops):
    """A NaN or infinite gradient makes its own parameter NaN at once or at the next step, and with 8 bits its block; no other."""
    p = [torch.ones(1000, device="cuda")]
    g = torch.full((1000,), 0.1, device="cuda")
    opt = ops.AdamW(p, state_bits=bits, **HYPER)
    opt.step([g])
    bad = g.clone()
    bad[300] = NAN
    opt.step([bad])
    opt.step([g])
    got = p[0].cpu()
    nan = torch.isnan(got)
    want = torch.zeros(1000, dtype=torch.bool)
    want[300 if bits == 32 else slice(256, 384)] = True
    if bits == 32:
        want[300] = True
    assert torch.equal(nan, want)
    if bits == 8:
        assert opt.m_scales.cpu()[2] == 255 and opt.v_scales.cpu()[2] == 255
        assert torch.all(opt.m.view(torch.uint8)[256:384] == 0) and torch.all(opt.v[256:384] == 0)


def test_adamw_ranges_of_8_bit_states(ops):
    """Gradients from subnormal to near the type's largest, zeros, and blocks of very different magnitudes."""
    n = 128 * 12 + 5
    g = gen(3)
    x = torch.randn(n, generator=g)
    for b, e in enumerate([-45, -38, -30, -20, -10, -3, 0, 4, 9, 15, 18]):
        x[b * 128:(b + 1) * 128] *= 10.0 ** e
    x[128 * 11:] = 0
    x[5:128 * 10:7] *= 1e-4
    p = [torch.zeros(n, device="cuda")]
    opt = ops.AdamW(p, state_bits=8, seed=1, **HYPER)
    ref = Plain([n], HYPER, 8, seed=1)
    for _ in range(3):
        w = p[0].cpu().double().numpy()
        opt.step([x.cuda()])
        ref.step([w], [x.numpy()])
        check_states(opt, ref)
    assert torch.all(torch.isfinite(p[0]))


def test_adamw_past_32_bits(ops):
    """A tensor of more than 2^31 elements: its last ones against a short tensor with the same random bits."""
    n = (1 << 31) + 384
    p = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    tail = torch.randn(384, generator=gen(2)).to(torch.bfloat16).cuda()
    g[-384:] = tail
    opt = ops.AdamW([p], state_bits=8, seed=3, **HYPER)
    opt.step([g])
    q = torch.zeros(384, dtype=torch.bfloat16, device="cuda")
    o32 = ops.AdamW([q], state_bits=32, seed=3, **HYPER)
    o32.step([tail])
    assert torch.equal(p[-384:], q) and torch.all(p[:1 << 20] == 0)
    key = rng.h_scalar(rng.h_scalar(3, TAG), 1)
    h = rng.h(key, np.arange(1 << 30, (1 << 30) + 192, dtype=np.uint64))
    r = np.empty(384, dtype=np.uint64)
    r[0::2], r[1::2] = h & np.uint64(0xFFFFFFFF), h >> np.uint64(32)
    m = o32.m.cpu().numpy()
    for b in range(3):
        x = m[b * 128:b * 128 + 128]
        e = block_exponent(x, 448.0)
        u = (r[b * 128:b * 128 + 128] & np.uint64(0xFFFF)).astype(F32) / F32(65536)
        want = np.copysign(round_random((np.abs(x).astype(np.float64) / pow2(e)).astype(F32), u, 3, -6), x)
        s = (1 << 31) + b * 128
        assert np.array_equal(opt.m[s:s + 128].cpu().double().numpy(), want)
        assert opt.m_scales[s // 128].item() == e + 127


def test_adamw_without_gradients_counts(ops):
    p = [torch.ones(300, device="cuda"), torch.ones(0, device="cuda")]
    opt = ops.AdamW(p, **HYPER)
    opt.step([None, None])
    assert opt.steps == 1 and torch.all(p[0] == 1) and torch.all(opt.m == 0)
    opt.step((torch.ones(300, device="cuda"), None))
    # step 2's factors: m = 0.1 of a gradient of 1 over 1 - 0.9^2
    d = HYPER["lr"] * (1 - HYPER["beta1"]) / (1 - HYPER["beta1"] ** 2) / (
        math.sqrt((1 - HYPER["beta2"]) / (1 - HYPER["beta2"] ** 2)) + HYPER["eps"])
    want = 1 - HYPER["lr"] * HYPER["weight_decay"] - d
    assert opt.steps == 2 and torch.all((p[0].double() - want).abs() <= 8 * U)


def test_adamw_refusals(ops):
    p = torch.zeros(8, device="cuda")
    for kw in (dict(lr=-1.0), dict(lr=NAN), dict(beta1=1.0), dict(beta2=-0.1), dict(eps=0.0), dict(eps=1e-60),
               dict(weight_decay=-1.0), dict(weight_decay=INF)):
        with pytest.raises(RuntimeError):
            ops.AdamW([p], **kw)
    for bad in (lambda: ops.AdamW([]), lambda: ops.AdamW([p], state_bits=16), lambda: ops.AdamW([p.cpu()]),
                lambda: ops.AdamW([p.double()]), lambda: ops.AdamW([p[::2]]), lambda: ops.AdamW([p], copies=[p, p]),
                lambda: ops.AdamW([p], copies=[p[:4]]), lambda: ops.AdamW([p], grad_dtype=torch.float64),
                lambda: ops.AdamW([p], seed=-1)):
        with pytest.raises(ValueError):
            bad()
    opt = ops.AdamW([p])
    for g in ([], [p[:4]], [p.bfloat16()], [p.cpu()], [torch.zeros(16, device="cuda")[::2]]):
        with pytest.raises(ValueError):
            opt.step(g)
    with pytest.raises(RuntimeError):
        opt.set_lr(NAN)
    with pytest.raises(RuntimeError):
        opt.set_step_count(-1)
    with pytest.raises(ValueError):
        opt.load_state(ops.AdamW([p], state_bits=8).state())
    assert torch.all(p == 0) and opt.steps == 0


@pytest.mark.parametrize("bits", [8, 32])
def test_adamw_smallest_eps(bits, ops):
    """The least eps that is taken: zeros stay, the first step of others is lr to float32's rounding."""
    p = torch.tensor([3.0, -2.0, 5.0], device="cuda")
    opt = ops.AdamW([p], lr=0.5, eps=2.0 ** -126, weight_decay=0.0, state_bits=bits)
    opt.step([torch.tensor([0.0, 2.0, -4.0], device="cuda")])
    # m / c1 and sqrt(v / c2): six roundings and the hardware's root and reciprocal, each within a step; then w's own
    assert float(p[0]) == 3.0 and torch.all((p.double().cpu() - torch.tensor([3.0, -2.5, 5.5])).abs() <= (10 * 0.5 + 6) * U)
    with pytest.raises(RuntimeError, match="overlap"):
        ops.AdamW([p, p[1:]])
    with pytest.raises(RuntimeError, match="overlap"):
        ops.AdamW([p], copies=[p])


# ------------------------------------------------------------------ 8-bit blocks
def quantize_reference(x, tiles):
    """Values of codes [R, Kp] and scale bytes [Rb, blocks] of x (float64 array) by the definition."""
    R, K = x.shape
    Kp, rb = -(-K // 128) * 128, 128 if tiles else 1
    q = np.zeros((R, Kp))
    s = np.zeros((-(-R // rb), Kp // 128), np.uint8)
    for i in range(0, R, rb):
        for k in range(0, K, 128):
            b = x[i:i + rb, k:k + 128]
            fin = b[np.isfinite(b)]
            e = block_exponent(fin, 448.0) if fin.size else 0
            s[i // rb, k // 128] = e + 127
            y = b / pow2(e)
            step = pow2(np.maximum(np.floor(np.log2(np.maximum(np.abs(np.where(np.isfinite(y), y, 0)), 2.0 ** -60))), -6) - 3)
            with np.errstate(invalid="ignore"):
                q[i:i + rb, k:k + b.shape[1]] = np.where(np.isfinite(b), np.rint(y / step) * step, NAN)
    return q, s


def same(a, b):
    return np.array_equal(a, b, equal_nan=True)


def check_blocks(t, x, tiles):
    q, s = quantize_reference(x, tiles)
    assert same(t.codes.cpu().double().numpy(), q)
    got = t.scales.cpu().numpy()
    assert np.array_equal(got[:, :s.shape[1]], s) and np.all(got[:, s.shape[1]:] == 0)


def quant_input(R, K, dtype, seed):
    g = gen(seed)
    x = torch.randn(R, K, generator=g) * torch.exp(3 * torch.randn(R, 1, generator=g))
    x[torch.rand(R, K, generator=g) < 0.1] = 0
    if R > 2 and K > 2:
        x[1, 2], x[R - 1, 0], x[0, K - 1] = NAN, INF, -INF
    return x.to(dtype)


QSHAPES = [(1, 1), (1, 128), (1, 5000), (3, 127), (5, 129), (16, 640), (127, 3), (128, 128), (129, 257), (300, 130),
           (64, 1000), (130, 1025)]


def test_quantize_rows_past_a_grid(ops):
    """More rows than one launch has waves for: slices around the border and at the ends against calls of their own."""
    rows = 2 ** 26 + 7
    x = torch.randn(rows, 8, dtype=torch.bfloat16, device="cuda",
                    generator=torch.Generator(device="cuda").manual_seed(3))
    q, _ = ops.quantize_blocks(x)
    for a in (0, 2 ** 26 - 16, rows - 32):
        part = slice(a, a + 32)
        one, _ = ops.quantize_blocks(x[part].clone())
        assert torch.equal(q.codes[part].view(torch.uint8), one.codes.view(torch.uint8))
        assert torch.equal(q.scales[part], one.scales)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("R,K", QSHAPES)
def test_quantize_blocks(R, K, dtype, ops):
    say("quantize", R, K, dtype)
    x = quant_input(R, K, dtype, R + K)
    xd = x.double().numpy()
    wide = torch.full((R, K + 5), 7.0).to(dtype)
    wide[:, :K] = x
    for xg in (x.cuda(), wide.cuda()[:, :K]):
        for tiles in (False, True):
            a, t = ops.quantize_blocks(xg, tiles=tiles, rows=True, columns=True)
            check_blocks(a, xd, tiles)
            check_blocks(t, xd.T, tiles)
            only, none = ops.quantize_blocks(xg, tiles=tiles)
            assert none is None and torch.equal(only.codes.view(torch.uint8), a.codes.view(torch.uint8))
            assert torch.equal(only.scales, a.scales)
            none, only = ops.quantize_blocks(xg, tiles=tiles, rows=False, columns=True)
            assert none is None and torch.equal(only.codes.view(torch.uint8), t.codes.view(torch.uint8))
            assert torch.equal(only.scales, t.scales)
    v = a.values(torch.float64).cpu().numpy()
    q, s = quantize_reference(xd, True)
    assert same(v, (q * np.repeat(np.repeat(pow2(s.astype(int) - 127), 128, 0)[:R], 128, 1))[:, :K])


def test_quantize_ranges(ops):
    """Every binade of float32, subnormals included, borders of a scale, ties of the rounding."""
    rows = [np.full(128, 2.0 ** e) * np.linspace(0.1, 1.9, 128) for e in range(-149, 127)]
    rows += [np.array([448.0] + [k * 0.5 + 0.25 for k in range(127)]), np.array([448.0001] * 128), np.zeros(128),
             np.array([np.finfo(F32).max] * 128), np.array([1e-45] * 128), np.array([448.0] + [2.0 ** -10 * k for k in range(127)])]
    x = np.array(rows).astype(F32)
    for dtype in (torch.float32,):
        xg = torch.tensor(x).to(dtype).cuda()
        a, t = ops.quantize_blocks(xg, rows=True, columns=True)
        check_blocks(a, x.astype(np.float64), False)
        check_blocks(t, x.astype(np.float64).T, False)


def product_reference(a, b):
    """In 64 bits, and the bound of the matrix cores' sums: each product of a
    block of 128 is kept to 2^-17 of the block's largest, the sums over blocks
    are in float32."""
    x, y = a.values(torch.float64).cpu(), b.values(torch.float64).cpu()
    K = x.shape[1]
    ref = x @ y.t()
    big = torch.zeros_like(ref)
    for k in range(0, K, 128):
        big += x[:, k:k + 128].abs().amax(1)[:, None] * y[:, k:k + 128].abs().amax(1)[None]
    total = x.abs() @ y.abs().t()
    return ref, 128 * 2.0 ** -17 * big + (K / 128 + 8) * U * total


PSHAPES = [(1, 1, 1), (1, 16, 128), (1, 1000, 5000), (2, 130, 1000), (3, 17, 129), (15, 300, 640), (16, 128, 256),
           (17, 129, 257), (33, 65, 1024), (64, 64, 128), (65, 200, 300), (100, 1030, 130), (128, 128, 128),
           (129, 257, 1025), (200, 300, 513), (256, 256, 512), (257, 511, 640), (300, 10, 2000), (512, 520, 2049),
           (5, 700, 20000), (700, 5, 20000), (40, 40, 40000), (2049, 4100, 130), (2049, 4100, 258), (2305, 4097, 700), (2048, 4352, 1153),
          (4100, 2050, 513)]


@pytest.mark.parametrize("M,N,K", PSHAPES)
def test_block_product(M, N, K, ops):
    say("product", M, N, K)
    g = gen(M + N + K)
    x = torch.randn(M, K, generator=g) * torch.exp(torch.randn(M, 1, generator=g))
    w = torch.randn(N, K, generator=g) + 0.2
    for at, bt, dtype in ((False, True, torch.bfloat16), (False, False, torch.float16), (True, False, torch.bfloat16)):
        a, _ = ops.quantize_blocks(x.cuda(), tiles=at)
        b, _ = ops.quantize_blocks(w.cuda(), tiles=bt)
        y = ops.block_product(a, b, dtype)
        ref, tol = product_reference(a, b)
        assert y.dtype == dtype and y.shape == (M, N)
        # fp16 outputs past its range are not met: |y| < 20000 here
        tol = tol + half_step(dtype) * (ref.abs() + tol) + torch.finfo(dtype).smallest_normal * half_step(dtype)
        assert torch.all((y.cpu().double() - ref).abs() <= tol)
        wide = torch.full((M, N + 3), 5.0, dtype=dtype, device="cuda")
        assert ops.block_product(a, b, out=wide[:, :N]).data_ptr() == wide.data_ptr()
        assert torch.equal(wide[:, :N], y) and torch.all(wide[:, N:] == 5.0)


def test_block_product_scales_and_nan(ops):
    """Scales from 2^-126 to 2^120 that cancel, and a NaN that reaches its row and column only."""
    x, w = torch.randn(20, 300, generator=gen(1)), torch.randn(30, 300, generator=gen(2))
    for s in (2.0 ** -100, 1.0, 2.0 ** 100):
        a, _ = ops.quantize_blocks((x * s).cuda())
        b, _ = ops.quantize_blocks((w / s).cuda())
        y = ops.block_product(a, b)
        if s == 2.0 ** -100:
            first = y
        assert torch.equal(y, first)
    x[3, 77] = NAN
    a, _ = ops.quantize_blocks(x.cuda())
    b, _ = ops.quantize_blocks(w.cuda())
    y = torch.isnan(ops.block_product(a, b)).cpu()
    assert torch.all(y[3]) and not torch.any(y[:3]) and not torch.any(y[4:])


def test_block_product_offsets_past_32_bits(ops):
    stride = (1 << 31) + 8
    buf = torch.zeros(stride + 40, dtype=torch.bfloat16, device="cuda")
    out = buf.as_strided((2, 40), (stride, 1))
    a, _ = ops.quantize_blocks(torch.randn(2, 200, generator=gen(1)).cuda())
    b, _ = ops.quantize_blocks(torch.randn(40, 200, generator=gen(2)).cuda())
    ops.block_product(a, b, out=out)
    assert torch.equal(out, ops.block_product(a, b))
    src = torch.zeros(stride + 200, dtype=torch.bfloat16, device="cuda")
    x = src.as_strided((2, 200), (stride, 1))
    x.copy_(torch.randn(2, 200, generator=gen(3)))
    c, ct = ops.quantize_blocks(x, columns=True)
    d, dt = ops.quantize_blocks(x.contiguous(), columns=True)
    assert torch.equal(c.codes.view(torch.uint8), d.codes.view(torch.uint8)) and torch.equal(c.scales, d.scales)
    assert torch.equal(ct.codes.view(torch.uint8), dt.codes.view(torch.uint8)) and torch.equal(ct.scales, dt.scales)


def test_blocks_refusals(ops):
    x = torch.zeros(4, 200, device="cuda")
    a, _ = ops.quantize_blocks(x)
    b, _ = ops.quantize_blocks(torch.zeros(4, 100, device="cuda"))
    for bad in (lambda: ops.quantize_blocks(x, rows=False), lambda: ops.quantize_blocks(x.t()),
                lambda: ops.quantize_blocks(x.double()), lambda: ops.quantize_blocks(x.cpu()),
                lambda: ops.quantize_blocks(x[:0]), lambda: ops.quantize_blocks(x[:, :0]),
                lambda: ops.block_product(a, b), lambda: ops.block_product(a, a, torch.float32),
                lambda: ops.block_product(a, a, out=torch.zeros(4, 5, dtype=torch.float16, device="cuda")),
                lambda: ops.BlockTensor(a.codes, a.scales, 4, 300), lambda: ops.BlockTensor(a.codes, a.scales, 4, 200, True),
                lambda: ops.BlockTensor(a.codes.view(torch.uint8), a.scales, 4, 200)):
        with pytest.raises(ValueError):
            bad()


# ------------------------------------------------------------------ together, streams, graphs
class Layer:
    """One training step of a layer with many classes on 8-bit products: y = x
    W^T, loss = -mean log p + 0.01 mean entropy, dx, AdamW on float32 weights."""

    def __init__(self, ops, N, C, K, bits, seed=0):
        g = gen(seed)
        self.ops, self.N = ops, N
        self.w = (torch.randn(C, K, generator=g) / math.sqrt(K)).cuda()
        self.x = torch.randn(N, K, generator=g).to(torch.bfloat16).cuda()
        y = torch.randint(0, C, (N,), generator=g)
        y[::7] = -1
        self.y = y.cuda()
        self.g = torch.full((N,), -1.0 / N, device="cuda")
        self.h = torch.full((N,), 0.01 / N, device="cuda")
        self.opt = ops.AdamW([self.w], grad_dtype=torch.bfloat16, state_bits=bits, lr=1e-2, seed=3)

    def step(self):
        o = self.ops
        x, xt = o.quantize_blocks(self.x, columns=True)
        w, wt = o.quantize_blocks(self.w, tiles=True, columns=True)
        logits = o.block_product(x, w)
        r = o.log_probs(logits, self.y, top=4)
        d = o.log_probs_grad(logits, self.y, r.lse, self.g, entropy=r.entropy, g_entropy=self.h)
        dq, dqt = o.quantize_blocks(d, columns=True)
        dx, dw = o.block_product(dq, wt), o.block_product(dqt, xt)
        self.opt.step([dw])
        return logits, r, d, dx, dw


@pytest.mark.parametrize("N,C,K", [(64, 1000, 300), (33, 515, 129)])
def test_training_step_of_a_layer(N, C, K, ops):
    say("layer", N, C, K)
    layer = Layer(ops, N, C, K, 32)
    w0 = layer.w.clone()
    logits, r, d, dx, dw = layer.step()
    # each stage against 64 bits on what it was given
    xv = ops.quantize_blocks(layer.x)[0].values(torch.float64)
    wv = ops.quantize_blocks(w0, tiles=True)[0].values(torch.float64)
    ref = xv @ wv.t()
    assert (logits.double() - ref).norm() <= (half_step(torch.bfloat16) + 2e-5) * ref.norm()
    check_log_probs(r, logits.cpu(), layer.y.cpu(), 4)
    want, tol = grad_reference(logits.cpu(), layer.y.cpu(), layer.g.cpu(), layer.h.cpu())
    assert torch.all((d.cpu().double() - want).abs() <= 1.01 * tol + half_step(torch.bfloat16) * want.abs() + 1e-40)
    dv, dvt = (t.values(torch.float64) for t in ops.quantize_blocks(d, columns=True))
    xvt = ops.quantize_blocks(layer.x, columns=True)[1].values(torch.float64)
    for got, ref in ((dx, dv @ wv), (dw, dvt @ xvt.t())):
        assert (got.double() - ref).norm() <= (half_step(torch.bfloat16) + 2e-5) * ref.norm()
    # the whole chain's gradient in W against that of the loss in 64 bits at the quantized operands: e4m3 keeps
    # 2^-4 of a value, its subnormals and the shared scales more of the small ones, bf16 2^-8
    lv = (xv @ wv.t()).requires_grad_(True)
    logs = torch.log_softmax(lv, 1)
    t = layer.y
    keep = t >= 0
    loss = -(logs.gather(1, t.clamp(min=0)[:, None])[:, 0][keep].sum() - 0.01 * -(logs.exp() * logs).sum()) / N
    loss.backward()
    full = lv.grad.t() @ xv
    assert (dw.double() - full).norm() <= 2 * 2.0 ** -4 * full.norm()
    # and the step took it
    ref = Plain([C * K], dict(lr=1e-2, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01), 32)
    (w, tol), = ref.step([w0.cpu().double().numpy().reshape(-1)], [dw.float().cpu().numpy().reshape(-1)])
    assert np.all(abs(layer.w.cpu().double().numpy().reshape(-1) - w) <= 1.01 * tol + U * abs(w))


@pytest.mark.parametrize("bits", [32, 8])
def test_layer_step_in_graphs(bits, ops):
    """Two captured steps of two layers, replayed in turn with eager work
    between them, against eager steps of copies."""
    layers = [Layer(ops, 40, 600, 200, bits, seed=s) for s in (1, 2)]
    twins = [Layer(ops, 40, 600, 200, bits, seed=s) for s in (1, 2)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for a in layers:
            a.step()  # the first, eager
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
            graphs[k].replay()
            want = twins[k].step()
            torch.cuda.synchronize()
            for x, y in zip(outs[k][:1] + outs[k][1] + outs[k][2:], want[:1] + want[1] + want[2:]):
                assert torch.equal(x, y), (i, k)
            assert torch.equal(layers[k].w, twins[k].w)
        ops.log_probs(torch.zeros(3, 70000, device="cuda"), top=9)  # other eager work
        if i == 1:
            for o in (layers[0].opt, twins[0].opt):
                o.set_lr(1e-3)
    assert layers[0].opt.steps == twins[0].opt.steps == 5


def test_streams_at_once(ops):
    """Calls on two streams at the same time, one of them named by the argument."""
    x = [torch.randn(200, 40000, generator=gen(s)).cuda() for s in (1, 2)]
    y = torch.zeros(200, dtype=torch.int64, device="cuda")
    want = [ops.log_probs(t, y, top=8) for t in x]
    streams = [torch.cuda.Stream() for _ in x]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        with torch.cuda.stream(streams[0]):
            got[0].append(ops.log_probs(x[0], y, top=8))
        got[1].append(ops.log_probs(x[1], y, top=8, stream=streams[1]))
    a, _ = ops.quantize_blocks(x[0], stream=streams[0].cuda_stream)
    c = ops.block_product(a, a, stream=streams[0].cuda_stream)
    opt = ops.AdamW([x[1]], lr=0.0, weight_decay=0.0)
    opt.step([x[1]], stream=streams[1])
    torch.cuda.synchronize()
    assert opt.steps == 1 and torch.equal(c, ops.block_product(*(ops.quantize_blocks(x[0])[0],) * 2))
    for k in (0, 1):
        for r in got[k]:
            for a, b in zip(r, want[k]):
                assert torch.equal(a, b)


def test_c_entries_refuse_on_the_device(gpu_lib):
    """Scratch that is too small or misaligned, pointers that are not aligned."""
    L = gpu_lib
    x = torch.zeros(2, 100000, device="cuda")
    out = torch.zeros(64, device="cuda")
    ids = torch.zeros(64, dtype=torch.int32, device="cuda")
    need = L.hieravg_log_probs_scratch(2, 100000, 8)
    p = lambda t, o=0: t.data_ptr() + o  # noqa: E731
    if need:
        s = torch.zeros(need + 16, dtype=torch.uint8, device="cuda")
        for ptr, n in ((None, need), (p(s), need - 1), (p(s, 8), need)):
            assert L.hieravg_log_probs(p(x), 0, 2, 100000, 100000, None, 8, 8, None, p(out), p(out, 64), p(ids), p(out, 128),
                                       ptr, n, None) == -1
            assert "scratch" in L.hieravg_last_error().decode()
    assert L.hieravg_log_probs(p(x, 2), 0, 1, 10, 10, None, 8, 0, None, p(out), None, None, None, None, 0, None) == -1
    assert "aligned" in L.hieravg_last_error().decode()
