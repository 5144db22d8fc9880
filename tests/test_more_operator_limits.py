"""Low-rank adapters, gradient norms and the verification of drafts at their limits:
many rows and many adapters, values at the ends of their types.  u = 2^-24 is
half a step of float32; tolerances count roundings as in test_more_operators.py."""

import pytest
import torch

from test_more_operators import (INF, TYPES, Adapters, check_verify, float32_by_default, gen, near, on_gpu, ops,  # noqa: F401
                                 plain_verify, say, verify_case)

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


# ------------------------------------------------------------------ adapters
def ids_of(rows, n, kind, seed):
    """Adapters of the rows: of requests one after the other, of single tokens, or most rows of two of them."""
    g = gen(seed)
    mixed = torch.randint(-1, n, (rows,), generator=g)
    if kind == "mixed":
        return mixed
    if kind == "runs":
        starts = torch.zeros(rows, dtype=torch.int64)
        starts[torch.randint(0, rows, (max(1, rows // 150),), generator=g)] = 1
        return mixed[starts.cumsum(0)]
    u = torch.rand(rows, generator=g)
    return torch.where(u < 0.45, n // 2, torch.where(u < 0.9, n - 1, mixed))


# Where a wave of the counting sort has more rows than it holds (1024: past 16384 rows
# of few adapters, past 1024 of 8192), where adapters have several units of rows beside
# others that have one or none, and where a sum has as many units as it may.
LONG = [(16385, 3), (40001, 70), (3000, 8192), (10000, 1000), (4097, 1), (9000, 2)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", ["runs", "mixed", "two"])
@pytest.mark.parametrize("rows,n", LONG)
def test_adapters_of_many_rows(rows, n, kind, dtype, ops):  # noqa: F811
    say("many rows", rows, n, kind, dtype)
    c = Adapters(rows, n, 3, 9, 12, dtype, rows + n, ids=ids_of(rows, n, kind, n))
    dy, x, ids, down, up, scales = on_gpu(c.dy, c.x, c.ids, c.down, c.up, c.scales)
    y, tol, h, th = c.forward(None)
    got, hidden = ops.adapter_product(x, ids, down, up, scales, dtype=torch.float32, hidden=True)
    near(got, y, tol, "y")
    near(hidden, h, th, "hidden")
    for i in (ids, ids.int()):
        r = ops.adapter_product_grad(dy, x, i, down, up, scales, out=torch.empty(rows, 9, device="cuda"))
        for g, (w, t), what in zip(r, c.backward(None), ("dx", "ddown", "dup")):
            near(g, w, t, what)


@pytest.mark.parametrize("dtype", TYPES)
def test_gradient_in_x_alone(dtype, ops):  # noqa: F811
    """The same bits as beside the other gradients, in less scratch; nothing past it is written."""
    from paper_1903_05133_amd import native
    for rows, n, rank, k, cols in ((1, 1, 1, 1, 1), (64, 5, 16, 40, 300), (5000, 3, 33, 260, 129)):
        say("dx alone", rows, n, rank, k, cols, dtype)
        c = Adapters(rows, n, rank, k, cols, dtype, rows)
        dy, x, ids, down, up, scales = on_gpu(c.dy, c.x, c.ids, c.down, c.up, c.scales)
        r = ops.adapter_product_grad(dy, x, ids, down, up, scales)
        assert torch.equal(ops.adapter_product_grad(dy, x, ids, down, up, scales, weights=False).dx, r.dx)
        L, t = native.lib(), ops.TYPES[dtype]
        w = native.Adapters(down.data_ptr(), up.data_ptr(), scales.data_ptr(), k, cols, n, rank, t)
        need = L.hieravg_adapter_dx_scratch(rows, w)
        scratch = torch.full((need + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
        dx = torch.empty_like(x)
        torch.cuda.synchronize()
        assert L.hieravg_adapter_grad(w, dy.data_ptr(), rows, cols, None, k, ids.data_ptr(), 8, None, None, 0, dx.data_ptr(), t, k, None, None,
                                      0, scratch.data_ptr(), need, None) == native.OK
        torch.cuda.synchronize()
        assert torch.equal(dx, r.dx) and torch.all(scratch[need:] == 0x5A)


# ------------------------------------------------------------------ norms
# Squares whose roundings all fall the same way where a chain of additions begins with
# the large one: such a sum of eight would be off by 4.99 u.
EIGHT = [1.0004229545593262, 0.008315023966133595, 0.011211877688765526, 0.011580153368413448, 0.0153886079788208, 0.00106743723154068,
         0.010706060566008091, 0.006982971914112568]


def test_norm_of_squares_that_round_alike(ops):  # noqa: F811
    """Sums of eight squares are off by 4 u at most, so a norm by 2 u and its own rounding: eights as a thread takes
    them, four elements and four 1024 further on, the large one at each place."""
    for swap in range(8):
        e = EIGHT[:]
        e[0], e[swap] = e[swap], e[0]
        e = torch.tensor(e, device="cuda")
        for steps in range(1, 41):
            t = e.view(2, 1, 4).expand(4 * steps, 2, 256, 4).contiguous().view(-1)
            want = t.double().square().sum().sqrt()
            got = ops.grad_norm([t]).norm.double()
            half = torch.finfo(torch.float32).eps / 2 * 2.0 ** torch.floor(torch.log2(want))
            assert torch.all((got - want).abs() <= (2 * U + 1e-12) * want + half), (swap, steps)


@pytest.mark.parametrize("bits", [32, 8])
def test_factor_inside_what_a_step_writes(bits, ops):  # noqa: F811
    p, c = torch.ones(300, device="cuda"), torch.ones(300, device="cuda")
    opt = ops.AdamW([p], copies=[c], state_bits=bits)
    g = torch.ones(300, device="cuda")
    inside = [p[:1], p[299:], c[17:18], opt.v.view(torch.float32)[3:4]]
    if bits == 32:
        inside.append(opt.m[383:])
    for f in inside:
        with pytest.raises(ops.native.HierAvgError, match="factor"):
            opt.step([g], factor=f)
    assert torch.all(p == 1) and opt.steps == 0
    opt.step([g], factor=g[:1])  # a gradient is only read
    assert opt.steps == 1 and torch.all(p < 1)


# ------------------------------------------------------------------ verification of drafts
LEAST = 2.0 ** -149
LOGITS = {
    "masked by the lowest number": (3e38, lambda g, *s: torch.where(torch.rand(*s, generator=g) < 0.3, torch.finfo(torch.float32).min,
                                                                     4 * torch.randn(*s, generator=g))),
    "of the largest size": (3e38, lambda g, *s: 1e38 * torch.randn(*s, generator=g).clamp(-3, 3)),
    "small": (1e-37, lambda g, *s: 1e-37 * torch.randn(*s, generator=g)),
    "subnormal": (2 * LEAST, lambda g, *s: torch.randint(0, 9, s, generator=g).float() * LEAST),
}


@pytest.mark.parametrize("kind", LOGITS)
@pytest.mark.parametrize("B,V", [(40, 300), (24, 3000), (3, 60001)])
def test_verify_at_extreme_temperatures(B, V, kind, ops):  # noqa: F811
    """Logits and temperatures at the ends of float32, whose quotient is an ordinary one: the distributions are
    those of the quotients, which float32 factors do not reach."""
    say("extreme temperatures", B, V, kind)
    t, logits = LOGITS[kind]
    g = gen(V)
    x, q = logits(g, B, 4, V), logits(g, B, 3, V)
    drafts, u = torch.randint(0, V, (B, 3), generator=g), torch.rand(B, 4, generator=g)
    temp = torch.full((B,), t)
    r = ops.verify_drafts(*on_gpu(x, drafts, u), draft_logits=q.cuda(), temperature=temp.cuda())
    want = plain_verify(x, drafts, u, q, None, temp)
    assert sum(want[1]) > 0
    check_verify(r, want, V)
    check_verify(ops.verify_drafts(*on_gpu(x, drafts, u), temperature=temp.cuda()), plain_verify(x, drafts, u, None, None, temp), V)


# Up to 2048 classes in one launch and in several; more than 2048 classes in one
# part of the float32 sums; more sequences than one set of launches takes.
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,G,V", [(1, 64, 512), (1, 64, 513), (2, 19, 1024), (2, 20, 1024), (2, 39, 1000), (3, 9, 2048), (3, 10, 2048),
                                   (1, 64, 2048), (900, 1, 2100), (2100, 1, 2100)])
def test_verify_by_every_launch(B, G, V, dtype, ops):  # noqa: F811
    say("launches", B, G, V, dtype)
    x, q, drafts, u, lengths, t = verify_case(B, G, V, dtype, dtype, B + G + V)
    xg, qg, dg, ug, lg, tg = on_gpu(x, q, drafts, u, lengths, t)
    check_verify(ops.verify_drafts(xg, dg, ug, draft_logits=qg, lengths=lg, temperature=tg), plain_verify(x, drafts, u, q, lengths, t), V)
    check_verify(ops.verify_drafts(xg, dg, ug, draft_logits=qg), plain_verify(x, drafts, u, q, None, None), V)
    check_verify(ops.verify_drafts(xg, dg, ug, temperature=tg), plain_verify(x, drafts, u, None, None, t), V)
