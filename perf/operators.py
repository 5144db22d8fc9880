"""What the performance of the tensor operators is measured on: log
probabilities of labels with entropy and top alternatives and their gradient,
the AdamW step over many tensors with states in 32 or 8 bits, and products of
8-bit floats with a scale for each block of 128.

A pass is one call as a training or serving program makes it.  `own` selects
the package's operators; otherwise the same results come from elementary
torch operations in float32.
"""

import math

import torch

own = False

DEV = "cuda"
DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BLOCK = 128


def listed():
    return [
        # One token's logits over a vocabulary, twenty alternatives: sampling
        # with reported alternatives.  The smallest call.
        dict(op="log_probs", rows=1, classes=32000, dtype="f32", top=20, pad=0, masked=0.0, name="log_probs_token"),
        # The head of the 1000-class MLP over the minibatches of 16 learners.
        dict(op="log_probs", rows=512, classes=1000, dtype="f32", top=5, pad=0, masked=0.0, name="log_probs_512x1000"),
        # An odd vocabulary in rows of a wider buffer, a tenth of the classes
        # masked, padded rows without a label.
        dict(op="log_probs", rows=300, classes=50001, dtype="f16", top=1, pad=7, masked=0.1, name="log_probs_ragged"),
        # A training batch of tokens over a large vocabulary.
        dict(op="log_probs", rows=2048, classes=131072, dtype="bf16", top=20, pad=0, masked=0.0,
             name="log_probs_batch"),
        # The gradient of the same batch, with the entropy's.
        dict(op="log_probs_grad", rows=2048, classes=131072, dtype="bf16", pad=0, masked=0.0, ent=True,
             name="log_probs_grad_batch"),
        # The gradient of the 1000-class head.
        dict(op="log_probs_grad", rows=512, classes=1000, dtype="f32", pad=0, masked=0.0, ent=False,
             name="log_probs_grad_512x1000"),
        # The four tensors of a 1000-300-37 MLP: a small model, where the
        # launch is the time.
        dict(op="adamw", layers="1000x300x37", copies=1, param="f32", grad="f32", bits=32, copy=False, decay=0.01,
             name="adamw_1000_300_37"),
        # The 155 million parameters of the 150528-1024-1000 MLP.
        dict(op="adamw", layers="150528x1024x1000", copies=1, param="f32", grad="f32", bits=32, copy=False,
             decay=0.01, name="adamw_150528_1024_1000"),
        # Sixteen learners of a 4097-1001-10 MLP (64 tensors of odd sizes),
        # states in 8 bits, bf16 gradients and bf16 working copies.
        dict(op="adamw", layers="4097x1001x10", copies=16, param="f32", grad="bf16", bits=8, copy=True, decay=0.1,
             name="adamw_8bit_16_learners"),
        # One token through a wide layer: the weights' bytes are the time.
        dict(op="linear", m=1, n=16384, k=4096, dtype="bf16", name="linear_token"),
        # A large batch through a square layer: the matrix rate is the time.
        dict(op="linear", m=8192, n=8192, k=8192, dtype="bf16", name="linear_8192"),
        # Both gradients of the first layer of the 150528-1024-1000 MLP over
        # 16 minibatches of 32: a short contraction and a long one.
        dict(op="linear_grad", m=512, n=1024, k=150528, dtype="bf16", name="linear_grad_150528_1024"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["log_probs", "log_probs", "log_probs_grad", "adamw", "adamw", "linear", "linear", "linear_grad"])
    if op.startswith("log_probs"):
        classes = _log(rng, 10, 131072)
        rows = min(_log(rng, 1, 4096), max(1, 200_000_000 // classes))
        c = dict(op=op, rows=rows, classes=classes, dtype=rng.choice(["f32", "bf16", "bf16", "f16"]),
                 pad=rng.choice([0, 0, rng.randint(1, 70)]), masked=rng.choice([0.0, 0.0, 0.3, 0.9]))
        if op == "log_probs":
            c["top"] = min(classes, rng.choice([0, 1, 5, 20, 64, rng.randint(0, 64)]))
        else:
            c["ent"] = rng.random() < 0.5
        return c
    if op == "adamw":
        layers = [_log(rng, 10, 20000), _log(rng, 10, 2000), _log(rng, 2, 1000)]
        size = layers[0] * layers[1] + layers[1] * layers[2]
        copies = min(rng.choice([1, 1, 2, 5, 16, 40]), max(1, 60_000_000 // size))
        param = rng.choice(["f32", "f32", "bf16"])
        return dict(op=op, layers="x".join(map(str, layers)), copies=copies, param=param,
                    grad=rng.choice(["f32", "bf16"]), bits=rng.choice([32, 8]),
                    copy=param == "f32" and rng.random() < 0.4, decay=rng.choice([0.0, 0.01, 0.1]))
    n, k = _log(rng, 16, 20000), _log(rng, 16, 20000)
    m = rng.choice([rng.randint(1, 16), _log(rng, 1, 8192), _log(rng, 1, 8192)])
    while m * n * k > 8192 ** 3 // (1 if op == "linear" else 4):
        m = m // 2 + 1
        n = n // 2 + 1
    return dict(op=op, m=m, n=n, k=k, dtype=rng.choice(["bf16", "bf16", "f32", "f16"]))


# ------------------------------------------------------------------ 8-bit blocks
def _up(n, m):
    return -(-n // m) * m


def _power(e, dtype):
    """2^e from its bits, -126 <= e <= 127."""
    if dtype == torch.float64:
        return ((e.to(torch.int64) + 1023) << 52).view(dtype)
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _ldexp(x, e):
    """x * 2^e (torch.ldexp takes its power from pow, which is not exact)."""
    half = e >> 1
    return x * _power(half, x.dtype) * _power(e - half, x.dtype)


def _scale_exponents(amax):
    """The least integers e with amax <= 448 * 2^e (0 for amax = 0), in [-127, 127]."""
    f, x = torch.frexp(amax)
    e = x - 9 + (f > 0.875).to(x.dtype)
    return torch.where(amax > 0, e, torch.zeros_like(e)).clamp(-127, 127)


def _quantize(x, rows_per_block):
    """x [R, K] as the values of its 8-bit floats [R, Kp] and the exponents of
    their blocks [ceil(R / rows_per_block), Kp / 128]; Kp is K rounded up to 128."""
    R, K = x.shape
    Rp, Kp = _up(R, rows_per_block), _up(K, BLOCK)
    x = torch.nn.functional.pad(x.float(), (0, Kp - K, 0, Rp - R))
    x = x.view(Rp // rows_per_block, rows_per_block, Kp // BLOCK, BLOCK)
    e = _scale_exponents(x.abs().amax(dim=(1, 3)))
    q = _ldexp(x, -e[:, None, :, None]).to(torch.float8_e4m3fn)
    return q.view(Rp, Kp)[:R], e


def _values(q, e, rows_per_block, dtype=torch.float32):
    """The values that the codes and their blocks' exponents stand for."""
    R, Kp = q.shape
    Rp = _up(R, rows_per_block)
    v = torch.nn.functional.pad(q.to(dtype), (0, 0, 0, Rp - R)).view(-1, rows_per_block, Kp // BLOCK, BLOCK)
    return _ldexp(v, e[:, None, :, None]).view(Rp, Kp)[:R]



def _as_scales(e):
    """Scale bytes [blocks, K blocks rounded up to 4] of the exponents."""
    s = torch.zeros(e.shape[0], _up(e.shape[1], 4), dtype=torch.uint8, device=e.device)
    s[:, :e.shape[1]] = (e + 127).to(torch.uint8)
    return s


# ------------------------------------------------------------------ random rounding
_GOLDEN, _MUL1, _MUL2 = 0x9E3779B97F4A7C15, 0xBF58476D1CE4E5B9, 0x94D049BB133111EB
_MASK = (1 << 64) - 1
_TAG = 0x68762E6164616D77  # "hv.adamw"


def _signed(x):
    x &= _MASK
    return x - (1 << 64) if x >> 63 else x


def _shr(z, n):
    return (z >> n) & ((1 << (64 - n)) - 1)


def _mix(z):
    z = (z ^ _shr(z, 30)) * _signed(_MUL1)
    z = (z ^ _shr(z, 27)) * _signed(_MUL2)
    return z ^ _shr(z, 31)


def _mix_int(z):
    z &= _MASK
    z = ((z ^ (z >> 30)) * _MUL1) & _MASK
    z = ((z ^ (z >> 27)) * _MUL2) & _MASK
    return z ^ (z >> 31)


def _hash_int(key, c):
    return _mix_int(key + (c + 1) * _GOLDEN)


def _draws(seed, step, n):
    """The 32 random bits of elements 0 .. n-1 (n even) of a step: the halves,
    low first, of the SplitMix64 output at each pair's counter."""
    key = _hash_int(_hash_int(seed, _TAG), step)
    c = torch.arange(1, n // 2 + 1, dtype=torch.int64, device=DEV)
    h = _mix(c * _signed(_GOLDEN) + _signed(key))
    return torch.stack((h & 0xFFFFFFFF, _shr(h, 32)), 1).view(-1)


def _round_down(y, u, mantissa, least):
    """y >= 0 on the grid with `mantissa` bits whose normal exponents start at
    `least`, the next value up where the fraction and u pass one."""
    _, x = torch.frexp(y)
    step = torch.clamp(x - 1, min=least) - mantissa
    return _ldexp(torch.floor(_ldexp(y, -step) + u), step)


def _v_values(c, dtype=torch.float32):
    e, f = (c >> 4).to(torch.int32), (c & 15).to(dtype)
    return torch.where(e == 0, _ldexp(f, torch.full_like(e, -18)), _ldexp(f + 16, e - 19))


def _v_codes(y):
    """Codes of values that lie on the grid: 16 exponents, four bits, least step 2^-18."""
    f, x = torch.frexp(y)
    e = torch.clamp(x + 14, min=0)
    fraction = _ldexp(y, 19 - torch.clamp(e, min=1)) - 16 * (e > 0)
    return (e * 16 + fraction.to(torch.int32)).to(torch.uint8)


def _block_exponents(a, top_fraction, top_exponent):
    """The least e with amax <= top * 2^e, top = 2 * top_fraction * 2^top_exponent."""
    amax = a.view(-1, BLOCK).abs().amax(1)
    f, x = torch.frexp(amax)
    e = x - 1 - top_exponent + (f > top_fraction).to(x.dtype)
    return torch.where(amax > 0, e, torch.zeros_like(e)).clamp(-127, 127)


def _spread(e):
    return e[:, None].expand(-1, BLOCK).reshape(-1)


def _pack_moments(m, v, seed, step):
    """The 8-bit states of m and v: codes and scale bytes."""
    r = _draws(seed, step, m.numel())
    um, uv = (r & 0xFFFF).float() / 65536, (r >> 16).float() / 65536
    em, ev = _block_exponents(m, 0.875, 8), _block_exponents(v, 0.96875, 0)
    ym, yv = _ldexp(m, -_spread(em)), _ldexp(v, -_spread(ev))
    qm = torch.copysign(_round_down(ym.abs(), um, 3, -6), m)
    qv = _round_down(yv, uv, 4, -14)
    qv = torch.where((v > 0) & (qv == 0), torch.full_like(qv, 2.0 ** -18), qv)
    return qm.to(torch.float8_e4m3fn), (em + 127).to(torch.uint8), _v_codes(qv), (ev + 127).to(torch.uint8)


def _moments(s, dtype=torch.float32):
    if s["case"]["bits"] == 32:
        return s["m"].to(dtype), s["v"].to(dtype)
    em, ev = (_spread(s[k].to(torch.int32) - 127) for k in ("m_scales", "v_scales"))
    return _ldexp(s["m"].to(dtype), em), _ldexp(_v_values(s["v"], dtype), ev)


# ------------------------------------------------------------------ the states
HYPER = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8)
STEPS = 1000  # steps taken before


def _sizes(case):
    i, h, o = map(int, case["layers"].split("x"))
    return [h * i, h, o * h, o] * case["copies"]


def _randn(g, *shape):
    return torch.randn(*shape, device=DEV, generator=g)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    s = {"case": case}
    dtype = DTYPE[case["dtype"]] if "dtype" in case else None
    if case["op"].startswith("log_probs"):
        rows, classes = case["rows"], case["classes"]
        x = _randn(g, rows, classes + case["pad"]).to(dtype)
        x *= 3
        x = x[:, :classes]
        if case["masked"]:
            # a mask of classes, as a grammar gives one; class 0 stays
            mask = torch.rand(classes, device=DEV, generator=g) < case["masked"]
            mask[0] = False
            x[:, mask] = -math.inf
        labels = torch.randint(0, classes, (rows,), device=DEV, generator=g)
        if case["masked"]:
            labels[mask[labels]] = 0
            if rows > 1:
                labels[::5] = -1
        s.update(logits=x, labels=labels)
        if case["op"] == "log_probs_grad":
            # what the forward left, and the weights of a loss: advantages over the batch
            _, s["entropy"], s["lse"] = _statistics(x, chunk=1 << 26)
            s["g_logp"] = _randn(g, rows) / rows
            s["g_entropy"] = -0.01 * torch.rand(rows, device=DEV, generator=g) / rows if case["ent"] else None
    elif case["op"] == "adamw":
        sizes = _sizes(case)
        starts = [0]
        for n in sizes:
            starts.append(starts[-1] + _up(n, BLOCK))
        total = starts[-1]
        # every tensor starts at a multiple of 128 elements of one buffer
        live = torch.zeros(total, dtype=torch.bool, device=DEV)
        for a, n in zip(starts, sizes):
            live[a:a + n] = True
        grad = _randn(g, total) * 0.01 * live
        m = (0.3 * grad + 0.002 * _randn(g, total)) * live
        v = (grad.square() * 0.5 + 1e-5 * torch.rand(total, device=DEV, generator=g)) * live
        s.update(sizes=sizes, starts=starts, params=(0.05 * _randn(g, total) * live).to(DTYPE[case["param"]]),
                 grads=grad.to(DTYPE[case["grad"]]), steps=STEPS, seed=seed)
        s["copy"] = s["params"].to(torch.bfloat16) if case["copy"] else None
        if case["bits"] == 32:
            s.update(m=m, v=v)
        else:
            s["m"], s["m_scales"], s["v"], s["v_scales"] = _pack_moments(m, v, seed, STEPS)
        if own:
            from paper_1903_05133_amd import operators
            views = lambda t: [t[a:a + n] for a, n in zip(starts, sizes)]  # noqa: E731
            opt = operators.AdamW(views(s["params"]), state_bits=case["bits"], weight_decay=case["decay"], seed=seed,
                                  copies=views(s["copy"]) if case["copy"] else None,
                                  grad_dtype=DTYPE[case["grad"]], **HYPER)
            for k in ("m", "v") + (("m_scales", "v_scales") if case["bits"] == 8 else ()):
                getattr(opt, k).copy_(s[k])
                s[k] = getattr(opt, k)
            opt.set_step_count(STEPS)
            s.update(opt=opt, grad_list=views(s["grads"]))
    else:
        M, N, K = case["m"], case["n"], case["k"]
        w, e = _quantize(_randn(g, N, K) / math.sqrt(K), BLOCK)
        s["x"] = (_randn(g, M, K) * torch.exp(_randn(g, M, 1))).to(dtype)
        # the weights as a program keeps them: 8-bit codes and scale bytes, for
        # the gradient in the transposed form too
        s["w"], s["w_scales"] = w.contiguous(), _as_scales(e)
        if case["op"] == "linear_grad":
            s["dy"] = (_randn(g, M, N) * 1e-3 * torch.exp(_randn(g, M, 1))).to(dtype)
            t = torch.zeros(K, _up(N, BLOCK), dtype=torch.uint8, device=DEV)
            t[:, :N] = w.view(torch.uint8)[:, :K].t()
            s["wt"], s["wt_scales"] = t.view(torch.float8_e4m3fn), _as_scales(e.t())
        if own:
            from paper_1903_05133_amd import operators
            s["W"] = operators.BlockTensor(s["w"], s["w_scales"], N, K, tiles=True)
            if case["op"] == "linear_grad":
                s["WT"] = operators.BlockTensor(s["wt"], s["wt_scales"], K, N, tiles=True)
    return s


# ------------------------------------------------------------------ the plain forms
def _statistics(x, chunk=None):
    """Greatest value, entropy and log of the sum of exponentials of each row."""
    if chunk and x.numel() > chunk:
        step = max(1, chunk // x.shape[1])
        return [torch.cat(p) for p in zip(*(_statistics(x[i:i + step]) for i in range(0, x.shape[0], step)))]
    x = x.float()
    most = x.amax(1, keepdim=True)
    t = x - most
    e = torch.exp(t)
    z = e.sum(1)
    entropy = torch.log(z) - torch.where(e > 0, e * t, torch.zeros_like(e)).sum(1) / z
    return most[:, 0], entropy, most[:, 0] + torch.log(z)


def _top(x, k):
    """Indices of the k greatest of each row, ties to the lowest index."""
    b = (x + 0.0).view(torch.int32)
    order = torch.where(b >= 0, b, b ^ 0x7FFFFFFF).to(torch.int64)
    place = 0xFFFFFFFF - torch.arange(x.shape[1], device=x.device)
    return 0xFFFFFFFF - (torch.topk((order << 32) | place, k, dim=1).values & 0xFFFFFFFF)


def _log_probs(s):
    x, labels, k = s["logits"].float(), s["labels"], s["case"]["top"]
    _, entropy, lse = _statistics(x)
    logp = x.gather(1, labels.clamp(min=0)[:, None])[:, 0] - lse
    out = {"logp": torch.where(labels < 0, torch.zeros_like(logp), logp), "entropy": entropy, "lse": lse}
    if k:
        ids = _top(x, k)
        out.update(top_ids=ids.to(torch.int32), top_logp=x.gather(1, ids) - lse[:, None])
    return out


def _log_probs_grad(s):
    labels, ent = s["labels"], s["g_entropy"]
    logs = s["logits"].float() - s["lse"][:, None]
    p = torch.exp(logs)
    g = torch.where(labels < 0, torch.zeros_like(s["g_logp"]), s["g_logp"])
    d = -g[:, None] * p
    if ent is not None:
        slope = torch.where(p > 0, p * (logs + s["entropy"][:, None]), torch.zeros_like(p))
        d -= ent[:, None] * slope
    d.scatter_add_(1, labels.clamp(min=0)[:, None], g[:, None])
    return {"dlogits": d.to(s["logits"].dtype)}


def _adamw(s):
    c, b1, b2 = s["case"], HYPER["beta1"], HYPER["beta2"]
    s["steps"] += 1
    t = s["steps"]
    g = s["grads"].float()
    m, v = _moments(s)
    m = m * b1 + g * (1 - b1)
    v = v * b2 + g * g * (1 - b2)
    d = m / (1 - b1 ** t) / (torch.sqrt(v) / math.sqrt(1 - b2 ** t) + HYPER["eps"])
    s["params"].copy_(s["params"].float() * (1 - HYPER["lr"] * c["decay"]) - HYPER["lr"] * d)
    if c["copy"]:
        s["copy"].copy_(s["params"])
    new = (m, v) if c["bits"] == 32 else _pack_moments(m, v, s["seed"], t)
    for k, x in zip(("m", "v") if c["bits"] == 32 else ("m", "m_scales", "v", "v_scales"), new):
        s[k].copy_(x)


def _adamw_outputs(s):
    return {k: s[k] for k in ("params", "copy", "m", "v", "m_scales", "v_scales") if s.get(k) is not None}


def _exponents(scales, cols):
    return scales[:, :_up(cols, BLOCK) // BLOCK].to(torch.int32) - 127


def _linear(s):
    x = _values(*_quantize(s["x"], 1), 1)
    w = _values(s["w"], _exponents(s["w_scales"], s["case"]["k"]), BLOCK)
    return {"y": (x @ w.t()).to(torch.bfloat16)}


def _linear_grad(s):
    N, K = s["case"]["n"], s["case"]["k"]
    w = _values(s["w"], _exponents(s["w_scales"], K), BLOCK)[:, :K]
    dy = _values(*_quantize(s["dy"], 1), 1)[:, :N]
    dyt = _values(*_quantize(s["dy"].t(), 1), 1)
    xt = _values(*_quantize(s["x"].t(), 1), 1)
    return {"dx": (dy @ w).to(torch.bfloat16), "dw": (dyt @ xt.t()).to(torch.bfloat16)}


def _run_own(s):
    from paper_1903_05133_amd import operators
    op = s["case"]["op"]
    if op == "log_probs":
        r = operators.log_probs(s["logits"], s["labels"], top=s["case"]["top"], entropy=True)
        return {k: v for k, v in r._asdict().items() if v is not None}
    if op == "log_probs_grad":
        return {"dlogits": operators.log_probs_grad(s["logits"], s["labels"], s["lse"], s["g_logp"],
                                                    entropy=s["entropy"], g_entropy=s["g_entropy"])}
    if op == "adamw":
        s["opt"].step(s["grad_list"])
        return _adamw_outputs(s)
    if op == "linear":
        x, _ = operators.quantize_blocks(s["x"])
        return {"y": operators.block_product(x, s["W"], torch.bfloat16)}
    dy, dyt = operators.quantize_blocks(s["dy"], rows=True, columns=True)
    _, xt = operators.quantize_blocks(s["x"], rows=False, columns=True)
    return {"dx": operators.block_product(dy, s["WT"], torch.bfloat16),
            "dw": operators.block_product(dyt, xt, torch.bfloat16)}


def run(s):
    if own:
        return _run_own(s)
    op = s["case"]["op"]
    if op == "log_probs":
        return _log_probs(s)
    if op == "log_probs_grad":
        return _log_probs_grad(s)
    if op == "adamw":
        _adamw(s)
        return _adamw_outputs(s)
    return _linear(s) if op == "linear" else _linear_grad(s)


# ------------------------------------------------------------------ from the definitions, in 64 bits
def _exact_log_probs(s):
    x, labels = s["logits"], s["labels"]
    k = s["case"].get("top", 0)
    got = {"logp": [], "entropy": [], "lse": [], "top_logp": []}
    step = max(1, (1 << 26) // x.shape[1])
    for i in range(0, x.shape[0], step):
        y, t = x[i:i + step].double(), labels[i:i + step]
        logs = torch.log_softmax(y, 1)
        p = logs.exp()
        got["lse"].append(torch.logsumexp(y, 1))
        got["entropy"].append(-torch.nan_to_num(p * logs, nan=0.0).sum(1))
        got["logp"].append(torch.where(t < 0, 0.0, logs.gather(1, t.clamp(min=0)[:, None])[:, 0]))
        if k:
            got["top_logp"].append(torch.topk(logs, k, dim=1).values)
    return {n: torch.cat(v) if v else None for n, v in got.items()}


def _exact_log_probs_grad(s):
    # the definition at the statistics that the call is given
    x = s["logits"]
    out = torch.empty(x.shape, dtype=torch.float64, device=DEV)
    step = max(1, (1 << 26) // x.shape[1])
    for i in range(0, x.shape[0], step):
        part = slice(i, i + step)
        y, t = x[part].double() - s["lse"][part].double()[:, None], s["labels"][part]
        p = y.exp()
        hot = torch.arange(x.shape[1], device=DEV)[None] == t[:, None]
        g = torch.where(t < 0, 0.0, s["g_logp"][part].double())[:, None]
        d = g * (hot.double() - p)
        if s["g_entropy"] is not None:
            h = s["g_entropy"][part].double()[:, None]
            d -= h * torch.nan_to_num(p * (y + s["entropy"][part].double()[:, None]), nan=0.0)
        out[part] = d
    return {"dlogits": out}


def _exact_adamw(s):
    c = s["case"]
    b1, b2, t = HYPER["beta1"], HYPER["beta2"], s["steps"] + 1
    m, v = _moments(s, torch.float64)
    g = s["grads"].double()
    m1, v1 = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    p = s["params"].double()
    p = p - HYPER["lr"] * (c["decay"] * p + m1 / (1 - b1 ** t) / ((v1 / (1 - b2 ** t)).sqrt() + HYPER["eps"]))
    # the codes of 8-bit states follow the roundings to float32 before them: whole numbers, no values in 64 bits
    return {"params": p, "copy": p if c["copy"] else None, "m": m1 if c["bits"] == 32 else None,
            "v": v1 if c["bits"] == 32 else None, "m_scales": None, "v_scales": None}


def _exact_blocks(x, dim):
    """x in 64 bits as its 8-bit floats stand for it: along `dim`, block by
    block, the nearest multiple of the format's step, ties to even."""
    x = x.double()
    if dim == 0:
        return _exact_blocks(x.t(), 1).t()
    R, K = x.shape
    x = torch.nn.functional.pad(x, (0, _up(K, BLOCK) - K)).view(R, -1, BLOCK)
    a = x.abs().amax(2, keepdim=True)
    e = torch.where(a > 0, torch.ceil(torch.log2(a / 448) - 1e-12), 0.0)
    unit = _power(e, torch.float64)
    y = x / unit
    step = _power(torch.clamp(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -30))), min=-6) - 3, torch.float64)
    return (torch.round(y / step) * step * unit).view(R, -1)[:, :K]


def _exact_weights(s):
    N, K = s["case"]["n"], s["case"]["k"]
    unit = _power(s["w_scales"].to(torch.int64) - 127, torch.float64)
    unit = unit.repeat_interleave(BLOCK, 0)[:N].repeat_interleave(BLOCK, 1)[:, :K]
    return s["w"].double()[:, :K] * unit


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "log_probs":
        return _exact_log_probs(s)
    if case["op"] == "log_probs_grad":
        return _exact_log_probs_grad(s)
    if case["op"] == "adamw":
        return _exact_adamw(s)
    if case["op"] == "linear":
        return {"y": _exact_blocks(s["x"], 1) @ _exact_weights(s).t()}
    return {"dx": _exact_blocks(s["dy"], 1) @ _exact_weights(s),
            "dw": _exact_blocks(s["dy"], 0).t() @ _exact_blocks(s["x"], 0)}


def work(case):
    size = {"f32": 4, "bf16": 2, "f16": 2}
    if case["op"].startswith("log_probs"):
        n = case["rows"] * case["classes"]
        if case["op"] == "log_probs":
            return {"bytes": n * size[case["dtype"]] + case["rows"] * (8 + 12 + 8 * case["top"]), "flops": 6 * n}
        return {"bytes": 2 * n * size[case["dtype"]] + 28 * case["rows"], "flops": 6 * n}
    if case["op"] == "adamw":
        n = sum(_sizes(case))
        each = 2 * size[case["param"]] + size[case["grad"]] + (2 if case["copy"] else 0)
        return {"bytes": n * (each + (16 if case["bits"] == 32 else 4 + 4 / BLOCK)), "flops": 15 * n}
    M, N, K = case["m"], case["n"], case["k"]
    x = size[case["dtype"]]
    if case["op"] == "linear":
        return {"bytes": M * K * x + N * K + 2 * M * N, "flops": 2 * M * N * K}
    return {"bytes": (M * K + M * N) * x + N * K + 2 * (M * K + N * K), "flops": 4 * M * N * K}
