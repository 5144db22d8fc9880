"""The tensor operators of include/hieravg.h on torch tensors (marshalling
only): log probabilities of labels with entropy and top alternatives and their
gradient, AdamW over many tensors with states in 32 or 8 bits, the norm of many
gradients and their clipping, products of 8-bit floats with a scale for each
block of 128, low-rank adapters of many requests beside such a product, and the
verification of drafted tokens.

Every call enqueues on `stream` (a torch stream or a raw hipStream_t; None:
the tensors' device's current torch stream) and returns without waiting; the
tensors that it makes, scratch among them, are allocated for that stream, as if
it were current.  As with torch's own operations, the caller orders streams
that share tensors.  The operators take no part in autograd: what they return
carries no gradient, also of tensors that require one.  Tensors that a call
writes in place count as modified there, so a backward pass that needs their
earlier values raises.
Bad arguments raise ValueError, errors of the library HierAvgError."""

import ctypes
from array import array
from collections import namedtuple

import torch
from torch.autograd.graph import increment_version

from . import native

TYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}
BLOCK = 128
TOP_MAX = 64

DRAFTS_MAX, RANK_MAX, ADAPTERS_MAX = 64, 128, 8192

LogProbs = namedtuple("LogProbs", "logp entropy lse top_ids top_logp")
GradNorm = namedtuple("GradNorm", "norm factor norms")
AdapterGrads = namedtuple("AdapterGrads", "dx down up")
Verified = namedtuple("Verified", "tokens accepted logp")


def _need(ok, msg):
    if not ok:
        raise ValueError(msg)


_lib = None


def _library():
    global _lib
    _lib = native.lib()
    return _lib


def _device(*tensors):
    """The one GPU that all given tensors are on."""
    dev = tensors[0].device
    for t in tensors:
        if t is not None and t.device != dev:
            raise ValueError("all tensors must be on one GPU")
    if dev.type != "cuda":
        raise ValueError("all tensors must be on one GPU")
    return dev


def _ptr(t):
    return None if t is None else t.data_ptr()


def _as_current(stream, dev):
    """A context in which `stream` is `dev`'s current stream."""
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream, device=dev) if stream else torch.cuda.default_stream(dev)
    _need(stream.device == dev, "the stream must be of the tensors' device")
    return torch.cuda.stream(stream)


def _call(dev, fn, *args):
    """fn(*args, current stream) with `dev` current."""
    index = dev.index
    # torch.cuda.current_stream(dev).cuda_stream without the stream object
    stream = torch._C._cuda_getCurrentRawStream(index)
    if torch._C._cuda_getDevice() == index:
        rc = fn(*args, stream)
    else:
        with torch.cuda.device(dev):
            rc = fn(*args, stream)
    if rc != native.OK:
        native.check(rc)


def _new(rows, cols, dtype, dev):
    """An uninitialised matrix (empty_strided takes the least time on the host)."""
    return torch.empty_strided((rows, cols), (cols, 1), dtype=dtype, device=dev)


def _rows_of(x, name):
    """x as rows: a view of two dimensions, their number and length, and the stride between them."""
    if x.dtype not in TYPES:
        raise ValueError(f"{name} must be float32, float16 or bfloat16")
    if x.dim() != 2:
        _need(x.dim() >= 1 and x.shape[-1] > 0, f"{name} must have a last dimension")
        try:
            x = x.view(-1, x.shape[-1])
        except RuntimeError as e:
            raise ValueError(f"{name} must be viewable as rows (make it contiguous)") from e
    rows, cols = x.shape
    stride, one = x.stride()
    if rows <= 1:
        stride = cols
    if cols == 0 or (one != 1 and cols != 1) or stride < cols:
        raise ValueError(f"rows of {name} must be contiguous, not empty and not overlap")
    return x, rows, cols, stride


def _label_size(labels, shape):
    if (labels.dtype is not torch.int64 and labels.dtype is not torch.int32) or labels.shape != shape \
            or not labels.is_contiguous():
        raise ValueError("labels must be contiguous int64 or int32 of the logits' shape without the last dimension")
    return 8 if labels.dtype is torch.int64 else 4


def _floats(t, shape, name):
    if t is not None and (t.dtype is not torch.float32 or t.shape != shape or not t.is_contiguous()):
        raise ValueError(f"{name} must be contiguous float32 with the logits' shape without the last dimension")


def log_probs(logits, labels=None, top=0, entropy=True, stream=None):
    """LogProbs(logp, entropy, lse, top_ids, top_logp) of each row of logits
    [..., classes]: the log probability of its label (0 for a label below 0),
    the entropy of its distribution, the log of its sum of exponentials, and
    the `top` largest classes (int32, ties to the lowest index) with their log
    probabilities.  What is not asked for is None."""
    if stream is not None:
        with _as_current(stream, _device(logits)):
            return log_probs(logits, labels, top, entropy)
    x, rows, classes, stride = _rows_of(logits, "logits")
    dev = _device(logits, labels)
    shape = logits.shape[:-1]
    if not isinstance(top, int) or not 0 <= top <= TOP_MAX or top > classes:
        raise ValueError(f"top must be in [0, min(classes, {TOP_MAX})]")
    L = _lib or _library()
    size, logp, ent, ids, top_logp, scratch = 0, None, None, None, None, None
    if labels is None:
        lse = torch.empty(shape, dtype=torch.float32, device=dev)
    else:
        size = _label_size(labels, shape)
        lse = torch.empty_like(labels, dtype=torch.float32)
        logp = torch.empty_like(lse)
    if entropy:
        ent = torch.empty_like(lse)
    if top:
        ids = _new(rows, top, torch.int32, dev)
        if logits.dim() != 2:
            ids = ids.view(*shape, top)
        top_logp = torch.empty_like(ids, dtype=torch.float32)
    need = L.hieravg_log_probs_scratch(rows, classes, top)
    if need:
        scratch = _new(1, need, torch.uint8, dev)
    _call(dev, L.hieravg_log_probs, x.data_ptr(), TYPES[x.dtype], rows, classes, stride, _ptr(labels), size,
          top, _ptr(logp), _ptr(ent), lse.data_ptr(), _ptr(ids), _ptr(top_logp), _ptr(scratch), need)
    return LogProbs(logp, ent, lse, ids, top_logp)


def log_probs_grad(logits, labels, lse, g_logp, entropy=None, g_entropy=None, out=None, stream=None):
    """The gradient of sum(g_logp * logp) + sum(g_entropy * entropy) in the
    logits, in their type; lse and entropy as log_probs returned them.  g_logp
    (and labels) or g_entropy may be None.  `out` may be the logits."""
    if stream is not None:
        with _as_current(stream, _device(logits)):
            return log_probs_grad(logits, labels, lse, g_logp, entropy, g_entropy, out)
    x, rows, classes, stride = _rows_of(logits, "logits")
    shape = logits.shape[:-1]
    given = out is not None
    if not given:
        out = o = _new(rows, classes, x.dtype, x.device)
        if logits.dim() != 2:
            out = o.view(logits.shape)
        o_stride = classes
    else:
        o, _, _, o_stride = _rows_of(out, "out")
        _need(out.shape == logits.shape and out.dtype == logits.dtype, "out must have the logits' shape and type")
    dev = _device(logits, labels, lse, g_logp, entropy, g_entropy, out)
    if g_logp is None:
        _need(g_entropy is not None, "g_logp or g_entropy must be given")
    elif labels is None:
        raise ValueError("g_logp needs labels")
    _need(g_entropy is None or entropy is not None, "g_entropy needs entropy")
    _need(lse is not None, "lse must be given")
    _floats(lse, shape, "lse")
    _floats(g_logp, shape, "g_logp")
    _floats(entropy, shape, "entropy")
    _floats(g_entropy, shape, "g_entropy")
    size = 0 if labels is None else _label_size(labels, shape)
    _call(dev, (_lib or _library()).hieravg_log_probs_grad, x.data_ptr(), TYPES[x.dtype], rows, classes, stride,
          _ptr(labels), size, lse.data_ptr(), _ptr(entropy), _ptr(g_logp), _ptr(g_entropy), o.data_ptr(), o_stride)
    if given:
        increment_version(out)
    return out


_ended = []  # handles of closed objects: a capture allows no wait for the device


def _destroy_ended():
    while _ended:
        dev, h = _ended.pop()
        torch.cuda.synchronize(dev)  # steps may still read the handle's tables
        native.lib().hieravg_adamw_destroy(h)


class AdamW:
    """AdamW over a list of tensors, all of them in one step() (see
    include/hieravg.h for the formulas and the layout of the states).

    params: contiguous float32, float16 or bfloat16 tensors on one GPU, stepped
    in place; the object keeps them, and step() refuses one whose memory has
    been replaced (p.data = ...).  copies: None, or a list with a tensor (or None) for each
    that takes the stepped parameter in its own type, as the working copies of
    float32 parameters.  grad_dtype: the type of the gradients (None: each
    parameter's own).  state_bits: 32 or 8.

    m, v: the moments of all tensors in one flat tensor each (float32; with 8
    bits float8_e4m3fn codes and uint8 codes with scale bytes m_scales,
    v_scales), tensor k's from element offsets[k].  One thread steps an object
    at a time, on streams that the caller orders."""

    def __init__(self, params, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, state_bits=32,
                 copies=None, grad_dtype=None, seed=0):
        self._h = None
        params = list(params)
        _need(params, "no parameters")
        copies = [None] * len(params) if copies is None else list(copies)
        _need(len(copies) == len(params), "one copy for each parameter")
        _need(state_bits in (8, 32), "state_bits must be 8 or 32")
        _need(isinstance(seed, int) and 0 <= seed < 1 << 64, "seed must be in [0, 2^64)")
        _need(grad_dtype is None or grad_dtype in TYPES, "grad_dtype must be float32, float16 or bfloat16")
        dev = _device(*params, *copies)
        self.device, self.params, self.copies = dev, params, copies
        table = (native.AdamWTensor * len(params))()
        self.offsets, total = [], 0
        for p, c, t in zip(params, copies, table):
            _need(p.dtype in TYPES and p.is_contiguous(), "parameters must be contiguous floats")
            _need(c is None or (c.dtype in TYPES and c.is_contiguous() and c.shape == p.shape),
                  "a copy must be contiguous floats of its parameter's shape")
            t.param, t.copy, t.n = p.data_ptr(), _ptr(c), p.numel()
            t.param_type, t.copy_type = TYPES[p.dtype], 0 if c is None else TYPES[c.dtype]
            t.grad_type = TYPES[grad_dtype or p.dtype]
            self.offsets.append(total)
            total += -(-p.numel() // BLOCK) * BLOCK
        self._expected = [(p.shape, grad_dtype or p.dtype, p, p.data_ptr(), c, _ptr(c)) for p, c in zip(params, copies)]
        self._written = [t for pair in zip(params, copies) for t in pair if t is not None]
        self.state_bits = state_bits
        self.m_scales = self.v_scales = None
        if state_bits == 32:
            self.m, self.v = (torch.zeros(total, dtype=torch.float32, device=dev) for _ in range(2))
        else:
            self.m = torch.zeros(total, dtype=torch.uint8, device=dev).view(torch.float8_e4m3fn)
            self.v = torch.zeros(total, dtype=torch.uint8, device=dev)
            self.m_scales, self.v_scales = (torch.full((total // BLOCK,), 127, dtype=torch.uint8, device=dev)
                                            for _ in range(2))
        cfg = native.AdamWConfig(lr=lr, beta1=beta1, beta2=beta2, eps=eps, weight_decay=weight_decay, seed=seed,
                                 state_bits=state_bits)
        L = _library()
        _destroy_ended()
        with torch.cuda.device(dev):
            self._h = L.hieravg_adamw_create(ctypes.byref(cfg), table, len(params), self.m.data_ptr(),
                                             self.v.data_ptr(), _ptr(self.m_scales), _ptr(self.v_scales))
        if not self._h:
            raise native.HierAvgError(L.hieravg_last_error().decode())
        self._grads = (ctypes.c_void_p * len(params))()

    def close(self):
        h = getattr(self, "_h", None)
        if h:
            self._h = None
            _ended.append((self.device, h))
        if _ended and not torch.cuda.is_current_stream_capturing():
            _destroy_ended()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __reduce_ex__(self, protocol):
        """A copy would free the same tables again."""
        raise TypeError("an AdamW object can be neither copied nor pickled: make another and load state() into it")

    def step(self, grads, stream=None, factor=None):
        """One step of every tensor on its gradient (None: that tensor stays;
        the step counts all the same) times `factor`, a float32 tensor of one
        element as grad_norm returns it."""
        if stream is not None:
            with _as_current(stream, self.device):
                return self.step(grads, factor=factor)
        if len(grads) != len(self.params):
            raise ValueError("one gradient for each parameter")
        dev, ptrs = self.device, self._grads
        k, stay = 0, False
        for g, (shape, t, p, place, c, c_place) in zip(grads, self._expected):
            if g is None:
                ptrs[k], stay = None, True
            elif g.dtype is t and g.shape == shape and g.device == dev and g.is_contiguous():
                ptrs[k] = g.data_ptr()
                if p.data_ptr() != place or (c is not None and c.data_ptr() != c_place):
                    raise ValueError(f"parameter {k} or its copy has other memory than when this object was made")
            else:
                raise ValueError(f"gradient {k} must be a contiguous {t} tensor of its parameter's shape and device")
            k += 1
        if factor is None:
            _call(dev, _lib.hieravg_adamw_step, self._h, ptrs)
        else:
            _need(factor.dtype is torch.float32 and factor.numel() == 1 and factor.device == dev,
                  "factor must be a float32 tensor of one element on the parameters' device")
            _call(dev, _lib.hieravg_adamw_step_scaled, self._h, ptrs, factor.data_ptr())
        increment_version([t for g, e in zip(grads, self._expected) if g is not None for t in (e[2], e[4]) if t is not None]
                          if stay else self._written)

    def set_lr(self, lr, stream=None):
        """Step size of the steps that follow on the stream."""
        if stream is not None:
            with _as_current(stream, self.device):
                return self.set_lr(lr)
        _call(self.device, _lib.hieravg_adamw_set_lr, self._h, lr)

    def set_step_count(self, t, stream=None):
        """Steps taken so far: the next is t + 1 (a resumed run)."""
        if stream is not None:
            with _as_current(stream, self.device):
                return self.set_step_count(t)
        _call(self.device, _lib.hieravg_adamw_set_steps, self._h, t)

    @property
    def steps(self):
        with torch.cuda.device(self.device):
            t = int(native.lib().hieravg_adamw_steps(self._h))
        if t < 0:
            native.check(t)
        return t

    @property
    def lr(self):
        """The step size set last (waits for the device, like steps)."""
        lr = ctypes.c_double()
        with torch.cuda.device(self.device):
            native.check(native.lib().hieravg_adamw_lr(self._h, ctypes.byref(lr)))
        return lr.value

    def state(self):
        """Moments (the tensors themselves), step count and step size, for a checkpoint."""
        return {"m": self.m, "v": self.v, "m_scales": self.m_scales, "v_scales": self.v_scales, "steps": self.steps,
                "lr": self.lr}

    def load_state(self, st):
        """Resume from state() of an object with the same tensors, bits, betas, eps, weight decay and seed."""
        for k in ("m", "v", "m_scales", "v_scales"):
            mine, other = getattr(self, k), st[k]
            _need((mine is None) == (other is None) and (mine is None or (mine.shape == other.shape
                                                                          and mine.dtype == other.dtype)),
                  f"{k} does not fit this object")
        for k in ("m", "v", "m_scales", "v_scales"):
            if getattr(self, k) is not None:
                getattr(self, k).copy_(st[k])
        self.set_step_count(int(st["steps"]))
        if "lr" in st:
            self.set_lr(st["lr"])


class BlockTensor:
    """A rows x cols matrix in 8-bit floats with a scale for each block of 128
    along its rows: codes [rows, cols rounded up to 128] (float8_e4m3fn),
    scales [rows, or rows / 128 with tiles; blocks rounded up to 4] (uint8,
    2^(byte - 127))."""

    __slots__ = ("codes", "scales", "rows", "cols", "tiles")

    def __init__(self, codes, scales, rows, cols, tiles=False):
        pitch, blocks, spitch = block_shape(rows, cols, tiles)
        _need(codes.dtype == torch.float8_e4m3fn and codes.shape == (rows, pitch) and codes.is_contiguous(),
              f"codes must be contiguous float8_e4m3fn [{rows}, {pitch}]")
        _need(scales.dtype == torch.uint8 and scales.shape == (blocks, spitch) and scales.is_contiguous(),
              f"scales must be contiguous uint8 [{blocks}, {spitch}]")
        self.codes, self.scales, self.rows, self.cols, self.tiles = codes, scales, rows, cols, bool(tiles)

    def values(self, dtype=torch.float32):
        """The matrix [rows, cols] that the codes and scales stand for."""
        byte = self.scales.to(torch.int32)
        bits = torch.where(byte == 0, 1 << 22, torch.where(byte == 255, 0x7FC00000, byte << 23))
        s = bits.view(torch.float32).to(dtype)
        if self.tiles:
            s = s.repeat_interleave(BLOCK, 0)[:self.rows]
        s = s.repeat_interleave(BLOCK, 1)[:, :self.codes.shape[1]]
        return (self.codes.to(dtype) * s)[:, :self.cols]


def block_shape(rows, cols, tiles=False):
    """(code pitch, rows of scales, scale pitch) of a rows x cols block form."""
    blocks = -(-cols // BLOCK)
    return blocks * BLOCK, -(-rows // BLOCK) if tiles else rows, -(-blocks // 4) * 4


def _new_blocks(rows, cols, tiles, dev):
    pitch, blocks, spitch = block_shape(rows, cols, tiles)
    t = BlockTensor.__new__(BlockTensor)
    t.codes = _new(rows, pitch, torch.float8_e4m3fn, dev)
    t.scales = _new(blocks, spitch, torch.uint8, dev)
    t.rows, t.cols, t.tiles = rows, cols, tiles
    return t


def quantize_blocks(x, tiles=False, rows=True, columns=False, stream=None):
    """The block form of x [..., K] as a matrix of rows (`rows`) and that of
    its transpose (`columns`), as a pair with None for what is not asked for.
    tiles: 128 x 128 blocks (weights), else 1 x 128 (activations, gradients)."""
    if stream is not None:
        with _as_current(stream, _device(x)):
            return quantize_blocks(x, tiles, rows, columns)
    if not (rows or columns):
        raise ValueError("rows or columns must be asked for")
    x, R, K, stride = _rows_of(x, "x")
    dev = _device(x)
    if R == 0:
        raise ValueError("x has no rows")
    tiles = bool(tiles)
    a = t = ac = asc = tc = tsc = None
    if rows:
        a = _new_blocks(R, K, tiles, dev)
        ac, asc = a.codes.data_ptr(), a.scales.data_ptr()
    if columns:
        t = _new_blocks(K, R, tiles, dev)
        tc, tsc = t.codes.data_ptr(), t.scales.data_ptr()
    _call(dev, (_lib or _library()).hieravg_quantize_blocks, x.data_ptr(), TYPES[x.dtype], R, K, stride, tiles,
          ac, asc, tc, tsc)
    return a, t


def block_product(a, b, dtype=torch.bfloat16, out=None, stream=None):
    """a b^T of two BlockTensors with the same cols, [a.rows, b.rows] in
    float16 or bfloat16 (dtype, or that of `out`)."""
    if stream is not None:
        with _as_current(stream, _device(a.codes)):
            return block_product(a, b, dtype, out)
    m, n, k = a.rows, b.rows, a.cols
    if b.cols != k:
        raise ValueError("a and b must have the same cols")
    dev = _device(a.codes, a.scales, b.codes, b.scales, out)
    given = out is not None
    if not given:
        if dtype is not torch.bfloat16 and dtype is not torch.float16:
            raise ValueError("a product is float16 or bfloat16")
        out, ldo = _new(m, n, dtype, dev), n
    else:
        _need(out.dtype in (torch.float16, torch.bfloat16), "a product is float16 or bfloat16")
        _need(out.shape == (m, n), "out must be [a.rows, b.rows]")
        ldo = _rows_of(out, "out")[3]
    L = _lib or _library()
    need = L.hieravg_block_product_scratch(m, n, k)
    scratch = _new(1, need, torch.uint8, dev) if need else None
    _call(dev, L.hieravg_block_product, a.codes.data_ptr(), a.scales.data_ptr(), a.tiles, b.codes.data_ptr(),
          b.scales.data_ptr(), b.tiles, m, n, k, out.data_ptr(), TYPES[out.dtype], ldo, _ptr(scratch), need)
    if given:
        increment_version(out)
    return out


def _table_of(grads, what="gradients"):
    """(their one GPU, the library's table) of a list of tensors, None for one that is absent."""
    dev = next((g.device for g in grads if g is not None), None)
    if dev is None or dev.type != "cuda":
        raise ValueError(f"{what} must be tensors on one GPU, one at least")
    index, words = dev.index, []  # three for each tensor, as hieravg_tensor lies in memory
    for g in grads:
        if g is None:
            words += (0, 0, 0)
        else:
            t = TYPES.get(g.dtype)
            if t is None or g.get_device() != index or not g.is_contiguous():
                raise ValueError(f"{what} must be contiguous float32, float16 or bfloat16 tensors on one GPU")
            words += (g.data_ptr(), g.numel(), t)
    return dev, array("q", words)


def _device_of(tensors):
    return next((t.device for t in tensors if t is not None), torch.device("cpu"))


def grad_norm(grads, max_norm=None, stream=None):
    """GradNorm(norm, factor, norms) of a list of gradients (None: absent): the
    norm of all of them together, the factor min(1, max_norm / norm) that
    brings it to max_norm at most (1 without one), and the norm of each, as
    float32 tensors, off by 3 2^-24 at most: squares are added in float32 by
    eights, their sums in 64 bits.  AdamW.step takes the factor."""
    grads = list(grads)
    if stream is not None:
        with _as_current(stream, _device_of(grads)):
            return grad_norm(grads, max_norm)
    most = float("inf") if max_norm is None else float(max_norm)
    if not most >= 0.0:
        raise ValueError("max_norm must be >= 0")
    return _grad_norm(*_table_of(grads), len(grads), most)


def _grad_norm(dev, table, count, most):
    norms = torch.empty_strided((count,), (1,), dtype=torch.float32, device=dev)
    norm = torch.empty_strided((), (), dtype=torch.float32, device=dev)
    factor = torch.empty_strided((), (), dtype=torch.float32, device=dev)
    L = _lib or _library()
    at = table.buffer_info()[0]
    need = L.hieravg_grad_norm_scratch(at, count)
    scratch = _new(1, need, torch.uint8, dev)
    _call(dev, L.hieravg_grad_norm, at, count, most, norms.data_ptr(), norm.data_ptr(), factor.data_ptr(),
          scratch.data_ptr(), need)
    return GradNorm(norm, factor, norms)


def clip_grads(grads, max_norm, out=None, stream=None):
    """Scales a list of gradients (None: absent) so that the norm of all of them
    together is max_norm at most, in place or into the tensors of `out`, and
    returns their GradNorm before that."""
    grads = list(grads)
    if stream is not None:
        with _as_current(stream, _device_of(grads)):
            return clip_grads(grads, max_norm, out)
    most = float(max_norm)
    if not most >= 0.0:
        raise ValueError("max_norm must be >= 0")
    dev, table = _table_of(grads)
    to = grads if out is None else list(out)
    if out is not None:
        if len(to) != len(grads):
            raise ValueError("one result for each gradient")
        index = dev.index
        for g, o in zip(grads, to):
            if g is not None and (o is None or o.dtype is not g.dtype or o.shape != g.shape or o.get_device() != index
                                  or not o.is_contiguous()):
                raise ValueError("a result must be a contiguous tensor of its gradient's shape, type and device")
    ptrs = array("q", [0 if g is None else o.data_ptr() for g, o in zip(grads, to)])
    r = _grad_norm(dev, table, len(grads), most)
    _call(dev, _lib.hieravg_scale_tensors, table.buffer_info()[0], ptrs.buffer_info()[0], len(to), r.factor.data_ptr())
    increment_version([o for g, o in zip(grads, to) if g is not None])
    return r


def _index_size(t, shape, what):
    if (t.dtype is not torch.int64 and t.dtype is not torch.int32) or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous int64 or int32 of shape {list(shape)}")
    return 8 if t.dtype is torch.int64 else 4


def _adapters(down, up, scales):
    """The library's table of adapters, and its in, out and rank."""
    if down.dim() != 3 or up.dim() != 3:
        raise ValueError("down must be [n, rank, in], up [n, rank, out]")
    n, rank, k = down.shape
    n_up, rank_up, cols = up.shape
    if n_up != n or rank_up != rank:
        raise ValueError("down must be [n, rank, in], up [n, rank, out]")
    dtype = down.dtype
    if dtype not in TYPES or up.dtype is not dtype or not down.is_contiguous() or not up.is_contiguous():
        raise ValueError("down and up must be contiguous floats of one type")
    if not (1 <= n <= ADAPTERS_MAX and 1 <= rank <= RANK_MAX and k > 0 and cols > 0):
        raise ValueError(f"down and up must have 1 to {ADAPTERS_MAX} adapters of 1 to {RANK_MAX} ranks, in and out above 0")
    if scales is not None and (scales.dtype is not torch.float32 or scales.dim() != 1 or len(scales) != n
                               or not scales.is_contiguous()):
        raise ValueError("scales must be contiguous float32 [n]")
    return native.Adapters(down.data_ptr(), up.data_ptr(), _ptr(scales), k, cols, n, rank, TYPES[dtype]), k, cols, rank


def _matrix(t, dtype, shape, name):
    """t as rows of `shape`'s last dimension: (view, stride)."""
    if t.dtype is not dtype or t.shape != shape:
        raise ValueError(f"{name} must be {dtype} {list(shape)}")
    t, _, _, stride = _rows_of(t, name)
    return t, stride


def adapter_product(x, ids, down, up, scales=None, base=None, out=None, dtype=None, hidden=False, stream=None):
    """base + s (x down^T) up of each row's adapter: x [..., in], ids [...]
    (int32 or int64; below 0: a row without an adapter, which gets base), down
    [n, rank, in] and up [n, rank, out] (both with the rank outermost, of x's type),
    scales float32 [n] or None (1), base [..., out] or None (0).  The result is
    in the type of `out`, or base, or `dtype` (None: x's); `out` may be base.
    hidden: also h = x down^T, float32 [..., rank], as a pair.  A row whose id
    is not below n gets NaN."""
    if stream is not None:
        with _as_current(stream, _device(x)):
            return adapter_product(x, ids, down, up, scales, base, out, dtype, hidden)
    w, k, cols, rank = _adapters(down, up, scales)
    xr, rows, K, x_stride = _rows_of(x, "x")
    if K != k or xr.dtype is not down.dtype:
        raise ValueError("x must be [..., in] of the adapters' type")
    lead = x.shape[:-1]
    size = _index_size(ids, lead, "ids")
    shape = (*lead, cols)
    dev = _device(x, ids, down, up, scales, base, out)
    given = out is not None
    if given:
        dtype = out.dtype
    elif base is not None:
        dtype = base.dtype
    elif dtype is None:
        dtype = x.dtype
    if dtype not in TYPES or not (dtype is torch.float32 or x.dtype is torch.float32 or dtype is x.dtype):
        raise ValueError("a result must be float32, of x's type, or any float beside float32")
    base_ptr, base_stride, o_stride = None, cols, cols
    if base is not None:
        b, base_stride = _matrix(base, dtype, shape, "base")
        base_ptr = b.data_ptr()
    if given:
        o, o_stride = _matrix(out, dtype, shape, "out")
    else:
        out = o = _new(rows, cols, dtype, dev)
        if x.dim() != 2:
            out = o.view(shape)
    h = torch.empty((*lead, rank), dtype=torch.float32, device=dev) if hidden else None
    if rows:
        L = _lib or _library()
        need = L.hieravg_adapter_product_scratch(rows, w)
        scratch = _new(1, need, torch.uint8, dev) if need else None
        _call(dev, L.hieravg_adapter_product, w, xr.data_ptr(), rows, x_stride, ids.data_ptr(), size, base_ptr, base_stride,
              o.data_ptr(), TYPES[dtype], o_stride, _ptr(h), _ptr(scratch), need)
        if given:
            increment_version(out)
    return (out, h) if hidden else out


def adapter_product_grad(grad, x, ids, down, up, scales=None, hidden=None, base=None, out=None, dx=True, weights=True,
                         grad_dtype=torch.float32, stream=None):
    """AdapterGrads(dx, down, up): the gradients of sum(grad * adapter_product(x, ...))
    in x (plus base, the gradient through the shared projection), down and up.
    hidden: what adapter_product returned as such, which saves a reading of x;
    dx is in the type of `out`, or base, or x's (`out` may be base), and None with
    dx=False; down and up are in grad_dtype, zeros for adapters without rows,
    and None with weights=False."""
    if stream is not None:
        with _as_current(stream, _device(grad)):
            return adapter_product_grad(grad, x, ids, down, up, scales, hidden, base, out, dx, weights, grad_dtype)
    w, k, cols, rank = _adapters(down, up, scales)
    xr, rows, K, x_stride = _rows_of(x, "x")
    if K != k or xr.dtype is not down.dtype:
        raise ValueError("x must be [..., in] of the adapters' type")
    size = _index_size(ids, x.shape[:-1], "ids")
    g, g_stride = _matrix(grad, down.dtype, (*x.shape[:-1], cols), "grad")
    if not (dx or weights):
        raise ValueError("dx or weights must be asked for")
    if not dx and (base is not None or out is not None):
        raise ValueError("base and out are of dx")
    if grad_dtype not in TYPES:
        raise ValueError("grad_dtype must be float32, float16 or bfloat16")
    if hidden is not None and (hidden.dtype is not torch.float32 or hidden.shape != (*x.shape[:-1], rank)
                               or not hidden.is_contiguous()):
        raise ValueError("hidden must be contiguous float32 [..., rank]")
    dev = _device(grad, x, ids, down, up, scales, hidden, base, out)
    given = out is not None
    dtype = out.dtype if given else base.dtype if base is not None else x.dtype
    if dtype not in TYPES or not (dtype is torch.float32 or x.dtype is torch.float32 or dtype is x.dtype):
        raise ValueError("dx must be float32, of x's type, or any float beside float32")
    base_ptr, base_stride, o, o_stride = None, K, None, K
    if base is not None:
        b, base_stride = _matrix(base, dtype, x.shape, "base")
        base_ptr = b.data_ptr()
    if given:
        o, o_stride = _matrix(out, dtype, x.shape, "out")
    elif dx:
        out = o = _new(rows, K, dtype, dev)
        if x.dim() != 2:
            out = o.view(x.shape)
    dd = du = None
    if weights:
        make = torch.empty if rows else torch.zeros
        dd, du = make(down.shape, dtype=grad_dtype, device=dev), make(up.shape, dtype=grad_dtype, device=dev)
    if rows:
        L = _lib or _library()
        need = L.hieravg_adapter_grad_scratch(rows, w, hidden is not None) if weights else L.hieravg_adapter_dx_scratch(rows, w)
        scratch = _new(1, need, torch.uint8, dev) if need else None
        _call(dev, L.hieravg_adapter_grad, w, g.data_ptr(), rows, g_stride, xr.data_ptr(), x_stride, ids.data_ptr(), size,
              _ptr(hidden), base_ptr, base_stride, _ptr(o), TYPES[dtype], o_stride, _ptr(dd), _ptr(du), TYPES[grad_dtype],
              _ptr(scratch), need)
        if given:
            increment_version(out)
    return AdapterGrads(out if dx else None, dd, du)


def verify_drafts(logits, drafts, uniforms, draft_logits=None, lengths=None, temperature=None, stream=None):
    """Verified(tokens, accepted, logp) of drafted tokens [sequences, drafts]
    (int32 or int64) against a target's logits [sequences, drafts + 1, classes], from
    uniform numbers in [0, 1) [sequences, drafts + 1] (float32; the last of a
    sequence draws its token): see hieravg_verify_drafts in include/hieravg.h.
    draft_logits [sequences, drafts, classes]: what the drafts were drawn from
    (None: certain ones); lengths int32 [sequences]: how many drafts there are;
    temperature float32 [sequences] (None: 1; 0: the largest class).
    tokens int32 [sequences, drafts + 1]: the accepted drafts, the drawn token
    and -1 behind; accepted int32 [sequences]; logp float32 like tokens, of
    accepted drafts from float32 sums, off by (classes / 256 + 110) 2^-24 at most.
    Rows of both logits must be viewable as one matrix (a slice of the drafts of
    a wider batch is not: make it contiguous)."""
    if stream is not None:
        with _as_current(stream, _device(logits)):
            return verify_drafts(logits, drafts, uniforms, draft_logits, lengths, temperature)
    if logits.dim() != 3 or drafts.dim() != 2 or logits.shape[1] < 1:
        raise ValueError("logits must be [sequences, drafts + 1, classes], drafts [sequences, drafts]")
    seqs, count, classes = logits.shape
    n = count - 1
    if n > DRAFTS_MAX:
        raise ValueError(f"at most {DRAFTS_MAX} drafts")
    x, _, _, stride = _rows_of(logits.flatten(0, 1) if seqs == 0 else logits, "logits")
    size = _index_size(drafts, (seqs, n), "drafts")
    if uniforms.dtype is not torch.float32 or uniforms.shape != (seqs, n + 1) or not uniforms.is_contiguous():
        raise ValueError("uniforms must be contiguous float32 [sequences, drafts + 1]")
    if lengths is not None and (lengths.dtype is not torch.int32 or lengths.shape != (seqs,) or not lengths.is_contiguous()):
        raise ValueError("lengths must be contiguous int32 [sequences]")
    if temperature is not None and (temperature.dtype is not torch.float32 or temperature.shape != (seqs,)
                                    or not temperature.is_contiguous()):
        raise ValueError("temperature must be contiguous float32 [sequences]")
    dev = _device(logits, drafts, uniforms, draft_logits, lengths, temperature)
    q_ptr, q_type, q_stride = None, 0, classes
    if draft_logits is not None:
        if draft_logits.shape != (seqs, n, classes):
            raise ValueError("draft_logits must be [sequences, drafts, classes]")
        if draft_logits.dtype not in TYPES:
            raise ValueError("draft_logits must be float32, float16 or bfloat16")
        if draft_logits.numel():
            q, _, _, q_stride = _rows_of(draft_logits, "draft_logits")
            q_ptr, q_type = q.data_ptr(), TYPES[q.dtype]
    tokens = _new(seqs, n + 1, torch.int32, dev)
    logp = _new(seqs, n + 1, torch.float32, dev)
    accepted = torch.empty_strided((seqs,), (1,), dtype=torch.int32, device=dev)
    if seqs:
        L = _lib or _library()
        need = L.hieravg_verify_drafts_scratch(seqs, n, classes, q_ptr is not None)
        scratch = _new(1, need, torch.uint8, dev)
        _call(dev, L.hieravg_verify_drafts, x.data_ptr(), TYPES[x.dtype], seqs, n, classes, stride, q_ptr, q_type, q_stride,
              drafts.data_ptr(), size, uniforms.data_ptr(), _ptr(lengths), _ptr(temperature), tokens.data_ptr(),
              accepted.data_ptr(), logp.data_ptr(), scratch.data_ptr(), need)
    return Verified(tokens, accepted, logp)
