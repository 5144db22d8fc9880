"""Argument checks of the tensor operators' C entries that need no GPU: they
run before any HIP call, so nothing is launched; and the sizes of scratch and
states.  The pointers are ordinary host memory that a refused call never
reads."""

import ctypes

import pytest

from paper_1903_05133_amd import native

BUF = (ctypes.c_double * 64)()
P = -(-ctypes.addressof(BUF) // 16) * 16


def refused(rc, word):
    msg = native.lib().hieravg_last_error().decode()
    assert rc == native.EINVAL and word in msg, (rc, msg)


def lp(x=P, type=0, rows=1, classes=4, stride=4, labels=P, size=8, top=0, logp=P, ids=None, tl=None):
    return native.lib().hieravg_log_probs(x, type, rows, classes, stride, labels, size, top, logp, None, None, ids, tl,
                                          None, 0, None)


@pytest.mark.parametrize("kw,word", [
    (dict(type=3), "type"), (dict(type=-1), "type"), (dict(rows=-1), "rows"), (dict(rows=1 << 31), "rows"),
    (dict(classes=0), "classes"), (dict(classes=(1 << 23) + 1), "classes"), (dict(stride=3), "row_stride"), (dict(x=None), "logits"),
    (dict(x=P + 2), "aligned"), (dict(top=5), "top"), (dict(top=-1), "top"),
    (dict(top=65, classes=100, stride=100), "top"), (dict(top=2), "top_ids"), (dict(size=2), "label_bytes"),
    (dict(labels=None), "labels"), (dict(labels=P + 4), "labels")])
def test_log_probs_refuses(kw, word):
    refused(lp(**kw), word)


def test_no_rows_is_no_call():
    L = native.lib()
    assert lp(rows=0, x=None) == 0
    assert L.hieravg_log_probs_grad(None, 0, 0, 4, 4, None, 8, None, None, None, None, None, 4, None) == 0
    assert L.hieravg_quantize_blocks(None, 0, 0, 4, 4, 0, P, P, None, None, None) == 0
    assert L.hieravg_block_product(None, None, 0, None, None, 0, 0, 5, 4, None, 1, 5, None, 0, None) == 0
    assert L.hieravg_block_product(None, None, 0, None, None, 0, 5, 0, 4, None, 1, 0, None, 0, None) == 0


def grad(x=P, rows=1, classes=4, stride=4, labels=P, size=8, lse=P, ent=P, g=P, h=P, out=P, ostride=4, type=0):
    return native.lib().hieravg_log_probs_grad(x, type, rows, classes, stride, labels, size, lse, ent, g, h, out, ostride,
                                               None)


@pytest.mark.parametrize("kw,word", [
    (dict(type=7), "type"), (dict(ostride=3), "grad_stride"), (dict(out=None), "grad"), (dict(out=P + 1), "grad"),
    (dict(lse=None), "lse"), (dict(g=None, h=None), "both NULL"), (dict(labels=None), "labels"),
    (dict(ent=None), "entropy"), (dict(size=1), "label_bytes"), (dict(x=None), "logits")])
def test_log_probs_grad_refuses(kw, word):
    refused(grad(**kw), word)


def quant(x=P, type=0, rows=1, cols=4, stride=4, tiles=0, c=P, s=P, ct=None, st=None):
    return native.lib().hieravg_quantize_blocks(x, type, rows, cols, stride, tiles, c, s, ct, st, None)


@pytest.mark.parametrize("kw,word", [
    (dict(type=9), "type"), (dict(rows=-1), "rows"), (dict(cols=0), "cols"), (dict(cols=1 << 31), "cols"),
    (dict(stride=3), "row_stride"), (dict(tiles=2), "tiles"), (dict(s=None), "together"), (dict(ct=P), "together"),
    (dict(c=None, s=None), "no block form"), (dict(x=None), "x must"), (dict(c=P + 8), "aligned"),
    (dict(s=P + 2), "aligned")])
def test_quantize_refuses(kw, word):
    refused(quant(**kw), word)


def prod(a=P, sa=P, ta=0, b=P, sb=P, tb=0, m=1, n=4, k=4, out=P, type=2, ldo=4):
    return native.lib().hieravg_block_product(a, sa, ta, b, sb, tb, m, n, k, out, type, ldo, None, 0, None)


@pytest.mark.parametrize("kw,word", [
    (dict(type=0), "out_type"), (dict(m=-1), "m and n"), (dict(n=1 << 31), "m and n"), (dict(k=0), "k in"), (dict(k=(1 << 23) + 1), "k in"),
    (dict(ta=2), "tiles"), (dict(tb=-1), "tiles"), (dict(ldo=3), "out_stride"), (dict(a=None), "NULL"),
    (dict(sb=None), "NULL"), (dict(out=None), "NULL"), (dict(a=P + 4), "aligned"), (dict(sa=P + 1), "aligned"),
    (dict(out=P + 1), "aligned")])
def test_product_refuses(kw, word):
    refused(prod(**kw), word)


@pytest.mark.parametrize("kw", [dict(m=1, n=0x7FFFFF00), dict(m=0x7FFFFF00, n=5), dict(m=0x7FFFFF00, n=300)])
def test_product_refuses_more_than_a_grid(kw):
    refused(prod(ldo=kw["n"], **kw), "too many tiles")


def adamw(n=(4,), m=P, v=P, ms=None, vs=None, param=P, ptype=0, gtype=0, copy=None, ctype=0, count=None, **kw):
    cfg = dict(lr=0.1, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.0, seed=0, state_bits=32)
    cfg.update(kw)
    c = native.AdamWConfig(**cfg)
    t = (native.AdamWTensor * len(n))(*[native.AdamWTensor(param=param, copy=copy, n=k, param_type=ptype, grad_type=gtype,
                                                           copy_type=ctype) for k in n])
    return native.lib().hieravg_adamw_create(ctypes.byref(c), t, len(n) if count is None else count, m, v, ms, vs)


@pytest.mark.parametrize("kw,word", [
    (dict(lr=-1.0), "lr"), (dict(lr=float("inf")), "lr"), (dict(beta1=1.0), "betas"), (dict(beta2=float("nan")), "betas"),
    (dict(eps=0.0), "eps"), (dict(eps=1e-50), "eps"), (dict(weight_decay=-0.1), "weight_decay"),
    (dict(state_bits=16), "state_bits"), (dict(count=0), "no tensors"), (dict(n=(-1,)), "size"), (dict(ptype=5), "type"),
    (dict(gtype=-1), "type"), (dict(copy=P, ctype=4), "type"), (dict(param=None), "parameter"),
    (dict(param=P + 2), "parameter"), (dict(copy=P + 1, ctype=2), "copy"), (dict(m=None), "m and v"),
    (dict(v=P + 8), "m and v"), (dict(state_bits=8), "scales")])
def test_adamw_create_refuses(kw, word):
    assert not adamw(**kw)
    assert word in native.lib().hieravg_last_error().decode()


@pytest.mark.parametrize("kw,word", [
    (dict(eps=1e-40), "eps"), (dict(eps=float("inf")), "eps"), (dict(n=(4, 4)), "overlap"),
    (dict(n=(4, 0, 1)), "overlap"), (dict(copy=P, ctype=2), "overlap"), (dict(copy=P + 12, ctype=0), "overlap"),
    (dict(copy=P - 6, ctype=2), "overlap")])
def test_adamw_refuses_overlap_and_small_eps(kw, word):
    assert not adamw(**kw)
    assert word in native.lib().hieravg_last_error().decode()


def test_adamw_null_handles():
    L = native.lib()
    L.hieravg_adamw_destroy(None)
    refused(L.hieravg_adamw_step(None, P, None), "NULL")
    refused(L.hieravg_adamw_set_lr(None, 0.1, None), "NULL")
    refused(L.hieravg_adamw_set_steps(None, 1, None), "NULL")
    assert L.hieravg_adamw_steps(None) == native.EINVAL
    assert not L.hieravg_adamw_create(None, None, 1, P, P, None, None)


def test_adamw_state_size():
    L = native.lib()
    size = lambda *n: L.hieravg_adamw_state_size((ctypes.c_int64 * len(n))(*n), len(n))  # noqa: E731
    assert size(0) == 0 and size(1) == 128 and size(128, 129, 0, 3) == 128 + 256 + 128
    assert size(1 << 33) == 1 << 33
    assert size(-1) == native.EINVAL and L.hieravg_adamw_state_size(None, 1) == native.EINVAL


def test_structures_match_the_header():
    """The two structures have the header's fields in its order."""
    import os
    import re
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "hieravg.h")).read()
    for name, struct in (("hieravg_adamw_config", native.AdamWConfig), ("hieravg_adamw_tensor", native.AdamWTensor)):
        body = re.sub(r"/\*.*?\*/", "", text[text.index(f"typedef struct {name} {{"):text.index(f"}} {name};")], flags=re.S)
        fields = []
        for line in re.findall(r"^\s*(?:double|uint64_t|int64_t|int32_t|void\s*\*)\s*([\w, ]+);", body, flags=re.M):
            fields += [f.strip() for f in line.split(",")]
        assert fields == [f for f, _ in struct._fields_]


def test_scores_refuses():
    L = native.lib()
    refused(L.hieravg_scores(None, 0, 0, 4, 0, None, P, None, None), "logp or entropy")
    refused(L.hieravg_scores(None, 0, 0, 4, 65, P, P, P, P), "top")
    refused(L.hieravg_scores(None, 0, 0, 4, 2, P, P, None, P), "top_ids")
    refused(L.hieravg_scores(None, 0, 0, 4, 2, P, P, P, P), "NULL handle")
