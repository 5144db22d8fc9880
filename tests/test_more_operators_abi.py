"""Argument checks of the C entries of low-rank adapters, gradient norms and the
verification of drafts that need no GPU: they run before any HIP call, so
nothing is launched, and the pointers are host memory that a refused call never
reads."""

import ctypes
import os
import re

import pytest

from paper_1903_05133_amd import native

BUF = (ctypes.c_double * 512)()
P = -(-ctypes.addressof(BUF) // 64) * 64


def refused(rc, word):
    msg = native.lib().hieravg_last_error().decode()
    assert rc == native.EINVAL and word in msg, (rc, msg)


def tensors(*t):
    return (native.Tensor * len(t))(*[native.Tensor(*x) for x in t]), len(t)


def norm(t=((P, 4, 0),), most=1.0, out=(P, P, P), scratch=P, size=1 << 20, count=None):
    table, n = tensors(*t)
    return native.lib().hieravg_grad_norm(table, n if count is None else count, most, *out, scratch, size, None)


@pytest.mark.parametrize("kw,word", [
    (dict(count=0), "no tensors"), (dict(t=((P, -1, 0),)), "size"), (dict(t=((P, (1 << 40) + 1, 0),)), "size"),
    (dict(t=((P, 4, 3),)), "type"), (dict(t=((P, 4, -1),)), "type"), (dict(t=((P + 2, 4, 0),)), "aligned"), (dict(t=((P + 1, 4, 2),)), "aligned"),
    (dict(most=-1.0), "max_norm"), (dict(most=float("nan")), "max_norm"), (dict(out=(None, None, None)), "all NULL"),
    (dict(scratch=None), "scratch"), (dict(scratch=P + 8), "scratch"), (dict(size=11), "scratch"),
    (dict(t=((P, 1 << 40, 2),) * 17), "2^44")])
def test_grad_norm_refuses(kw, word):
    refused(norm(**kw), word)


def test_grad_norm_scratch():
    L = native.lib()
    size = lambda *t: L.hieravg_grad_norm_scratch(*tensors(*t))  # noqa: E731
    assert size((P, 4, 0)) == 8 + 4 and size((P, 4, 0), (None, 0, 0), (P, 16385, 1)) == 8 * 4 + 4 * 3
    assert size((P, -4, 0)) == 0 and L.hieravg_grad_norm_scratch(None, 1) == 0
    assert size((P, 1 << 40, 2)) <= 8 * 65537 + 16


def scaled(t, out, factor=P):
    table, n = tensors(*t)
    return native.lib().hieravg_scale_tensors(table, None if out is None else (ctypes.c_void_p * n)(*out), n, factor, None)


@pytest.mark.parametrize("t,out,kw,word", [
    (((P, 4, 0),), None, {}, "NULL"), (((P, 4, 0),), (P,), dict(factor=None), "NULL"), (((P, 4, 0),), (P,), dict(factor=P + 2), "aligned"),
    (((P, 4, 0),), (None,), {}, "aligned"), (((P, 4, 0),), (P + 2,), {}, "aligned"), (((P, 4, 0),), (P + 4,), {}, "overlap"),
    (((P, 4, 0),), (P - 12,), {}, "overlap"), (((P, 4, 0), (P + 16, 4, 0)), (P + 16, P), {}, "overlap"),
    (((P, 4, 0), (P + 16, 4, 0)), (P, P + 12), {}, "overlap"), (((P, 4, 0), (P + 16, 4, 0)), (P + 64, P + 72), {}, "overlap"),
    (((P, 4, 0), (P, 4, 0)), (P, P), {}, "overlap"), (((P, 8, 0), (P + 64, 8, 0)), (P, P + 16), {}, "overlap")])
def test_scale_refuses(t, out, kw, word):
    refused(scaled(t, out, **kw), word)


def test_scale_of_nothing_is_no_call():
    assert scaled(((None, 5, 0), (P, 0, 1)), (None, None)) == 0


def verify(x=P, type=0, seqs=1, drafts=2, classes=4, stride=4, q=None, qtype=0, qstride=4, tok=P, size=4, u=P, out=(P, P, P), scratch=P,
           n=1 << 20):
    return native.lib().hieravg_verify_drafts(x, type, seqs, drafts, classes, stride, q, qtype, qstride, tok, size, u, None, None,
                                              *out, scratch, n, None)


@pytest.mark.parametrize("kw,word", [
    (dict(type=3), "type"), (dict(q=P, qtype=9), "type"), (dict(seqs=-1), "seqs"), (dict(seqs=(1 << 24) + 1), "seqs"),
    (dict(drafts=-1), "drafts"), (dict(drafts=65), "drafts"), (dict(classes=0), "classes"), (dict(classes=(1 << 23) + 1), "classes"),
    (dict(stride=3), "row_stride"), (dict(q=P, qstride=3), "draft_stride"), (dict(size=2), "token_bytes"), (dict(x=None), "logits"),
    (dict(x=P + 2), "aligned"), (dict(q=P + 1, qtype=2), "aligned"), (dict(tok=None), "draft_tokens"), (dict(tok=P + 4, size=8), "draft_tokens"),
    (dict(u=None), "uniforms"), (dict(out=(None, P, P)), "tokens"), (dict(out=(P, None, P)), "accepted"), (dict(out=(P, P, None)), "logp"),
    (dict(scratch=None), "scratch"), (dict(scratch=P + 8), "scratch"), (dict(n=64), "scratch"), (dict(stride=1 << 60), "2^56")])
def test_verify_refuses(kw, word):
    refused(verify(**kw), word)


def test_no_sequences_is_no_call():
    assert verify(seqs=0, x=None, u=None) == 0
    L = native.lib()
    assert L.hieravg_verify_drafts_scratch(0, 2, 4, 1) == 0 and L.hieravg_verify_drafts_scratch(1, 65, 4, 1) == 0
    most = L.hieravg_verify_drafts_scratch(1 << 24, 64, 1 << 23, 1)
    assert 0 < most < 1 << 30


def adapters(down=P, up=P, scales=None, k=4, cols=4, n=2, rank=2, type=0):
    return native.Adapters(down, up, scales, k, cols, n, rank, type)


def product(x=P, rows=2, stride=4, ids=P, size=4, base=None, bstride=4, out=P + 1024, otype=0, ostride=4, hidden=None, scratch=P,
            n=1 << 20, w=None, **kw):
    return native.lib().hieravg_adapter_product(adapters(**kw) if w is None else w, x, rows, stride, ids, size, base, bstride, out, otype,
                                                ostride, hidden, scratch, n, None)


COMMON = [(dict(type=5), "type"), (dict(rows=-1), "rows"), (dict(rows=(1 << 24) + 1), "rows"), (dict(n=1, rank=0), "rank"),
          (dict(rank=129), "rank"), (dict(k=0), "in and out"), (dict(cols=(1 << 24) + 1), "in and out"), (dict(down=None), "down and up"),
          (dict(up=P + 2), "down and up"), (dict(scales=P + 1), "scales"), (dict(ids=None), "ids"), (dict(size=1), "id_bytes"),
          (dict(ids=P + 4, size=8), "ids"), (dict(x=None), "x must"), (dict(x=P + 1), "x must"), (dict(stride=3), "x must"),
          (dict(scratch=None), "scratch"), (dict(scratch=P + 4), "scratch")]


@pytest.mark.parametrize("kw,word", COMMON + [
    (dict(otype=3), "type of out"), (dict(out=None), "out must"), (dict(ostride=3), "out must"), (dict(base=P + 2), "base must"),
    (dict(base=P, bstride=3), "base must"), (dict(out=P), "overlap"), (dict(out=P + 16), "overlap"), (dict(base=P + 1028), "overlap"),
    (dict(base=P + 1024, bstride=5), "overlap"), (dict(rows=1 << 24, stride=1 << 40), "x must"),
    (dict(rows=1 << 24, cols=1 << 24, ostride=1 << 24, n=1 << 62), "too many tiles")])
def test_product_refuses(kw, word):
    if kw.get("n") == 1 << 62:
        kw = dict(kw, n=None)
        w = adapters(cols=1 << 24)
        refused(native.lib().hieravg_adapter_product(w, P, 1 << 24, 4, P, 4, None, 4, P + (1 << 40), 0, 1 << 24, None, P, 1 << 62, None), word)
    else:
        n = kw.pop("n", None)
        refused(product(w=adapters(n=n, rank=kw.pop("rank", 2)) if n else None, **kw), word)


@pytest.mark.parametrize("n", [0, -1, 8193])
def test_adapters_refuse_counts(n):
    w = adapters(n=n)
    refused(product(w=w), "n must")
    assert native.lib().hieravg_adapter_product_scratch(2, w) == 0 and native.lib().hieravg_adapter_grad_scratch(2, w, 0) == 0
    refused(product(w=ctypes.POINTER(native.Adapters)()), "no adapters")


def grad(g=P, rows=2, gstride=4, x=P + 512, stride=4, ids=P, size=4, hidden=None, base=None, bstride=4, dx=P + 1024, dtype=0, dstride=4,
         dd=P + 2048, du=P + 2048, wtype=0, scratch=P, n=1 << 20, **kw):
    return native.lib().hieravg_adapter_grad(adapters(**kw), g, rows, gstride, x, stride, ids, size, hidden, base, bstride, dx, dtype, dstride,
                                             dd, du, wtype, scratch, n, None)


@pytest.mark.parametrize("kw,word", [c for c in COMMON if "n" not in c[0]] + [
    (dict(dtype=4), "type of dx"), (dict(wtype=-1), "type of dx"), (dict(dx=None, dd=None, du=None), "all NULL"), (dict(dd=P + 2), "ddown"),
    (dict(du=P + 1, wtype=2), "ddown"), (dict(rows=0), "no rows"), (dict(g=None), "grad must"), (dict(gstride=3), "grad must"),
    (dict(hidden=P + 2), "hidden"), (dict(dx=P + 1026), "dx must"), (dict(dstride=2), "dx must"), (dict(base=P, bstride=2), "base must"),
    (dict(dx=P + 512), "overlap"), (dict(dx=P + 16), "overlap"), (dict(base=P + 1020), "overlap"), (dict(n=16), "scratch")])
def test_grad_refuses(kw, word):
    refused(grad(**kw), word)


def test_no_rows_is_no_call():
    assert product(rows=0, x=None, out=None, ids=None) == 0
    assert grad(rows=0, dd=None, du=None) == 0


def test_scaled_step_refuses():
    refused(native.lib().hieravg_adamw_step_scaled(None, P, None, None), "NULL")


def test_structures_match_the_header():
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "hieravg.h")).read()
    for name, struct in (("hieravg_tensor", native.Tensor), ("hieravg_adapters", native.Adapters)):
        body = re.sub(r"/\*.*?\*/", "", text[text.index(f"typedef struct {name} {{"):text.index(f"}} {name};")], flags=re.S)
        fields = []
        for line in re.findall(r"^\s*(?:const )?(?:double|float|uint64_t|int64_t|int32_t|void)\s*([\w, *]+);", body, flags=re.M):
            fields += [f.strip(" *") for f in line.split(",")]
        assert fields == [f.rstrip("_") for f, _ in struct._fields_]
