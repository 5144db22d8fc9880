"""Checks of the tensor operators' C entries that need no GPU (nothing is
launched): what later entries and rules refuse."""

import ctypes

from paper_1903_05133_amd import native


def refused(rc, word):
    msg = native.lib().hieravg_last_error().decode()
    assert rc == native.EINVAL and word in msg, (rc, msg)


def test_adamw_lr_of_no_handle():
    lr = ctypes.c_double(7.0)
    refused(native.lib().hieravg_adamw_lr(None, ctypes.byref(lr)), "NULL")
    assert lr.value == 7.0


BUF = (ctypes.c_double * 64)()
P = -(-ctypes.addressof(BUF) // 64) * 64


def grad(x, stride, out, out_stride, rows=3, classes=4, type=0, lse=None):
    """A call that is refused at the latest for its lse."""
    return native.lib().hieravg_log_probs_grad(x, type, rows, classes, stride, P, 8, lse, P, P, P, out, out_stride, None)


def test_gradient_over_part_of_the_logits_is_refused():
    for out, s in ((P + 4, 6), (P - 4, 6), (P + 24, 6), (P + 24 + 12, 6), (P + 24 - 12, 6), (P, 5), (P, 4), (P + 24, 4),
                   (P - 48, 6), (P + 48, 6)):
        refused(grad(P, 6, out, s), "overlap")
    refused(grad(P, 6, P + 4, 6, rows=1), "overlap")
    refused(grad(P, 6, P + 8, 6, type=1), "overlap")


def test_gradient_beside_or_over_the_logits_is_not():
    for out, s, rows in ((P, 8, 3), (P + 16, 8, 3), (P - 16, 8, 3), (P + 80, 8, 3), (P + 3 * 32, 4, 3), (P, 9, 1),
                         (P + 16, 8, 1), (P - 16, 5, 1), (P + 32 * 2 + 16, 8, 3), (P - 32 * 2 - 16, 8, 3)):
        refused(grad(P, 8, out, s, rows=rows), "lse is NULL")


def test_adamw_objects_are_not_copied():
    """Two objects with one handle would free it twice."""
    import copy
    import pickle

    import pytest
    from paper_1903_05133_amd import operators
    a = operators.AdamW.__new__(operators.AdamW)
    for f in (copy.copy, copy.deepcopy, pickle.dumps):
        with pytest.raises(TypeError, match="state"):
            f(a)
