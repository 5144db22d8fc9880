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
