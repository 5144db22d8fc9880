"""Low-rank adapters, gradient norms and the verification of drafts at their limits,
without a GPU: sizes of scratch, and refusals, which come before any launch."""

import ctypes

import pytest

from paper_1903_05133_amd import native

BUF = (ctypes.c_double * 512)()
P = -(-ctypes.addressof(BUF) // 64) * 64


def adapters(n, rank, k, cols, type=2):
    return native.Adapters(P, P, None, k, cols, n, rank, type)


@pytest.mark.parametrize("rows", [1000, 8192, 100000])
def test_adapter_grad_scratch_grows_with_rows(rows):
    """With the rows given, more adapters take tables of some 50 bytes each, and not sums of their own: only adapters
    with several units of rows have such, 2 rows / 64 at most."""
    L = native.lib()
    rank, k, cols = 16, 4096, 4096
    # h and dh in up to 16 parts, and by place in three parts of 2 bytes, four ints a tile and a unit, the order
    most = lambda n: rows * 16 * (2 * 4 * 16 + 2 * 6) + (n + 2 * (rows // 64 + 1)) * 64 + 4 * rows + 1024  # noqa: E731
    for n in (1, 8, 1000, 8192):
        sums = min(2 * (rows // 4096), rows // 4096 + n) * 4 * rank * (k + cols) if n >= 1000 else (rows // 64 + 8) * 4 * rank * (k + cols)
        for hidden in (0, 1):
            size = L.hieravg_adapter_grad_scratch(rows, adapters(n, rank, k, cols), hidden)
            assert 0 < size <= most(n) + sums, (n, hidden, size)


def grad(rows, w, scratch=None):
    return native.lib().hieravg_adapter_grad(w, P, rows, w.out, P, w.in_, P, 4, None, None, 0, None, 0, 0, P, P, 0, scratch, 0, None)


@pytest.mark.parametrize("rows,n,rank,k,cols", [(100, 8192, 128, 8192, 8192), (4096, 8192, 128, 8192, 8192), (100000, 4000, 64, 16384, 16384)])
def test_adapter_grad_of_many_adapters_is_not_refused(rows, n, rank, k, cols):
    """Sums of several units are joined for the few adapters that have several, so their number is no limit: such a call
    gets as far as its missing scratch."""
    rc = grad(rows, adapters(n, rank, k, cols))
    assert rc == native.EINVAL and "scratch" in native.lib().hieravg_last_error().decode()


@pytest.mark.parametrize("rows", [1, 64, 65, 5000])
@pytest.mark.parametrize("n", [1, 300])
def test_gradient_in_x_alone_needs_no_sums(rows, n):
    """Its scratch: the rows' order and tiles, and the parts of dh, which is 64 bytes a row in each of up to 16 parts."""
    L = native.lib()
    w = adapters(n, 16, 4096, 4096)
    size = L.hieravg_adapter_dx_scratch(rows, w)
    assert 0 < size <= rows * (64 * 16 + 4) + (rows // 64 + n + 2) * 16 + 64
    assert size < L.hieravg_adapter_grad_scratch(rows, w, 1) < L.hieravg_adapter_grad_scratch(rows, w, 0)
    assert L.hieravg_adapter_dx_scratch(0, w) == 0 and L.hieravg_adapter_dx_scratch(rows, adapters(n, 129, 8, 8)) == 0

    def call(x, dx, dd, n_bytes):
        rc = L.hieravg_adapter_grad(w, P, rows, 4096, x, 4096, P, 4, None, None, 0, dx, 0, 4096, dd, None, 0, P + 4, n_bytes, None)
        return rc, L.hieravg_last_error().decode()

    # (the misaligned scratch is refused whatever its size, so that nothing is launched)
    far = P + (1 << 40)
    for rc, msg in (call(None, far, None, size), call(far, None, far, 1 << 40)):
        assert rc == native.EINVAL and "scratch" in msg
