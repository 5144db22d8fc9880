"""Low-rank adapters, gradient norms and the verification of drafts at their limits,
without a GPU: sizes of scratch, and refusals, which come before any launch."""

import ctypes
import os
import shutil
import subprocess

import pytest

from paper_1903_05133_amd import build, native

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


def test_overlap_of_operands(tmp_path):
    """meet() against a search over all bytes, under sanitizers."""
    if not shutil.which(build.hipcc()):
        pytest.skip("hipcc not found")
    exe = str(tmp_path / "operand_overlap_check")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    cmd = [build.hipcc(), "-x", "hip", "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-Xarch_host", "-fsanitize=address", "-Xarch_host",
           "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=undefined", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
           "-I", os.path.join(root, "include"), "-I", build.CSRC, os.path.join(root, "tests", "operand_overlap_check.cpp"), "-o", exe]
    res = subprocess.run(cmd, capture_output=True, text=True, timeout=300)
    assert res.returncode == 0, res.stderr[-4000:]
    run = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert run.returncode == 0 and "overlap ok" in run.stdout, run.stdout[-2000:] + run.stderr[-2000:]


BIG = (ctypes.c_double * 4096)()
Q = -(-ctypes.addressof(BIG) // 64) * 64
# 3 rows of 8 float32, 2 adapters of rank 2: every operand at a place of its own
PLACES = dict(down=Q, up=Q + 256, scales=Q + 512, x=Q + 1024, ids=Q + 2048, base=Q + 3072, out=Q + 4096, hidden=Q + 5120, grad=Q + 6144,
              ddown=Q + 7168, dup=Q + 8192, scratch=Q + 16384)
SIZES = dict(down=128, up=128, scales=8, x=96, ids=12, base=96, out=96, hidden=24, grad=96)


def product(scratch_bytes=1 << 13, **kw):
    p = dict(PLACES, **kw)
    w = native.Adapters(p["down"], p["up"], p["scales"], 8, 8, 2, 2, 0)
    rc = native.lib().hieravg_adapter_product(w, p["x"], 3, p.get("x_stride", 8), p["ids"], 4, p["base"], 8, p["out"], 0, p.get("out_stride", 8),
                                              p["hidden"], p["scratch"], scratch_bytes, None)
    return rc, native.lib().hieravg_last_error().decode()


def gradient(scratch_bytes=1 << 13, **kw):
    p = dict(PLACES, **kw)
    w = native.Adapters(p["down"], p["up"], p["scales"], 8, 8, 2, 2, 0)
    rc = native.lib().hieravg_adapter_grad(w, p["grad"], 3, 8, p["x"], 8, p["ids"], 4, p["hidden"], p["base"], 8, p["out"], 0, 8, p["ddown"],
                                           p["dup"], 0, p["scratch"], scratch_bytes, None)
    return rc, native.lib().hieravg_last_error().decode()


@pytest.mark.parametrize("call,result,others", [
    (product, "out", "down up scales x ids base"), (product, "hidden", "down up scales x ids base out"),
    (gradient, "out", "down up scales x ids base hidden grad"), (gradient, "ddown", "down up scales x ids base hidden grad out dup"),
    (gradient, "dup", "down up scales x ids base hidden grad out ddown")])
def test_results_overlap_no_operand(call, result, others):
    for other in others.split():
        for at in (0, 4, -4):  # first byte on first, one element on, one before
            rc, msg = call(**{result: PLACES[other] + at})
            if (result, other, at) == ("out", "base", 0):  # in place
                continue
            assert rc == native.EINVAL and "overlap" in msg, (result, other, at, msg)


def test_results_beside_operands_are_not_refused():
    """Neighbours, and ids in a gap between rows: such calls get as far as their scratch, which is too small."""
    for call in (product, gradient):
        for result in ("out", "hidden") if call is product else ("out", "ddown", "dup"):
            for other, size in SIZES.items():
                if other != result:
                    rc, msg = call(scratch_bytes=4, **{result: PLACES[other] + size})
                    assert rc == native.EINVAL and "scratch" in msg, (result, other, msg)
    rc, msg = product(scratch_bytes=4, out=Q + 1024 + 32, out_stride=16, x=Q + 1024, x_stride=16)
    assert rc == native.EINVAL and "scratch" in msg
    rc, msg = product(scratch_bytes=4, out_stride=16, ids=PLACES["out"] + 32 + 4)
    assert rc == native.EINVAL and "scratch" in msg
    rc, msg = product(scratch_bytes=4, out_stride=16, ids=PLACES["out"] + 32 + 24)
    assert rc == native.EINVAL and "overlap" in msg


@pytest.mark.parametrize("place", range(3))
def test_norm_results_are_aligned(place):
    t = (native.Tensor * 1)(native.Tensor(P, 4, 0))
    out = [P + 1024, P + 2048, P + 2052]
    out[place] += 2
    rc = native.lib().hieravg_grad_norm(t, 1, 1.0, *out, Q, 1 << 13, None)
    assert rc == native.EINVAL and "aligned" in native.lib().hieravg_last_error().decode()


def test_hidden_is_aligned():
    rc, msg = product(hidden=PLACES["hidden"] + 2)
    assert rc == native.EINVAL and "hidden" in msg and "aligned" in msg


# 2 sequences of 2 drafts over 4 classes, every operand at a place of its own
DRAFTS = dict(x=Q, q=Q + 1024, drafts=Q + 2048, uniforms=Q + 3072, lengths=Q + 4096, temperature=Q + 5120, tokens=Q + 6144, accepted=Q + 7168,
              logp=Q + 8192, scratch=Q + 16384)


def verify(scratch_bytes=1 << 13, **kw):
    p = dict(DRAFTS, **kw)
    rc = native.lib().hieravg_verify_drafts(p["x"], 0, 2, 2, 4, p.get("stride", 4), p["q"], 0, 4, p["drafts"], 4, p["uniforms"], p["lengths"],
                                            p["temperature"], p["tokens"], p["accepted"], p["logp"], p["scratch"], scratch_bytes, None)
    return rc, native.lib().hieravg_last_error().decode()


@pytest.mark.parametrize("what", ["uniforms", "lengths", "temperature", "tokens", "accepted", "logp"])
def test_operands_of_verification_are_aligned(what):
    for off in (1, 2, 3):
        rc, msg = verify(**{what: DRAFTS[what] + off})
        assert rc == native.EINVAL and "aligned" in msg, msg
    rc, msg = verify(scratch_bytes=4)
    assert rc == native.EINVAL and "scratch" in msg


@pytest.mark.parametrize("result", ["tokens", "accepted", "logp"])
def test_results_of_verification_overlap_nothing(result):
    sizes = dict(x=96, q=64, drafts=16, uniforms=24, lengths=8, temperature=8, tokens=24, accepted=8, logp=24)
    for other, size in sizes.items():
        if other == result:
            continue
        for at in (0, 4, -4):
            rc, msg = verify(**{result: DRAFTS[other] + at})
            assert rc == native.EINVAL and "overlap" in msg, (result, other, at, msg)
        rc, msg = verify(scratch_bytes=4, **{result: DRAFTS[other] + size})
        assert rc == native.EINVAL and "scratch" in msg


@pytest.mark.parametrize("at,place", [(0, 0), (12, 0), (0, 1), (28, 1)])
def test_factor_is_no_result(at, place):
    """A factor inside a tensor that is scaled, in place or into another."""
    t = (native.Tensor * 2)(native.Tensor(Q, 4, 0), native.Tensor(Q + 1024, 8, 0))
    out = (ctypes.c_void_p * 2)(Q, Q + 2048)
    rc = native.lib().hieravg_scale_tensors(t, out, 2, out[place] + at, None)
    assert rc == native.EINVAL and "factor" in native.lib().hieravg_last_error().decode()
