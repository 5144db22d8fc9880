"""The tensor operators where their arithmetic is at a limit: sums whose terms
cancel, logits of large magnitude, second moments below the normal range, and
what a state leaves out.  u = 2^-24 is half a step of float32."""

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module")
def ops(gpu_lib):
    from paper_1903_05133_amd import operators
    return operators


@pytest.fixture(autouse=True)
def float32_by_default():
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


# ------------------------------------------------------------------ 8-bit blocks
# Every form of the product: few rows on either side, split and not, 128 x 128
# tiles, split and not, 256 x 256 tiles, with contractions of every rest of 4 blocks.
SUMS = [(1, 100, 128), (1, 40, 9000), (16, 50, 500), (20, 300, 1100), (700, 32, 386), (64, 64, 4000), (130, 129, 258),
        (129, 200, 1026), (300, 515, 640), (2304, 2304, 100), (2304, 2050, 254), (2304, 2050, 514), (2100, 4097, 640), (2049, 2304, 770), (2304, 2304, 1030)]


@pytest.mark.parametrize("m,n,k", SUMS)
def test_block_product_of_terms_that_cancel(m, n, k, ops):
    """Two products of 448 x 448 that cancel in every block beside integers up to
    9: every partial sum is a whole number below 2^24, which float32 holds, so
    the result is the exact sum, rounded once to the output's type."""
    say("products that cancel", m, n, k)
    x = torch.randint(-3, 4, (m, k), generator=gen(k)).float()
    w = torch.randint(-3, 4, (n, k), generator=gen(k + 1)).float()
    x[:, 0::128] = 448
    x[:, 1::128] = 448
    w[:, 0::128] = 448
    w[:, 1::128] = -448
    a, _ = ops.quantize_blocks(x.cuda())
    want = (x.cuda().double() @ w.cuda().double().t()).float()  # whole numbers: exact in both
    for tiles in (False, True):
        b, _ = ops.quantize_blocks(w.cuda(), tiles=tiles)
        for dtype in (torch.bfloat16, torch.float16):
            got = ops.block_product(a, b, dtype)
            assert torch.equal(got, want.to(dtype))


@pytest.mark.parametrize("m,n,k", [(2, 40, 130), (100, 130, 300), (2304, 2304, 514)])
def test_block_product_at_every_scale(m, n, k, ops):
    """Scale bytes 0 to 254 against their inverses, ones for codes: k exactly
    (2^-127 is below the normal range).  Byte 255 is NaN."""
    say("scales", m, n, k)

    def ones(rows, byte):
        pitch, blocks, spitch = ops.block_shape(rows, k)
        codes = torch.zeros(rows, pitch, dtype=torch.uint8, device="cuda")
        codes[:, :k] = 0x38
        scales = torch.full((blocks, spitch), byte, dtype=torch.uint8, device="cuda")
        return ops.BlockTensor(codes.view(torch.float8_e4m3fn), scales, rows, k)

    want = torch.full((m, n), float(k), device="cuda").to(torch.float16)
    for byte in (0, 1, 2, 3, 60, 127, 200, 253, 254):
        assert torch.equal(ops.block_product(ones(m, byte), ones(n, 254 - byte), torch.float16), want), byte
    assert torch.all(torch.isnan(ops.block_product(ones(m, 255), ones(n, 127))))
    assert torch.all(torch.isnan(ops.block_product(ones(m, 127), ones(n, 255))))
