"""Products of matrices in 8-bit floating point on the GPU, against 64 bits on the CPU."""
import numpy as np
import pytest
import torch

import fp8_reference as fp8
import stage_reference as ref
from paper_2410_12707_amd import binding as B

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def operands(rng, rows, n_out, n_in):
    """Buffers and values of x and w, blocks of very different scales among them."""
    x = rng.standard_normal((rows, n_in)) * np.exp2(rng.integers(-8, 8, (rows, -(-n_in // 128)))).repeat(128, axis=1)[:, :n_in]
    w = rng.standard_normal((n_out, n_in)) * np.exp2(rng.integers(-3, 3, (n_out, 1)))
    x, w = ref.rounded(x, F32), ref.rounded(w, F32)
    return (torch.from_numpy(fp8.fp8_buffer(x)).cuda(), torch.from_numpy(fp8.fp8_buffer(w, 128)).cuda(), fp8.fp8_encode(x)[2], fp8.fp8_encode(w, 128)[2])


def workspace(rows, n_out, n_in):
    return torch.full((max(B.adatopk_fp8_product_workspace_bytes(rows, n_out, n_in), 256),), 0xFF, dtype=torch.uint8, device="cuda")


def product(rng, dtype, rows, n_out, n_in, bias=False, add=False, wide=False, slack=0, in_place=False):
    bx, bw, x, w = operands(rng, rows, n_out, n_in)
    kind = F32 if wide else dtype
    b = ref.rounded(rng.standard_normal(n_out), kind) if bias else None
    a = ref.rounded(rng.standard_normal((rows, n_out)), dtype) if add else None
    out = torch.full((rows, n_out + slack), 7.0, dtype=dtype, device="cuda")
    y = out[:, :n_out]
    summand = None
    if add:
        summand = y.copy_(torch.from_numpy(a).to(dtype)) if in_place else ref.on_device(a, dtype, slack, 1 if slack else 0)
    ws = workspace(rows, n_out, n_in)
    B.adatopk_fp8_product(bx, bw, n_in, y, ws, bias=None if b is None else torch.from_numpy(b).to(kind).cuda(), add=summand)
    expected = x @ w.T + (0.0 if b is None else b) + (0.0 if a is None else a)
    bound = fp8.product_bound(x, w, expected, dtype) + 2 * fp8.U * ((0.0 if b is None else np.abs(b)) + (0.0 if a is None else np.abs(a)))
    got = ref.host(y)
    off = np.abs(got - expected) / bound
    assert off.max() <= 1, (off.max(), np.unravel_index(off.argmax(), off.shape))
    assert (ref.host(out)[:, n_out:] == 7.0).all()
    if not in_place:
        again = torch.zeros_like(y)
        B.adatopk_fp8_product(bx, bw, n_in, again, ws, bias=None if b is None else torch.from_numpy(b).to(kind).cuda(), add=summand)
        assert torch.equal(again, y)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("shape", [(1, 1, 1), (1, 17, 128), (2, 40, 129), (15, 33, 1000), (16, 100, 640), (17, 31, 300), (32, 64, 256), (33, 16, 200), (63, 50, 4500),
                                   (64, 129, 1100)])
def test_few_tokens(dtype, shape):
    rng = np.random.default_rng(sum(shape))
    product(rng, dtype, *shape)
    product(rng, dtype, *shape, bias=True, add=True, slack=3)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("shape", [(65, 1, 1), (65, 64, 128), (70, 65, 129), (100, 200, 1000), (300, 77, 385), (257, 513, 260), (129, 1000, 5000), (512, 768, 768)])
def test_tiles(dtype, shape):
    rng = np.random.default_rng(sum(shape))
    product(rng, dtype, *shape)
    product(rng, dtype, *shape, bias=True, add=True, slack=3)


@pytest.mark.parametrize("dtype,shape", [(BF16, (4100, 4099, 300)), (F32, (4096, 4096, 128)), (F16, (2300, 2049, 1000))])
def test_large_tiles(dtype, shape):
    product(np.random.default_rng(sum(shape)), dtype, *shape, bias=True)


@pytest.mark.parametrize("shape", [(1, 40, 130), (90, 70, 300), (300, 260, 520)])
def test_wide_bias_and_summand_in_place(shape):
    rng = np.random.default_rng(5)
    product(rng, BF16, *shape, bias=True, wide=True)
    product(rng, F16, *shape, bias=True, add=True, in_place=True)
    product(rng, BF16, *shape, add=True, in_place=True, slack=5)


@pytest.mark.parametrize("rows", [3, 100])
def test_nothing_to_add_up(rows):
    y, bias = torch.full((rows, 21), 7.0, device="cuda"), torch.randn(21, device="cuda")
    nothing = torch.empty(16, dtype=torch.uint8, device="cuda")
    B.adatopk_fp8_product(nothing, nothing, 0, y, None)
    assert (y == 0).all()
    B.adatopk_fp8_product(nothing, nothing, 0, y, None, bias=bias)
    assert torch.equal(y, bias.expand(rows, 21))


@pytest.mark.parametrize("rows", [5, 200])
def test_rows_that_are_no_numbers_stay_alone(rows):
    rng = np.random.default_rng(6)
    x, w = rng.standard_normal((rows, 300)), rng.standard_normal((90, 300))
    x[2, 140], w[3, 5] = np.inf, np.nan
    x, w = ref.rounded(x, F32), ref.rounded(w, F32)
    y = torch.empty(rows, 90, device="cuda")
    B.adatopk_fp8_product(torch.from_numpy(fp8.fp8_buffer(x)).cuda(), torch.from_numpy(fp8.fp8_buffer(w)).cuda(), 300, y, workspace(rows, 90, 300))
    nan = np.isnan(ref.host(y))
    expected = np.zeros((rows, 90), dtype=bool)
    expected[2], expected[:, 3] = True, True
    assert np.array_equal(nan, expected)


@pytest.mark.parametrize("rows", [2, 150])
def test_scales_from_end_to_end(rows):
    # the largest scales against the smallest, and sums that pass out of the type
    x, w = np.zeros((rows, 256)), np.zeros((16, 256))
    x[:, 0], w[:, 0] = 2.0 ** 127, 2.0 ** -126
    x[:, 200], w[:, 200] = 2.0 ** -100, 2.0 ** 101
    w[3, 0], w[4, 200] = 2.0, 0.0
    y = torch.empty(rows, 16, device="cuda")
    B.adatopk_fp8_product(torch.from_numpy(fp8.fp8_buffer(x)).cuda(), torch.from_numpy(fp8.fp8_buffer(w)).cuda(), 256, y, workspace(rows, 16, 256))
    expected = x @ w.T
    expected[:, 3] = np.inf
    assert np.array_equal(ref.host(y), expected)
