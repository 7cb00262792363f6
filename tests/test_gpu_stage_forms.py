"""Every form of the kernels of a stage's training step (tests/stage_forms.py), against the definitions in 64 bits on the device.

Weights' gradients are compared to the bit: their operands are whole numbers and powers of two whose sums fp32 holds exactly, in whatever order."""
import pytest
import torch

import stage_forms as forms
from paper_2410_12707_amd import binding as B

pytestmark = pytest.mark.gpu


def generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def whole(gen, low, high, *shape):
    return torch.randint(low, high + 1, shape, device="cuda", generator=gen)


def spaced(t, dtype, slack):
    """t as the type, in rows with something else between them."""
    wide = torch.full((t.shape[0], t.shape[1] + slack), 1e4, dtype=dtype, device="cuda")
    wide[:, :t.shape[1]] = t.to(dtype)
    return wide[:, :t.shape[1]]


def kept(x):
    """The 8-bit form of whole numbers, which it holds exactly."""
    buffer, back = B.new_act8(*x.shape), torch.empty(x.shape, device="cuda")
    B.adatopk_act8_store(x.float(), buffer)
    B.adatopk_act8_load(buffer, back)
    assert torch.equal(back, x.float())
    return buffer


def operands(dtype, rows, n_out, n_in, seed):
    """A gradient of small whole numbers with a few tokens that use all bits of the type's pieces, an input of small ones at two scales, weight and bias."""
    gen = generator(seed)
    dy = whole(gen, -3, 3, rows, n_out)
    bits = {torch.bfloat16: 8, torch.float16: 11, torch.float32: 18}[dtype]
    picked = torch.randperm(rows, device="cuda", generator=gen)[:min(rows, 7)]
    picked[0] = rows - 1
    dy[picked] = whole(gen, -(1 << bits) + 1, (1 << bits) - 1, len(picked), n_out)
    x = whole(gen, -1, 1, rows, n_in) * (1 + whole(gen, 0, 1, rows, 1))
    return dy, x, whole(gen, -2, 2, n_in), whole(gen, -2, 2, n_in)


def check_weight_grad(dtype, rows, n_out, n_in, slack, d=None, seed=0):
    dy, x, w, b = operands(dtype, rows, n_out, n_in, seed)
    assert float((dy.double().abs().sum(0).max() * 6)) < 2 ** 24  # |weight * input + bias| <= 6: no sum leaves what fp32 holds exactly
    d = spaced(dy, dtype, slack) if d is None else d.copy_(dy.to(dtype))
    assert torch.equal(d.double(), dy.double())
    buffer, turned = kept(x), dy.double().t().contiguous()
    product, total = turned @ x.double(), dy.double().sum(0)
    del turned
    dw, db = torch.full((n_out + 1, n_in), 9.0, device="cuda"), torch.full((n_out + 1,), 9.0, device="cuda")
    ws = torch.randint(0, 256, (B.adatopk_weight_grad_workspace_bytes(rows, n_out, n_in, dtype),), dtype=torch.uint8, device="cuda")

    def check(want, of_bias, what):
        assert torch.equal(dw[:n_out].double(), want), what
        assert torch.equal(db[:n_out].double(), of_bias), what
        assert bool((dw[n_out:] == 9.0).all()) and float(db[n_out]) == 9.0, what

    B.adatopk_weight_grad(d, buffer, dw[:n_out], db[:n_out], ws)
    check(product, total, "plain")
    B.adatopk_weight_grad(d, buffer, dw[:n_out], db[:n_out], ws, accumulate=True)
    check(2 * product, 2 * total, "accumulated")
    for kind in {dtype, torch.float32}:
        wd, bd = w.to(kind), b.to(kind)
        B.adatopk_weight_grad(d, buffer, dw[:n_out], db[:n_out], ws, weight=wd, bias=bd)
        affine = product * w.double() + total[:, None] * b.double()
        check(affine, total, "weight and bias")
        B.adatopk_weight_grad(d, buffer, dw[:n_out], db[:n_out], ws, weight=wd, accumulate=True)
        check(affine + product * w.double(), 2 * total, "weight, accumulated")
        B.adatopk_weight_grad(d, buffer, dw[:n_out], None, ws, bias=bd)
        check(product + total[:, None] * b.double(), 2 * total, "bias")


@pytest.mark.parametrize("form", forms.WEIGHT_GRADIENTS, ids=lambda f: "%s-%dx%d%s%s" % (str(f[0])[6:], *f[1], "-bounded" if f[2] else "", "-shared" if f[3] else ""))
def test_weight_gradient(form):
    dtype, tile, bounded, shared, (rows, n_out, n_in) = form
    for slack in (0, 5):
        cut = B.measure_weight_grad_cut(rows, n_out, n_in, dtype, n_out + slack)
        assert cut[:2] == (tile, bounded) and (cut[2] > 1) == shared
        check_weight_grad(dtype, rows, n_out, n_in, slack, seed=rows + slack)


@pytest.mark.parametrize("size", forms.MODEL_SIZES, ids=lambda f: "%s-%dx%dx%d" % (str(f[0])[6:], *f[2]))
def test_weight_gradient_of_model_sizes(size):
    dtype, tile, (rows, n_out, n_in) = size
    assert B.measure_weight_grad_cut(rows, n_out, n_in, dtype, n_out)[:2] == (tile, False)
    check_weight_grad(dtype, rows, n_out, n_in, 0, seed=rows)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,n_out,n_in", [(5, 70, 100), (130, 200, 129), (300, 64, 64)])
def test_weight_gradient_of_rows_far_apart(dtype, rows, n_out, n_in):
    stride = (1 << 22) + 3
    assert B.measure_weight_grad_cut(rows, n_out, n_in, dtype, stride)[1]
    flat = torch.empty((rows - 1) * stride + n_out + 1, dtype=dtype, device="cuda")
    d = flat[1:].as_strided((rows, n_out), (stride, 1))
    for before in range(1, 9):  # what stands beside the rows is not read
        flat.as_strided((rows - 1, 1), (stride, 1), n_out + before).fill_(float("nan"))
        flat.as_strided((rows - 1, 1), (stride, 1), stride + 1 - before).fill_(float("nan"))
    check_weight_grad(dtype, rows, n_out, n_in, None, d=d, seed=rows)
