"""Every form of the kernels of a stage's training step (tests/stage_forms.py), against the definitions in 64 bits on the device.

Weights' gradients are compared to the bit: their operands are whole numbers and powers of two whose sums fp32 holds exactly, in whatever order."""
import pytest
import torch

import stage_forms as forms
import stage_reference as ref
from paper_2410_12707_amd import binding as B

pytestmark = pytest.mark.gpu
U = ref.U


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


# ---------------------------------------------------------------- layer norm
def dx_and_bound(dy, h, d_h, rstd, weight, dsum, dtype):
    """The input's gradient in 64 bits, and by how much 32-bit sums in a team and the roundings behind them may miss it (stage_reference's bounds)."""
    g, r = dy * weight, rstd[:, None]
    level, along = g.mean(1, keepdim=True), (g * h).mean(1, keepdim=True)
    dx = r * (g - level - h * along) + dsum
    size_level, size_along = g.abs().mean(1, keepdim=True), (g * h).abs().mean(1, keepdim=True)
    d = (ref.DEPTH + 6) * U * (size_level + h.abs() * size_along) + 6 * U * g.abs() + d_h * size_along + h.abs() * (g.abs() * d_h).mean(1, keepdim=True)
    return dx, r * d + 2 * U * dsum.abs() + (ref.HALF_ULP[dtype] + U) * dx.abs() + ref.SMALLEST[dtype]


@pytest.mark.parametrize("keep", [False, True], ids=["from-x", "from-8-bits"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("form", forms.BACKWARD, ids=lambda f: "%dx%d-%dx%d" % (f[0], f[1], *f[2]))
def test_layer_norm_backward_with_the_sums_beside_the_rows(form, dtype, keep):
    lanes, octets, (rows, cols) = form
    cut = B.measure_layernorm_cut(rows, cols, True)
    assert cut[:2] == (lanes, octets) and cut[3] == 0 and cut[2] < rows
    gen = generator(rows)
    dy, x = whole(gen, -3, 3, rows, cols), whole(gen, -4, 4, rows, cols)
    # h = (x - mean) * rstd exactly: means are whole numbers, 1 / deviations powers of two
    mean, rstd = whole(gen, -2, 2, rows), torch.exp2(whole(gen, -1, 1, rows).double())
    h = x.double() if keep else (x - mean[:, None]).double() * rstd[:, None]
    weight = 1 + 0.3 * torch.randn(cols, device="cuda", generator=gen, dtype=torch.float64)
    weight = weight.to(dtype if cols % 2 else torch.float32)
    dsum = torch.randn(rows, cols, device="cuda", generator=gen).to(dtype)
    buffer = kept(x) if keep else None
    d, x_d = spaced(dy, dtype, 3 if cols % 2 else 0), None if keep else spaced(x, dtype, 5 if cols % 2 else 0)
    mean_d, rstd_d = None if keep else mean.float(), rstd.float()
    want_w, want_b = (dy.double() * h).sum(0), dy.double().sum(0)
    ws = torch.randint(0, 256, (B.adatopk_layernorm_backward_workspace_bytes(rows, cols),), dtype=torch.uint8, device="cuda")
    dx, dw, db = torch.empty(rows, cols, dtype=dtype, device="cuda"), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    for add in (None, dsum):
        want, bound = dx_and_bound(dy.double(), h, 0.0 * h, rstd, weight.double(), torch.zeros_like(h) if add is None else add.double(), dtype)
        B.adatopk_layernorm_backward(d, x_d, buffer, mean_d, rstd_d, weight, dx, dw, db, ws, dsum=add)
        assert torch.equal(dw.double(), want_w) and torch.equal(db.double(), want_b)
        assert bool(((dx.double() - want).abs() <= bound).all())
    B.adatopk_layernorm_backward(d, x_d, buffer, mean_d, rstd_d, weight, torch.empty_like(dx), dw, db, ws, accumulate=True)
    assert torch.equal(dw.double(), 2 * want_w) and torch.equal(db.double(), 2 * want_b)
    B.adatopk_layernorm_backward(d, x_d, buffer, mean_d, rstd_d, weight, d, None, db, ws, dsum=dsum)  # over dy
    assert torch.equal(d, dx) and torch.equal(db.double(), want_b)


@pytest.mark.parametrize("keep", [False, True], ids=["from-x", "from-8-bits"])
def test_layer_norm_backward_weights_over_very_many_rows(keep):
    # 2.16 G elements; 1319 rows of each of the 1024 teams pass through its 32-bit sums
    rows, cols = 1_350_000, 1601
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    dy = torch.empty_like(x)
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    want_w, want_b = (torch.zeros(cols, dtype=torch.float64, device="cuda") for _ in range(2))
    for lo in range(0, rows, 50_000):
        gen = generator(lo)
        part = slice(lo, lo + 50_000)
        x[part], dy[part] = (whole(gen, -1, 1, 50_000, cols).to(torch.bfloat16) for _ in range(2))
        mean[part], rstd[part] = whole(gen, -1, 1, 50_000).float(), torch.exp2(whole(gen, 0, 1, 50_000).float())
        h = x[part].float() if keep else (x[part].float() - mean[part, None]) * rstd[part, None]
        want_w += (dy[part].float() * h).sum(0)  # (whole numbers below 2^24)
        want_b += dy[part].float().sum(0)
    buffer = None
    if keep:
        buffer = torch.empty(B.adatopk_act8_bytes(rows, cols), dtype=torch.uint8, device="cuda")
        B.adatopk_act8_store(x, buffer)
    ws = torch.empty(B.adatopk_layernorm_backward_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    dw, db = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    dx = torch.empty_like(x)
    B.adatopk_layernorm_backward(dy, None if keep else x, buffer, None if keep else mean, rstd, None, dx, dw, db, ws)
    assert torch.equal(dw.double(), want_w) and torch.equal(db.double(), want_b)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("form", forms.FORWARD, ids=lambda f: "%dx%d-%dx%d" % (f[0], f[1], *f[2]))
def test_layer_norm_forward_where_teams_go_round(form, dtype):
    lanes, octets, (rows, cols) = form
    cut = B.measure_layernorm_cut(rows, cols, False)
    assert cut[:2] == (lanes, octets) and cut[2] < rows
    gen = generator(rows)
    x, r = (torch.randn(rows, cols, device="cuda", generator=gen).to(dtype) for _ in range(2))
    w, b = (1 + 0.3 * torch.randn(cols, device="cuda", generator=gen)).to(dtype), (0.3 * torch.randn(cols, device="cuda", generator=gen)).to(dtype)
    d = spaced(x, dtype, 3 if cols % 2 else 0)
    for residual in (None, r):
        s = x.double() if residual is None else (x.float() + r.float()).to(dtype).double()  # (a 32-bit sum of two 16-bit values rounds as the exact one does)
        mean, rstd, y = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty_like(x)
        total = None if residual is None else torch.empty_like(x)
        buffer = B.new_act8(rows, cols)
        B.adatopk_layernorm_forward(d, w, b, 1e-5, y, mean, rstd, residual=residual, sum_out=total, act8=buffer)
        if residual is not None:
            assert torch.equal(total.double(), s)
        want_mean = s.mean(1)
        left = s - want_mean[:, None]
        want_rstd = 1.0 / torch.sqrt((left * left).mean(1) + 1e-5)
        h = left * want_rstd[:, None]
        d_mean = mean_bound(s, want_mean, dtype)
        assert bool(((mean.double() - want_mean).abs() <= d_mean).all())
        r_rstd = (ref.DEPTH + 6) * U + (d_mean * want_rstd) ** 2 + 2 * d_mean * want_rstd * h.abs().mean(1)
        assert bool(((rstd.double() - want_rstd).abs() <= r_rstd * want_rstd).all())
        d_h = (d_mean * want_rstd)[:, None] + U * h.abs() + h.abs() * (r_rstd[:, None] + 3 * U)
        want = h * w.double() + b.double()
        d_y = w.double().abs() * d_h + 3 * U * ((h * w.double()).abs() + b.double().abs())
        assert bool(((y.double() - want).abs() <= d_y + ref.HALF_ULP[dtype] * (want.abs() + d_y) + ref.SMALLEST[dtype]).all())
        back = torch.empty(rows, cols, device="cuda")
        B.adatopk_act8_load(buffer, back)
        # a number is off by half a step, a 128th of the group's largest power of two, or a whole one where it is clamped: a 64th of the largest value
        groups = torch.nn.functional.pad(h, (0, -cols % 32)).view(rows, -1, 32).abs().amax(2).repeat_interleave(32, 1)[:, :cols]
        assert bool(((back.double() - h).abs() <= groups / 127.5 + 2 * d_h + U * groups).all())


def mean_bound(s, mean, dtype):
    """A mean's sum is held in 64 bits: one 32-bit rounding of the result, and for 16-bit types three additions of eight values in 32 bits before it."""
    size = s.abs().mean(1)
    return mean.abs() * (1.0 + 2.0 ** -20) * U + size * (2.0 ** -44 + (0.0 if dtype == torch.float32 else 3 * U)) + 2.0 ** -149


@pytest.mark.parametrize("cols", [17, 64, 250, 768, 1601, 4095, 8190, 16379, 32767])
def test_means_of_values_that_cancel(cols):
    # magnitudes of up to 1e4, each with its negative somewhere else in the row, and an exact rest: the mean is a millionth of them and less, which a sum
    # in 32 bits would miss altogether
    gen = generator(cols)
    rows = 40
    half = torch.randn(rows, cols // 2, device="cuda", generator=gen) * torch.exp2(whole(gen, 0, 13, rows, 1).float())
    x = torch.cat([half, -half, torch.zeros(rows, cols % 2, device="cuda")], 1)[:, torch.randperm(cols, device="cuda", generator=gen)].contiguous()
    x += torch.randn(rows, cols, device="cuda", generator=gen) * 1e-3
    mean, rstd, y = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty_like(x)
    B.adatopk_layernorm_forward(x, None, None, 1e-5, y, mean, rstd)
    want = x.double().mean(1)
    assert bool(((mean.double() - want).abs() <= mean_bound(x.double(), want, torch.float32)).all())
    in_32 = x.float().sum(1).double() / cols
    if cols > 1000:  # the test tells the two apart
        assert bool(((in_32 - want).abs() > mean_bound(x.double(), want, torch.float32)).any())
