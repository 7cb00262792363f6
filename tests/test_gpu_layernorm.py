"""Layer norm's forward and backward pass on the GPU, against the plain statements in 64 bits (tests/stage_reference.py)."""
import numpy as np
import pytest
import torch

import stage_reference as ref
from paper_2410_12707_amd import binding as B

pytestmark = pytest.mark.gpu
DTYPES = [torch.float32, torch.bfloat16, torch.float16]
SHAPES = [(1, 1), (1, 2), (1, 7), (5, 8), (1, 31), (3, 33), (9, 64), (2, 511), (3, 512), (3, 513), (4, 768), (6, 1023), (5, 1024), (17, 1025), (130, 1600),
          (7, 1601), (5, 2048), (5, 2049), (3, 4096), (3, 4097), (2, 8192), (2, 8199), (2, 16384), (2, 16390), (2, 32768), (1000, 40), (2100, 130)]
EPS = 1e-5


def weights(cols, dtype, seed):
    rng = np.random.default_rng(seed)
    w, b = ref.rounded(1 + 0.3 * rng.normal(size=cols), dtype), ref.rounded(0.3 * rng.normal(size=cols), dtype)
    return w, b, torch.from_numpy(w).to(dtype).cuda(), torch.from_numpy(b).to(dtype).cuda()


def check_forward(x, y, mean, rstd, w, b, eps, dtype):
    ey, em, er, h = ref.layernorm(x, w, b, eps)
    dy, dm, dr, dh = ref.layernorm_bounds(x, w, b, em, er, h, ey, dtype)
    assert (np.abs(ref.host(y) - ey) <= dy).all()
    if mean is not None:
        assert (np.abs(ref.host(mean) - em) <= dm).all() and (np.abs(ref.host(rstd) - er) <= dr).all()
    return h, dh


@pytest.mark.parametrize("dtype", DTYPES)
def test_forward(dtype):
    for i, (rows, cols) in enumerate(SHAPES):
        rng = np.random.default_rng(i)
        x = ref.rounded(rng.normal(size=(rows, cols)) * (1 + 10 * (rng.random(cols) < 0.02)) + 0.5, dtype)
        w, b, dw, db = weights(cols, dtype if i % 2 else torch.float32, i)
        for slack, offset in ((0, 0), (5, 1)):
            d, y = ref.on_device(x, dtype, slack, offset), ref.on_device(np.zeros_like(x), dtype, slack, offset)
            mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
            B.adatopk_layernorm_forward(d, dw, db, EPS, y, mean, rstd)
            check_forward(x, y, mean, rstd, w, b, EPS, dtype)
            whole = y._base
            gaps = whole.clone()
            gaps[offset:offset + rows * (cols + slack)].view(rows, cols + slack)[:, :cols] = 7.0
            assert bool((gaps == 7.0).all()), "wrote between or behind the rows"
        B.adatopk_layernorm_forward(d, dw, db, EPS, d, None, None)  # in place, no statistics
        assert torch.equal(d, y)


@pytest.mark.parametrize("dtype", DTYPES)
def test_forward_with_residual_and_rows_kept(dtype):
    for i, (rows, cols) in enumerate(SHAPES):
        rng = np.random.default_rng(50 + i)
        x, r = ref.rounded(rng.normal(size=(rows, cols)), dtype), ref.rounded(rng.normal(size=(rows, cols)) * 2, dtype)
        total = ref.rounded(x + r, dtype)  # (both fp32 sums of two 16-bit values and their rounding are exact roundings of the sum)
        w, b, dw, db = weights(cols, dtype, i)
        d, e = ref.on_device(x, dtype, 3), ref.on_device(r, dtype, 9, 1)
        s, y = torch.empty(rows, cols, dtype=dtype, device="cuda"), torch.empty(rows, cols, dtype=dtype, device="cuda")
        mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        n = B.adatopk_act8_bytes(rows, cols)
        buffer = torch.full((n + 64,), 0xAB, dtype=torch.uint8, device="cuda")
        B.adatopk_layernorm_forward(d, dw, db, EPS, y, mean, rstd, residual=e, sum_out=s, act8=buffer[:n])
        assert np.array_equal(ref.host(s), total)
        h, dh = check_forward(total, y, mean, rstd, w, b, EPS, dtype)
        # what is kept is within half a step of a value within dh of h (a whole step at the clamped end)
        back = torch.empty(rows, cols, device="cuda")
        B.adatopk_act8_load(buffer[:n], back)
        numbers, exponents = ref.act8_split(buffer.cpu().numpy()[:n], rows, cols)
        step = np.repeat(np.ldexp(1.0, exponents.astype(np.int64) - 133), 32, axis=1)[:, :cols]
        clamped = np.abs(numbers[:, :cols].astype(np.int64)) == 127
        assert (np.abs(ref.host(back) - h) <= step * np.where(clamped, 1.0, 0.5) + dh).all(), (rows, cols)
        amax = np.abs(np.pad(h, ((0, 0), (0, -cols % 32)))).reshape(rows, -1, 32).max(axis=2)
        slack = np.pad(dh, ((0, 0), (0, -cols % 32))).reshape(rows, -1, 32).max(axis=2)
        top = np.ldexp(1.0, exponents.astype(np.int64) - 126)  # the group's largest magnitude lies in [top / 2, top)
        assert ((amax < top + slack) & ((amax >= top / 2 - slack) | (exponents == 7))).all()
        assert (numbers[:, cols:] == 0).all() and bool((buffer[n:] == 0xAB).all())
        only = torch.empty_like(y)
        B.adatopk_layernorm_forward(d, dw, db, EPS, only, None, None, residual=e)  # no sum, nothing kept
        assert torch.equal(only, y)
        B.adatopk_layernorm_forward(s, dw, db, EPS, only, None, None)  # the sum alone
        assert torch.equal(only, y)
        wide = torch.empty_like(y)
        B.adatopk_layernorm_forward(d, dw, db, EPS, wide, None, None, residual=e, sum_out=e)  # the sum over the residual
        assert torch.equal(wide, y) and torch.equal(e, s)


def test_forward_without_weights_and_rows_that_are_alike():
    for dtype in DTYPES:
        x = torch.randn(9, 100, device="cuda").to(dtype)
        ones, zeros = torch.ones(100, device="cuda", dtype=dtype), torch.zeros(100, device="cuda", dtype=dtype)
        a, b = torch.empty_like(x), torch.empty_like(x)
        for w, v in ((None, zeros), (ones, None), (None, None)):
            B.adatopk_layernorm_forward(x, w, v, EPS, a, None, None)
            B.adatopk_layernorm_forward(x, ones, zeros, EPS, b, None, None)
            assert torch.equal(a, b)
        x = torch.full((4, 257), 3.0, device="cuda", dtype=dtype)  # no variance: the sum is exact, so is the mean up to its division
        y, mean, rstd = torch.empty_like(x), torch.empty(4, device="cuda"), torch.empty(4, device="cuda")
        B.adatopk_layernorm_forward(x, None, None, EPS, y, mean, rstd)
        assert bool((mean - 3.0).abs().max() <= 1e-6) and bool((rstd - EPS ** -0.5).abs().max() <= 0.01) and bool(y.float().abs().max() <= 1e-3)


def test_nonfinite_rows_stay_to_themselves():
    for cols in (40, 1600, 3000):
        x = torch.randn(6, cols, device="cuda")
        x[1, 3], x[4, cols - 1] = float("nan"), float("inf")
        y, buffer, back = torch.empty_like(x), B.new_act8(6, cols), torch.empty_like(x)
        B.adatopk_layernorm_forward(x, None, None, EPS, y, None, None, act8=buffer)
        B.adatopk_act8_load(buffer, back)
        for row in range(6):
            bad = row in (1, 4)
            assert bool(torch.isnan(y[row]).all()) == bad and bool(torch.isnan(back[row]).all()) == bad
            assert bad or bool(torch.isfinite(y[row]).all())


@pytest.mark.parametrize("keep", [False, True])
@pytest.mark.parametrize("dtype", DTYPES)
def test_backward(dtype, keep):
    for i, (rows, cols) in enumerate(SHAPES):
        rng = np.random.default_rng(200 + i)
        x, dy = ref.rounded(rng.normal(size=(rows, cols)) + 0.3, dtype), ref.rounded(rng.normal(size=(rows, cols)), dtype)
        w, _, dw, _ = weights(cols, dtype if i % 2 else torch.float32, i)
        mean, rstd = (x.mean(axis=1)).astype(np.float32).astype(np.float64), (1 / np.sqrt(x.var(axis=1) + EPS)).astype(np.float32).astype(np.float64)
        exact = (x - mean[:, None]) * rstd[:, None]
        h = ref.act8_encode(exact)[2] if keep else exact
        d_h = np.zeros_like(h) if keep else ref.U * (np.abs(x - mean[:, None]) * rstd[:, None] + np.abs(h) * 2)
        with_sum = i % 3 != 0
        dsum = ref.rounded(rng.normal(size=(rows, cols)), dtype) if with_sum else np.zeros((rows, cols))
        expected = ref.layernorm_backward(dy, h, rstd, w, dsum)
        bounds = ref.layernorm_backward_bounds(dy, h, d_h, rstd, w, dsum, expected[0], dtype)
        buffer = torch.from_numpy(ref.act8_buffer(exact)).cuda() if keep else None
        ws = torch.empty(max(B.adatopk_layernorm_backward_workspace_bytes(rows, cols), 256), dtype=torch.uint8, device="cuda")
        dm, dr = torch.from_numpy(mean).float().cuda(), torch.from_numpy(rstd).float().cuda()
        for slack, offset in ((0, 0), (3, 1)):
            d, dx = ref.on_device(dy, dtype, slack, offset), ref.on_device(np.zeros_like(dy), dtype, slack, offset)
            dsum_d = ref.on_device(dsum, dtype, slack, offset) if with_sum else None
            x_d = None if keep else ref.on_device(x, dtype, slack, offset)
            gw, gb = torch.full((cols,), 9.0, device="cuda"), torch.full((cols,), 9.0, device="cuda")
            B.adatopk_layernorm_backward(d, x_d, buffer, None if keep else dm, dr, dw, dx, gw, gb, ws, dsum=dsum_d)
            for got, want, bound in zip((dx, gw, gb), expected, bounds):
                assert (np.abs(ref.host(got) - want) <= bound).all(), (rows, cols, slack)
        ws.random_(0, 256)
        again = [torch.empty_like(dx), torch.empty_like(gw), torch.empty_like(gb)]
        B.adatopk_layernorm_backward(d, x_d, buffer, None if keep else dm, dr, dw, *again, ws, dsum=dsum_d)
        assert torch.equal(again[0], dx) and torch.equal(again[1], gw) and torch.equal(again[2], gb)  # equal calls, equal bits
        more = [torch.full((cols,), 2.0, device="cuda"), torch.full((cols,), -1.0, device="cuda")]
        B.adatopk_layernorm_backward(d, x_d, buffer, None if keep else dm, dr, dw, again[0], *more, ws, dsum=dsum_d, accumulate=True)
        assert torch.equal(more[0], gw + 2.0) and torch.equal(more[1], gb - 1.0)
        B.adatopk_layernorm_backward(d, x_d, buffer, None if keep else dm, dr, dw, again[0], None, None, None, dsum=dsum_d)
        assert torch.equal(again[0], dx)
        B.adatopk_layernorm_backward(d, x_d, buffer, None if keep else dm, dr, dw, again[0], None, more[0], ws, dsum=dsum_d)
        assert torch.equal(more[0], gb)
        B.adatopk_layernorm_backward(d, x_d, buffer, None if keep else dm, dr, dw, d, gw, gb, ws, dsum=dsum_d)  # in place
        assert torch.equal(d, dx) and torch.equal(gw, again[1])


def test_backward_against_differences():
    # the loss sum(dy * layernorm(x)) moved by a step in x, in 64 bits
    rng = np.random.default_rng(5)
    rows, cols = 3, 45
    x, dy = ref.rounded(rng.normal(size=(rows, cols)), torch.float32), ref.rounded(rng.normal(size=(rows, cols)), torch.float32)
    w, b, dw, _ = weights(cols, torch.float32, 3)
    d, dx = ref.on_device(dy, torch.float32), torch.empty(rows, cols, device="cuda")
    mean, rstd, y = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty(rows, cols, device="cuda")
    gw, gb = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    ws = torch.empty(B.adatopk_layernorm_backward_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    x_d = ref.on_device(x, torch.float32)
    B.adatopk_layernorm_forward(x_d, dw, None, EPS, y, mean, rstd)
    B.adatopk_layernorm_backward(d, x_d, None, mean, rstd, dw, dx, gw, gb, ws)

    def loss(x, w):
        return (ref.layernorm(x, w, 0.0, EPS)[0] * dy).sum()

    for got, at in ((dx, "x"), (gw, "w")):
        for i in np.ndindex(tuple(got.shape)):
            step = np.zeros(tuple(got.shape))
            step[i] = 1e-5
            slope = (loss(x + step, w) - loss(x - step, w) if at == "x" else loss(x, w + step) - loss(x, w - step)) / 2e-5
            assert abs(slope - float(got[i])) < 2e-5, (at, i)


def test_nothing_to_do():
    x = torch.empty(0, 64, device="cuda")
    B.adatopk_layernorm_forward(x, None, None, EPS, x, None, None)
    gw, gb = torch.full((64,), 3.0, device="cuda"), torch.full((64,), 4.0, device="cuda")
    ws = torch.empty(256, dtype=torch.uint8, device="cuda")
    none = torch.empty(0, device="cuda")
    B.adatopk_layernorm_backward(x, x, None, none, none, None, x, gw, gb, ws, accumulate=True)
    assert bool((gw == 3.0).all()) and bool((gb == 4.0).all())
    B.adatopk_layernorm_backward(x, x, None, none, none, None, x, gw, gb, ws)
    assert bool((gw == 0.0).all()) and bool((gb == 0.0).all())


def test_refusals():
    x, y, w, s = torch.randn(4, 64, device="cuda"), torch.empty(4, 64, device="cuda"), torch.ones(64, device="cuda"), torch.empty(4, device="cuda")
    ws = torch.empty(1 << 16, dtype=torch.uint8, device="cuda")
    for call, word in ((lambda: B.adatopk_layernorm_forward(x, w[:63], None, EPS, y, s, s), "weight must"),
                       (lambda: B.adatopk_layernorm_forward(x, w.half(), None, EPS, y, s, s), "weight must"),
                       (lambda: B.adatopk_layernorm_forward(x.half(), w, w.half(), EPS, y.half(), s, s), "bias must"),
                       (lambda: B.adatopk_layernorm_forward(x, w, w, EPS, y.half(), s, s), "y must"),
                       (lambda: B.adatopk_layernorm_forward(x, w, w, EPS, y, s[:3], s), "mean must"),
                       (lambda: B.adatopk_layernorm_forward(x, w, w, EPS, y, s, s, residual=y[:3]), "residual must"),
                       (lambda: B.adatopk_layernorm_forward(x, w, w, EPS, y, s, s, act8=ws[:10]), "act8 must"),
                       (lambda: B.adatopk_layernorm_backward(x, y.half(), None, s, s, w, y, w, w, ws), "x must"),
                       (lambda: B.adatopk_layernorm_backward(x, y, None, s, s, w, y, w[:60], w, ws), "dweight must")):
        with pytest.raises(ValueError, match=word):
            call()
    for call in (lambda: B.adatopk_layernorm_forward(x, w, w, EPS, y, s, s, sum_out=y), lambda: B.adatopk_layernorm_forward(x, w, w, -1.0, y, s, s),
                 lambda: B.adatopk_layernorm_backward(x, None, None, s, s, w, y, w, w, ws), lambda: B.adatopk_layernorm_backward(x, x, None, s, s, w, y, w, w, ws[:256])):
        with pytest.raises(B.AdaTopKError):
            call()


def test_more_elements_than_32_bits_count():
    rows, cols = 1_350_000, 1601  # 2.16 G elements, rows at odd places
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    for lo in range(0, rows, 90_000):
        x[lo:lo + 90_000] = torch.randn(90_000, cols, device="cuda", generator=torch.Generator(device="cuda").manual_seed(lo)).to(torch.bfloat16)
    y, mean, rstd = torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    buffer = torch.empty(B.adatopk_act8_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    B.adatopk_layernorm_forward(x, None, None, EPS, y, mean, rstd, act8=buffer)
    picked = [0, 1, 1_341_332, 1_341_333, 1_349_999]
    check_forward(ref.host(x[picked]), y[picked], mean[picked], rstd[picked], np.ones(cols), np.zeros(cols), EPS, torch.bfloat16)
    gw, gb = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    ws = torch.empty(B.adatopk_layernorm_backward_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    dx = torch.empty_like(x)
    B.adatopk_layernorm_backward(y, x, None, mean, rstd, None, dx, gw, gb, ws)
    h = (ref.host(x[picked]) - ref.host(mean[picked])[:, None]) * ref.host(rstd[picked])[:, None]
    dy, r = ref.host(y[picked]), ref.host(rstd[picked])
    expected = ref.layernorm_backward(dy, h, r, 1.0, 0.0)[0]
    d_h = ref.U * 4 * (np.abs(h) + 1)
    bound = ref.layernorm_backward_bounds(dy, h, d_h, r, np.ones(cols), np.zeros_like(dy), expected, torch.bfloat16)[0]
    assert (np.abs(ref.host(dx[picked]) - expected) <= bound).all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_backward_of_many_rows_that_are_wide(dtype):
    """Above 16384 columns the sums over the rows go in shares of at most 1024 rows: one and two of them, added to what is there, dx over dy."""
    cols = 16401
    for rows in (1024, 1030):
        gen = torch.Generator(device="cuda").manual_seed(rows)
        x, dy = ((torch.randn(rows, cols, device="cuda", generator=gen) + 0.25).to(dtype) for _ in range(2))
        y, mean, rstd = torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        buffer = B.new_act8(rows, cols)
        B.adatopk_layernorm_forward(x, None, None, EPS, y, mean, rstd, act8=buffer)
        kept = torch.empty(rows, cols, device="cuda")
        B.adatopk_act8_load(buffer, kept)
        ws = torch.empty(B.adatopk_layernorm_backward_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
        for keep in (False, True):
            source = (None, buffer, None) if keep else (x, None, mean)
            alone, dx = torch.empty_like(x), dy.clone()
            B.adatopk_layernorm_backward(dy, *source, rstd, None, alone, None, None, None)
            dw, db = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
            B.adatopk_layernorm_backward(dx, *source, rstd, None, dx, dw, db, ws)
            assert torch.equal(dx, alone)
            g = dy.double()
            h = kept.double() if keep else (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
            # every term is rounded twice before it is added, the sum at most once for each row
            error = (rows + 4) * 2.0 ** -24
            assert bool(((dw - (g * h).sum(0)).abs() <= error * (g * h).abs().sum(0)).all())
            assert bool(((db - g.sum(0)).abs() <= error * g.abs().sum(0)).all())
            first_w, first_b = dw.clone(), db.clone()
            B.adatopk_layernorm_backward(dy, *source, rstd, None, dx, dw, db, ws, accumulate=True)
            assert torch.equal(dw, first_w + first_w) and torch.equal(db, first_b + first_b) and torch.equal(dx, alone)
