"""The weight gradient from an 8-bit input on the GPU, against the plain statements in 64 bits (tests/stage_reference.py)."""
import numpy as np
import pytest
import torch

import stage_reference as ref
from paper_2410_12707_amd import binding as B

pytestmark = pytest.mark.gpu
DTYPES = [torch.float32, torch.bfloat16, torch.float16]
# rows, n_out, n_in: a token, odd sizes, edges of the tiles, splits that end inside a tile of tokens
SHAPES = [(1, 1, 1), (1, 5, 33), (2, 8, 8), (15, 32, 32), (16, 33, 31), (17, 128, 128), (31, 129, 127), (32, 64, 200), (33, 256, 256), (63, 257, 255), (64, 100, 1),
          (65, 1, 100), (100, 300, 40), (257, 130, 514), (1000, 77, 95), (2049, 40, 33), (4097, 130, 129), (515, 768, 768), (9000, 16, 24), (700, 520, 1030)]


def workspace(rows, n_out, n_in, dtype):
    n = B.adatopk_weight_grad_workspace_bytes(rows, n_out, n_in, dtype)
    return torch.randint(0, 256, (n,), dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("dtype", DTYPES)
def test_whole_numbers_are_exact(dtype):
    # small whole numbers: every sum is exact in fp32, whatever its order, so the result is the definition's to the bit
    for i, (rows, n_out, n_in) in enumerate(SHAPES):
        rng = np.random.default_rng(i)
        dy, x = rng.integers(-4, 5, size=(rows, n_out)).astype(np.float64), rng.integers(-3, 4, size=(rows, n_in)).astype(np.float64)
        assert np.array_equal(ref.act8_encode(x)[2], x)
        buffer = torch.from_numpy(ref.act8_buffer(x)).cuda()
        ws = workspace(rows, n_out, n_in, dtype)
        dw_e, db_e = ref.weight_grad(dy, x)
        for slack, offset in ((0, 0), (5, 1), (8, 8)):
            d = ref.on_device(dy, dtype, slack, offset)
            dw, db = torch.full((n_out + 1, n_in), 9.0, device="cuda"), torch.full((n_out + 1,), 9.0, device="cuda")
            B.adatopk_weight_grad(d, buffer, dw[:n_out], db[:n_out], ws)
            assert np.array_equal(ref.host(dw[:n_out]), dw_e), (rows, n_out, n_in, slack)
            assert np.array_equal(ref.host(db[:n_out]), db_e), (rows, n_out, n_in, slack)
            assert bool((dw[n_out:] == 9.0).all()) and float(db[n_out]) == 9.0
        B.adatopk_weight_grad(d, buffer, dw[:n_out], db[:n_out], ws, accumulate=True)
        assert np.array_equal(ref.host(dw[:n_out]), 2 * dw_e) and np.array_equal(ref.host(db[:n_out]), 2 * db_e)
        B.adatopk_weight_grad(d, buffer, dw[:n_out], None, ws)
        assert np.array_equal(ref.host(dw[:n_out]), dw_e)
        w, b = rng.integers(-2, 3, size=n_in).astype(np.float64), rng.integers(-2, 3, size=n_in).astype(np.float64)
        for use_w, use_b in ((True, True), (True, False), (False, True)):
            for kind in {dtype, torch.float32}:
                wd, bd = (torch.from_numpy(v).to(kind).cuda() if use else None for v, use in ((w, use_w), (b, use_b)))
                B.adatopk_weight_grad(d, buffer, dw[:n_out], db[:n_out], ws, weight=wd, bias=bd)
                want = ref.weight_grad(dy, x, w if use_w else None, b if use_b else None)
                assert np.array_equal(ref.host(dw[:n_out]), want[0]) and np.array_equal(ref.host(db[:n_out]), db_e), (rows, n_out, n_in, use_w, use_b)


@pytest.mark.parametrize("dtype", DTYPES)
def test_real_numbers(dtype):
    for i, (rows, n_out, n_in) in enumerate(SHAPES):
        rng = np.random.default_rng(300 + i)
        dy = ref.rounded(rng.standard_t(3, size=(rows, n_out)) * 1e-3, dtype)
        x = rng.normal(size=(rows, n_in)) * np.exp2(rng.integers(-6, 6, size=(rows, 1)).astype(np.float64))
        held = ref.act8_encode(x)[2]
        buffer = torch.from_numpy(ref.act8_buffer(x)).cuda()
        w, b = ref.rounded(1 + 0.2 * rng.normal(size=n_in), dtype), ref.rounded(0.2 * rng.normal(size=n_in), dtype)
        d, ws = ref.on_device(dy, dtype), workspace(rows, n_out, n_in, dtype)
        dw, db = torch.empty(n_out, n_in, device="cuda"), torch.empty(n_out, device="cuda")
        for affine in (False, True):
            v = (w, b) if affine else (None, None)
            wd, bd = (None if a is None else torch.from_numpy(a).to(dtype).cuda() for a in v)
            B.adatopk_weight_grad(d, buffer, dw, db, ws, weight=wd, bias=bd)
            want, bounds = ref.weight_grad(dy, held, *v), ref.weight_grad_bounds(dy, held, *v)
            assert (np.abs(ref.host(dw) - want[0]) <= bounds[0]).all(), (rows, n_out, n_in, affine)
            assert (np.abs(ref.host(db) - want[1]) <= bounds[1]).all(), (rows, n_out, n_in, affine)
        again, ws2 = torch.empty_like(dw), workspace(rows, n_out, n_in, dtype)
        B.adatopk_weight_grad(d, buffer, again, db, ws2, weight=wd, bias=bd)
        assert torch.equal(again, dw)  # equal calls, equal bits


@pytest.mark.parametrize("dtype", DTYPES)
def test_every_bit_of_a_gradient_counts(dtype):
    # one token, an input of ones: the result is the gradient itself, over the type's whole range
    rng = np.random.default_rng(2)
    if dtype == torch.float32:
        bits = rng.integers(0, 1 << 32, size=4096, dtype=np.uint64).astype(np.uint32)
        dy = torch.from_numpy(bits.view(np.float32).copy())
        dy = torch.where(torch.isfinite(dy) & (dy.abs() > 1e-30), dy, torch.full_like(dy, 1.5))  # the last piece of smaller ones is no normal number
    else:
        dy = torch.from_numpy(rng.integers(0, 1 << 16, size=4096, dtype=np.uint32).astype(np.uint16).view(np.int16)).view(dtype)
        dy = torch.where(torch.isfinite(dy) & (dy.float().abs() > 1e-30), dy, torch.full_like(dy, 1.5))
    dy = dy.view(1, -1).cuda()
    buffer = torch.from_numpy(ref.act8_buffer(np.ones((1, 2)))).cuda()
    dw, db = torch.empty(4096, 2, device="cuda"), torch.empty(4096, device="cuda")
    B.adatopk_weight_grad(dy, buffer, dw, db, workspace(1, 4096, 2, dtype))
    assert torch.equal(dw[:, 0], dy[0].float()) and torch.equal(dw[:, 1], dy[0].float()) and torch.equal(db, dy[0].float())


@pytest.mark.parametrize("dtype", DTYPES)
def test_nonfinite_values_stay_in_their_rows_and_columns(dtype):
    rng = np.random.default_rng(4)
    rows, n_out, n_in = 70, 150, 96
    dy, x = ref.rounded(rng.normal(size=(rows, n_out)), dtype), rng.normal(size=(rows, n_in))
    dy[3, 7], dy[69, 149] = np.inf, np.nan
    x[5, 40] = np.nan  # its group: columns 32 to 63
    dw, db = torch.empty(n_out, n_in, device="cuda"), torch.empty(n_out, device="cuda")
    buffer = torch.from_numpy(ref.act8_buffer(x)).cuda()
    B.adatopk_weight_grad(ref.on_device(dy, dtype), buffer, dw, db, workspace(rows, n_out, n_in, dtype))
    bad = np.zeros((n_out, n_in), dtype=bool)
    bad[7], bad[149], bad[:, 32:64] = True, True, True
    assert np.array_equal(~np.isfinite(ref.host(dw)), bad)
    finite = np.isfinite(ref.host(db))
    assert np.array_equal(~finite, np.isin(np.arange(n_out), (7, 149))) and float(db[7]) == np.inf and np.isnan(float(db[149]))


def test_no_rows():
    dw, db, ws = torch.full((5, 7), 3.0, device="cuda"), torch.full((5,), 3.0, device="cuda"), workspace(0, 5, 7, torch.float32)
    dy, buffer = torch.empty(0, 5, device="cuda"), torch.zeros(16, dtype=torch.uint8, device="cuda")
    B.adatopk_weight_grad(dy, buffer, dw, db, ws, accumulate=True)
    assert bool((dw == 3.0).all()) and bool((db == 3.0).all())
    B.adatopk_weight_grad(dy, buffer, dw, db, ws)
    assert bool((dw == 0.0).all()) and bool((db == 0.0).all())


def test_refusals():
    dy, buffer, ws = torch.randn(64, 48, device="cuda"), B.new_act8(64, 96), workspace(64, 48, 96, torch.float32)
    dw, db, w = torch.empty(48, 96, device="cuda"), torch.empty(48, device="cuda"), torch.ones(96, device="cuda")
    for call, word in ((lambda: B.adatopk_weight_grad(dy, buffer, dw[:47], db, ws), "dw must"), (lambda: B.adatopk_weight_grad(dy, buffer, dw.half(), db, ws), "dw must"),
                       (lambda: B.adatopk_weight_grad(dy, buffer, dw[:, :95], db, ws), "contiguous"), (lambda: B.adatopk_weight_grad(dy, buffer[:-100], dw, db, ws), "act8_x must"),
                       (lambda: B.adatopk_weight_grad(dy, buffer, dw, db[:47], ws), "db must"), (lambda: B.adatopk_weight_grad(dy, buffer, dw, db, ws, weight=w[:95]), "weight must"),
                       (lambda: B.adatopk_weight_grad(dy, buffer, dw, db, ws, bias=w.half()), "bias must")):
        with pytest.raises(ValueError, match=word):
            call()
    if B.adatopk_weight_grad_workspace_bytes(64, 48, 96, torch.float32) > 0:
        with pytest.raises(B.AdaTopKError):
            B.adatopk_weight_grad(dy, buffer, dw, db, ws[:0])


def test_more_elements_than_32_bits_count():
    rows, n_out, n_in = 300_000, 7_500, 40  # 2.25 G elements of the gradient
    dy = torch.randint(-1, 2, (rows, n_out), dtype=torch.int8, device="cuda").to(torch.bfloat16)
    x = torch.randint(-1, 2, (rows, n_in), dtype=torch.int8, device="cuda").float()
    buffer = B.new_act8(rows, n_in)
    B.adatopk_act8_store(x, buffer)
    dw, db = torch.empty(n_out, n_in, device="cuda"), torch.empty(n_out, device="cuda")
    B.adatopk_weight_grad(dy, buffer, dw, db, torch.empty(B.adatopk_weight_grad_workspace_bytes(rows, n_out, n_in, torch.bfloat16), dtype=torch.uint8, device="cuda"))
    for n in (0, 1, 4_000, 7_499):
        column = dy[:, n].float()
        assert torch.equal(dw[n], (column[:, None] * x).sum(0)) and float(db[n]) == float(column.sum())


@pytest.mark.parametrize("dtype", DTYPES)
def test_larger_tiles_whole_numbers(dtype):
    # products large enough for every tile that there is, with edges that are no multiples of it, and a token or two into a tile's tokens
    for rows, n_out, n_in in ((130, 6400, 1600), (65, 4099, 4100), (257, 2000, 1700), (1029, 1030, 771), (64, 5000, 200), (193, 300, 3333), (33, 3001, 6001), (5000, 1281, 1601)):
        gen = torch.Generator(device="cuda").manual_seed(rows)
        dy = torch.randint(-4, 5, (rows, n_out + 8), device="cuda", generator=gen).to(dtype)[:, :n_out]
        x = torch.randint(-3, 4, (rows, n_in), device="cuda", generator=gen).float()
        w, b = (torch.randint(-2, 3, (n_in,), device="cuda", generator=gen).to(dtype) for _ in range(2))
        buffer = B.new_act8(rows, n_in)
        B.adatopk_act8_store(x, buffer)
        dw, db = torch.full((n_out + 1, n_in), 9.0, device="cuda"), torch.empty(n_out, device="cuda")
        ws = workspace(rows, n_out, n_in, dtype)
        for affine in (False, True):
            B.adatopk_weight_grad(dy, buffer, dw[:n_out], db, ws, weight=w if affine else None, bias=b if affine else None)
            held = x.double() * w.double() + b.double() if affine else x.double()
            assert torch.equal(dw[:n_out].double(), dy.double().t().contiguous() @ held), (rows, n_out, n_in, affine)
            assert torch.equal(db.double(), dy.double().sum(0)) and bool((dw[n_out] == 9.0).all())
        B.adatopk_weight_grad(dy, buffer, dw[:n_out], db, ws, accumulate=True)
        assert torch.equal(dw[:n_out].double(), dy.double().t().contiguous() @ (held + x.double())), (rows, n_out, n_in)
