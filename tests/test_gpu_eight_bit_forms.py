"""Every form of the kernels behind products in 8-bit floating point and updates of weights (tests/eight_bit_forms.py), against their definitions in 64 bits on the device."""
import pytest
import torch

import eight_bit_forms as forms
import stage_reference as ref
from paper_2410_12707_amd import binding as B

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
EPS = 1e-7


def generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def dirty(size):
    return torch.full((max(size, 256),), 0xFF, dtype=torch.uint8, device="cuda")


def stored(t, store):
    """A matrix's buffer and what it holds."""
    buffer, back = B.new_fp8(*t.shape), torch.empty(t.shape, device="cuda")
    store(t, buffer)
    B.adatopk_fp8_load(buffer, back)
    return buffer, back.double()


def largest_of_eight(t):
    t = torch.nn.functional.pad(t.abs(), (0, -t.shape[1] % 8))
    return t.view(t.shape[0], -1, 8).amax(2)


def product_bound(x, w, y, dtype):
    """fp8_reference.product_bound on the device."""
    bound = (x.abs() @ w.abs().t().contiguous()) * (2 * ref.U * (8 + 2 * x.shape[1] ** 0.5)) + 2 * ref.U * y.abs() + ref.HALF_ULP[dtype] * y.abs() * (1 + 2.0 ** -8)
    if dtype != F32:
        bound += 2.0 ** -10 * (largest_of_eight(x) @ largest_of_eight(w).t().contiguous())
    return bound + ref.SMALLEST[dtype]


@pytest.mark.parametrize("dtype,form,size", [form for form in forms.PRODUCTS] + [(F16, form, size) for dtype, form, size in forms.PRODUCTS if dtype == BF16])
def test_product(dtype, form, size):
    rows, n_out, n_in = size
    gen = generator(sum(size))
    scales = torch.exp2(torch.randint(-6, 7, (rows, (n_in + 127) // 128), device="cuda", generator=gen).float()).repeat_interleave(128, 1)[:, :n_in]
    bx, x = stored(torch.randn(rows, n_in, device="cuda", generator=gen) * scales, B.adatopk_fp8_store)
    bw, w = stored(torch.randn(n_out, n_in, device="cuda", generator=gen) * n_in ** -0.5, B.adatopk_fp8_store_weight)
    bias, add = (torch.randn(*shape, device="cuda", generator=gen).to(dtype) for shape in ((n_out,), (rows, n_out)))
    wide = torch.full((rows + 1, n_out + 3), 7.0, dtype=dtype, device="cuda")
    y, ws = wide[:rows, :n_out], dirty(B.adatopk_fp8_product_workspace_bytes(*size))
    B.adatopk_fp8_product(bx, bw, n_in, y, ws, bias=bias, add=add)
    want = x @ w.t().contiguous() + bias.double() + add.double()
    bound = product_bound(x, w, want, dtype) + 2 * ref.U * (bias.double().abs() + add.double().abs())
    assert float(((y.double() - want).abs() / bound).max()) <= 1
    assert bool((wide[rows:] == 7.0).all()) and bool((wide[:, n_out:] == 7.0).all())
    again = torch.empty(rows, n_out, dtype=dtype, device="cuda")
    B.adatopk_fp8_product(bx, bw, n_in, again, ws, bias=bias, add=add)
    assert torch.equal(again, y)


def update_steps(x, steps):
    x = x / (x.double().norm() + EPS).to(x.dtype)
    for _ in range(steps):
        gram = x @ x.t().contiguous()
        x = 3.4445 * x + (-4.7750 * gram + 2.0315 * (gram @ gram)) @ x
    return x


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("size", sorted({size for *_, size in forms.UPDATES}))
def test_update(dtype, size):
    # three steps: where w has 16 bits and a shorter side of 256 or more, the first is a coarse one and so is the last one's product in bf16
    rows, cols = size
    gen = generator(rows + cols)
    g = torch.randn(rows, cols, device="cuda", generator=gen) + 3 * torch.randn(rows, 6, device="cuda", generator=gen) @ torch.randn(6, cols, device="cuda", generator=gen)
    wide = torch.full((rows + 1, cols + 5), 7.0, dtype=dtype, device="cuda")
    w, ws = wide[:rows, :cols], dirty(B.adatopk_muon_update_workspace_bytes(rows, cols))
    w.fill_(0.5)
    B.adatopk_muon_update(g, None, 0.0, False, w, 1.0, 0.0, ws, steps=3)
    turned = rows > cols
    x = g.t().contiguous() if turned else g
    exact, single = update_steps(x.double(), 3), update_steps(x, 3).double()
    got = w.double().t() if turned else w.double()
    # as in test_gpu_muon.tolerance: four times what fp32 is off by, the pairs' own roundings, products of 11 bits and w's rounding
    tol = 4 * float((single - exact).norm() / exact.norm()) + 64 * 2.0 ** -22 + ref.HALF_ULP[dtype] * 1.01 + (4e-3 if dtype == BF16 and min(size) >= 256 else 0.0)
    assert float((got - exact).norm() / exact.norm()) <= tol
    # a tile or a slice that is left out or taken twice shows in its own rows and columns
    for axis in (0, 1):
        assert float(((got - exact).norm(dim=axis) / exact.norm(dim=axis).clamp_min(float(exact.norm(dim=axis).mean()))).max()) <= 4 * tol
    assert bool((wide[rows:] == 7.0).all()) and bool((wide[:, cols:] == 7.0).all())
    again = torch.empty(rows, cols, dtype=dtype, device="cuda")
    B.adatopk_muon_update(g, None, 0.0, False, again, 1.0, 0.0, ws, steps=3)
    assert torch.equal(again, w)


def test_what_the_workspace_held_is_not_in_an_update():
    rng = torch.Generator().manual_seed(8)
    for n in range(40):
        less, more = (int(torch.randint(1, most, (1,), generator=rng)) for most in ((330, 30000) if n % 2 == 0 else (2500, 2500)))
        for rows, cols in ((less, more), (more, less)):
            g = torch.randn(rows, cols, device="cuda", generator=generator(n))
            out = [torch.empty(rows, cols, dtype=BF16 if n % 4 < 2 else F32, device="cuda") for _ in range(2)]
            for w, value in zip(out, (0, 0xFF)):
                ws = torch.full((B.adatopk_muon_update_workspace_bytes(rows, cols),), value, dtype=torch.uint8, device="cuda")
                B.adatopk_muon_update(g, None, 0.0, False, w, 1.0, 0.0, ws, steps=3)
            assert torch.equal(*out), (rows, cols)
