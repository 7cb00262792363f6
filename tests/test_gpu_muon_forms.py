"""Updates as a training step makes them (momentum, decay, weights in a wider tensor) at sizes for every form of their products, five steps and three, against their definition
in 64 bits on the device."""
import pytest
import torch

import eight_bit_forms
import muon_forms
import stage_reference as ref
from paper_2410_12707_amd import binding as B

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
EPS = 1e-7
# what a caller's constants are in fp32
MU, SCALE, DECAY = (float(torch.tensor(v)) for v in (0.95, -0.75, 0.625))


def coarse_products(dtype, steps, size):
    """Steps whose products are of 11 bits, and whether the last one's is: as the header has it."""
    if dtype == F32 or min(size) < 256:
        return 0, False
    first, behind = (2, 3) if dtype == F16 else (3, 2)
    return max(0, min(first, steps - behind)), dtype == BF16


def iterate(u, steps, coarse=0, last=False):
    """X, and how much products of 11 bits may put in: 2^-11 of their terms (roundings of 2^-12 and less in their factors) over what the step leaves, in the 2-norm; what is
    there grows by 1.6 in a step at the most (the polynomial's slope around its values, on average)."""
    x = u if u.shape[0] <= u.shape[1] else u.t().contiguous()
    x = x / (x.double().norm() + EPS).to(x.dtype)
    more = 0.0
    for step in range(steps):
        gram = x @ x.t().contiguous()
        cubic, quintic = gram @ x, gram @ (gram @ x)
        following = 3.4445 * x - 4.7750 * cubic + 2.0315 * quintic
        more *= 1.6
        if step < coarse or (last and step + 1 == steps):
            terms = 4.7750 * float(cubic.norm()) + 2.0315 * float(quintic.norm()) + (3.4445 * float(x.norm()) if step >= coarse or step + 1 == steps else 0.0)
            more += 2.0 ** -11 * terms / float(following.norm())
        x = following
    return (x if u.shape[0] <= u.shape[1] else x.t().contiguous()), more


def check(size, dtype, steps, coarse, seed=0):
    rows, cols = size
    gen = torch.Generator(device="cuda").manual_seed(rows + cols + seed)
    wide_g = torch.randn(rows, cols + 3, device="cuda", generator=gen)
    g, momentum = wide_g[:, :cols], torch.randn(rows, cols, device="cuda", generator=gen)
    wide = torch.full((rows + 1, cols + 5), 7.0, dtype=dtype, device="cuda")
    w = wide[:rows, :cols]
    w.copy_(torch.randn(rows, cols, device="cuda", generator=gen) * max(size) ** -0.5)  # of X's size
    before, after = w.double(), MU * momentum.double() + g.double()
    ws = torch.full((B.adatopk_muon_update_workspace_bytes(rows, cols),), 0xFF, dtype=torch.uint8, device="cuda")
    B.adatopk_muon_update(g, momentum, MU, True, w, SCALE, DECAY, ws, steps=steps, coarse=coarse)
    assert bool(((momentum.double() - after).abs() <= ref.U * after.abs() + ref.SMALLEST[F32]).all())
    u = g.double() + MU * momentum.double()
    exact, more = iterate(u, steps, *(coarse_products(dtype, steps, size) if coarse else (0, False)))
    single, _ = iterate(u.float(), steps)
    # as in test_gpu_muon.tolerance: four times what fp32 is off by and the pairs' own roundings; and u is rounded to fp32, which is two roundings of 2^-24
    tol = 4 * float((single.double() - exact).norm() / exact.norm()) + 64 * 2.0 ** -22 + more
    want = DECAY * before + SCALE * exact
    off = w.double() - want
    rounding = (ref.HALF_ULP[dtype] + 4 * ref.U) * 1.01

    def bound(*dim):
        kw = {"dim": dim} if dim else {}
        x = exact.norm(**kw)
        # (errors need not be spread like X is: a row or a column may have four times its share of them)
        share = x.clamp_min(float(x.mean())) * (4 if dim else 1)
        return abs(SCALE) * tol * share + rounding * (want.norm(**kw) + abs(SCALE) * tol * share) + ref.SMALLEST[dtype] * exact.numel() ** 0.5

    assert float(off.norm()) <= float(bound())
    for axis in (0, 1):  # a tile, a slice or a summand that is left out or taken twice shows in its own rows and columns
        assert bool((off.norm(dim=axis) <= bound(axis)).all())
    assert bool((wide[rows:] == 7.0).all()) and bool((wide[:, cols:] == 7.0).all())
    return w.clone(), want, float(bound())


SIZES = sorted({size for which, *_, size in eight_bit_forms.UPDATES if which < 4} | {size for which, *_, size in muon_forms.NEXT if which == 0})
COARSE_SIZES = sorted({size for *_, size in eight_bit_forms.UPDATES if min(size) >= 256} | {size for which, *_, size in muon_forms.NEXT if which > 0})


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("size", SIZES)
def test_every_form(size, dtype):
    check(size, dtype, 3, False)


@pytest.mark.parametrize("steps", [3, 4, 5])
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("size", COARSE_SIZES)
def test_every_coarse_form(size, dtype, steps):
    check(size, dtype, steps, True)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("size", [(257, 267), (1419, 1421), (1600, 6400), (2002, 6011), (6011, 2002), (258, 11728)])
def test_what_the_workspace_held_is_not_in_a_coarse_update(size, dtype):
    gen = torch.Generator(device="cuda").manual_seed(3)
    g, out = torch.randn(*size, device="cuda", generator=gen), [torch.empty(*size, dtype=dtype, device="cuda") for _ in range(2)]
    for steps in (1, 2, 3, 5, 7):
        for w, value in zip(out, (0, 0xFF)):
            ws = torch.full((B.adatopk_muon_update_workspace_bytes(*size),), value, dtype=torch.uint8, device="cuda")
            B.adatopk_muon_update(g, None, 0.0, False, w, 1.0, 0.0, ws, steps=steps, coarse=True)
        assert torch.equal(*out) and bool(torch.isfinite(out[0]).all()), steps


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("size", [(70, 131), (131, 70), (260, 400), (1419, 1421)])
def test_what_is_left_out_would_show(size, dtype):
    # the bound of check() against what a mistake in the update would change: no look ahead, no decay, a scale that is 5 percent off
    w, want, bound = check(size, dtype, 5, False, seed=1)
    rows, cols = size
    gen = torch.Generator(device="cuda").manual_seed(rows + cols + 1)
    g, m = torch.randn(rows, cols + 3, device="cuda", generator=gen)[:, :cols].double(), torch.randn(rows, cols, device="cuda", generator=gen).double()
    before = (torch.randn(rows, cols, device="cuda", generator=gen) * max(size) ** -0.5).to(dtype).double()
    exact = (want - DECAY * before) / SCALE
    for wrong in (DECAY * before + SCALE * iterate(MU * m + g, 5)[0], before + SCALE * exact, DECAY * before + 1.05 * SCALE * exact):
        assert float((wrong - want).norm()) > 2 * bound


@pytest.mark.parametrize("coarse", [False, True])
def test_coarse_is_the_callers_choice_alone(coarse):
    g = torch.randn(300, 520, device="cuda")
    ws = torch.empty(B.adatopk_muon_update_workspace_bytes(300, 520), dtype=torch.uint8, device="cuda")
    whole, halves = torch.empty(300, 520, device="cuda"), torch.empty(300, 520, dtype=BF16, device="cuda")
    B.adatopk_muon_update(g, None, 0.0, False, whole, 1.0, 0.0, ws, coarse=coarse)  # fp32 weights: the same bits
    B.adatopk_muon_update(g, None, 0.0, False, halves, 1.0, 0.0, ws, coarse=coarse)
    assert torch.equal(halves, whole.to(BF16)) is not coarse
    small = [torch.empty(255, 520, dtype=BF16, device="cuda") for _ in range(2)]  # and so have smaller ones
    for w, c in zip(small, (False, True)):
        B.adatopk_muon_update(g[:255], None, 0.0, False, w, 1.0, 0.0, ws, coarse=c)
    assert torch.equal(*small)
