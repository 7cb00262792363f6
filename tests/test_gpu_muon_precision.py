"""How far the orthogonalised update of 16-bit weights is off, apart from the weights' own rounding, over gradients that treat roundings differently."""
import numpy as np
import pytest
import torch

import stage_reference as ref
from paper_2410_12707_amd import binding as B

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
EPS = 1e-7


def few_rows(gen, rows, cols, k):
    g = torch.zeros(rows, cols, device="cuda")
    g[torch.randperm(rows, device="cuda", generator=gen)[:k]] = torch.randn(k, cols, device="cuda", generator=gen)
    return g


def low_rank(gen, rows, cols, k, noise):
    n = lambda *s: torch.randn(*s, device="cuda", generator=gen)  # noqa: E731
    return n(rows, k) @ n(k, cols) * k ** -0.5 + noise * n(rows, cols)


def of_many_sizes(gen, rows, cols):
    return torch.exp(3 * torch.randn(rows, 1, device="cuda", generator=gen)) * torch.randn(rows, cols, device="cuda", generator=gen)


# a rounding where singular values are small grows in the steps that follow, one where they are near 1 stays, and one in few rows is not levelled by sums over many
GRADIENTS = {
    "noise": lambda gen, r, c: torch.randn(r, c, device="cuda", generator=gen),
    "one row": lambda gen, r, c: few_rows(gen, r, c, 1),
    "20 rows": lambda gen, r, c: few_rows(gen, r, c, 20),
    "rows of many sizes": of_many_sizes,
    "rank 4": lambda gen, r, c: low_rank(gen, r, c, 4, 0.0),
    "rank 16 and noise": lambda gen, r, c: low_rank(gen, r, c, 16, 0.5),
}
SIZES = [(256, 256), (512, 1024), (700, 300)]


def orthogonalised(g, steps):
    x = g if g.shape[0] <= g.shape[1] else g.t().contiguous()
    x = x / (x.double().norm() + EPS).to(x.dtype)
    for _ in range(steps):
        gram = x @ x.t().contiguous()
        x = 3.4445 * x + (-4.7750 * gram + 2.0315 * (gram @ gram)) @ x
    return x if g.shape[0] <= g.shape[1] else x.t().contiguous()


def remainder(g, exact, dtype, steps, **kw):
    """How far X is off where w's rounding does not hide it: w holds minus the rounded X before, so what is stored is what they differ by, in steps of its own size."""
    w = (-exact).to(dtype)
    before = w.double()
    ws = torch.full((B.adatopk_muon_update_workspace_bytes(*g.shape),), 0xFF, dtype=torch.uint8, device="cuda")
    B.adatopk_muon_update(g, None, 0.0, False, w, 1.0, 1.0, ws, steps=steps, **kw)
    return float((w.double() - (before + exact)).norm() / exact.norm())


@pytest.mark.parametrize("steps", [4, 5, 6, 8, 12])
@pytest.mark.parametrize("kind", GRADIENTS)
@pytest.mark.parametrize("size", SIZES)
def test_16_bit_weights_get_an_update_of_all_bits(size, kind, steps):
    gen = torch.Generator(device="cuda").manual_seed(sum(size) + steps)
    g = GRADIENTS[kind](gen, *size)
    exact, single = orthogonalised(g.double(), steps), orthogonalised(g, steps).double()
    # The pairs carry 22 bits where fp32 has 24: four times what that is off by, and where fp32 happens to be nearer a singular value's own way, six roundings of
    # 2^-22 in each of five steps, which grow by 1.6 in each step behind the fifth (as in test_gpu_muon.py).
    bound = 4 * float((single - exact).norm() / exact.norm()) + 64 * 2.0 ** -22 * max(1.0, 1.6 ** (steps - 5))
    for dtype in (BF16, F16):
        # what is stored is at most half a step of X and the error itself, rounded to half of its own step (or of the smallest one)
        stored = ref.HALF_ULP[dtype] * (ref.HALF_ULP[dtype] + bound) * 1.01 + ref.SMALLEST[dtype] / 2 * exact.numel() ** 0.5 / float(exact.norm())
        assert remainder(g, exact, dtype, steps) <= bound + stored, dtype


@pytest.mark.parametrize("steps", [5, 6, 8, 12])
@pytest.mark.parametrize("kind", ["noise", "rank 16 and noise"])
@pytest.mark.parametrize("size", SIZES[1:])
def test_coarse_steps_are_those_of_small_singular_values(size, kind, steps):
    g = GRADIENTS[kind](torch.Generator(device="cuda").manual_seed(sum(size) + steps), *size)
    exact, single = orthogonalised(g.double(), steps), orthogonalised(g, steps).double()
    s = np.linalg.svd(g.double().cpu().numpy(), compute_uv=False)
    s /= np.sqrt((s * s).sum())
    # A product of 11 bits puts in 2^-11 of what its terms b x^3 and c x^5 are (2^-12 from either factor); the two steps of fp16 weights are the first, and like every error theirs
    # grows by 1.6 in each step behind the fifth.
    coarse = 0.0
    for _ in range(2):
        following = 3.4445 * s - 4.7750 * s ** 3 + 2.0315 * s ** 5
        coarse += 2.0 ** -11 * np.linalg.norm(4.7750 * s ** 3 + 2.0315 * s ** 5) / np.linalg.norm(following)
        s = following
    growth = max(1.0, 1.6 ** (steps - 5))
    bound = 4 * float((single - exact).norm() / exact.norm()) + (64 * 2.0 ** -22 + coarse) * growth
    stored = ref.HALF_ULP[F16] * (ref.HALF_ULP[F16] + bound) * 1.01 + ref.SMALLEST[F16] / 2 * exact.numel() ** 0.5 / float(exact.norm())
    assert remainder(g, exact, F16, steps, coarse=True) <= bound + stored
