"""The orthogonalised update of a weight matrix on the GPU, against its definition in 64 bits on the CPU."""
import numpy as np
import pytest
import torch

import stage_reference as ref
from paper_2410_12707_amd import binding as B

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
EPS = 1e-7


def newton_schulz(u, steps, eps=EPS):
    """In u's precision, its shorter side first."""
    x = u if u.shape[0] <= u.shape[1] else u.T
    x = x / (np.sqrt((x.astype(np.float64) ** 2).sum()) + eps).astype(u.dtype)
    a, b, c = (u.dtype.type(v) for v in (3.4445, -4.7750, 2.0315))
    for _ in range(steps):
        gram = x @ x.T
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return x if u.shape[0] <= u.shape[1] else x.T


def off_by(got, exact):
    return np.linalg.norm(got - exact) / np.linalg.norm(exact)


def tolerance(u, exact, steps, dtype=F32):
    """The same steps in fp32 carry 24 bits where the pairs carry 22: four times their distance.  Where fp32 happens to be nearer (the smallest matrices) a singular value's
    own way counts: some six roundings of 2^-22 in each of five steps, their growth by the polynomial's slope of 1 around its values of 0.7 to 1.2.
    Where w has 16 bits and the shorter side 256 or more, some products take 11: a rounding of at most 2^-11 of either factor, 2^-11 / sqrt 3 of both in the root mean square,
    times what the terms of a x + b x^3 + c x^5 are together, 10.3 where x is 1, over the 0.7 that they come to: 4e-3 for the last step's (bf16).  fp16's come
    three steps before the end and leave a x in full, whose other terms are 6.8: 3e-3, of which three steps with slopes of 0.7, 1.1 and 1.3 leave as much."""
    more = {F32: 0.0, F16: 3e-3, BF16: 4e-3}[dtype] if min(u.shape) >= 256 else 0.0
    return 4 * off_by(newton_schulz(u.astype(np.float32), steps).astype(np.float64), exact) + 64 * 2.0 ** -22 + more


def gradient(rng, rows, cols):
    strong = max(1, min(rows, cols) // 16)
    g = rng.standard_normal((rows, strong)) @ rng.standard_normal((strong, cols)) * strong ** -0.5 + 0.5 * rng.standard_normal((rows, cols))
    return ref.rounded(1e-3 * g, F32)


def workspace(rows, cols):
    return torch.full((B.adatopk_muon_update_workspace_bytes(rows, cols),), 0xFF, dtype=torch.uint8, device="cuda")


SHAPES = [(1, 1), (1, 40), (3, 2), (31, 33), (64, 64), (65, 200), (200, 65), (128, 1000), (257, 255), (300, 700), (513, 520), (40, 5000), (2100, 64)]


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("shape", SHAPES)
def test_orthogonalised_gradient(dtype, shape):
    rows, cols = shape
    rng = np.random.default_rng(rows * 10007 + cols)
    g = gradient(rng, rows, cols)
    exact = newton_schulz(g, 5)
    out = torch.full((rows, cols + 3), 7.0, dtype=dtype, device="cuda")
    B.adatopk_muon_update(ref.on_device(g, F32, 5, 1), None, 0.0, False, out[:, :cols], 1.0, 0.0, workspace(rows, cols))
    got = ref.host(out)
    assert off_by(got[:, :cols], exact) <= tolerance(g, exact, 5, dtype) + ref.HALF_ULP[dtype] * 1.01
    assert (got[:, cols:] == 7.0).all()


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("steps", [1, 2, 3, 4, 7])
@pytest.mark.parametrize("shape", [(150, 260), (300, 270)])
def test_steps(dtype, steps, shape):
    g = gradient(np.random.default_rng(steps), *shape)
    exact = newton_schulz(g, steps)
    out = torch.empty(*shape, dtype=dtype, device="cuda")
    B.adatopk_muon_update(ref.on_device(g, F32), None, 0.0, False, out, 1.0, 0.0, workspace(*shape), steps=steps)
    # (the slope at 1.2 is 4, between 0.7 and 1.2 on average below 1.6)
    assert off_by(ref.host(out), exact) <= tolerance(g, exact, steps, dtype) * max(1.0, 1.6 ** (steps - 5)) + ref.HALF_ULP[dtype] * 1.01


def test_singular_values():
    rng = np.random.default_rng(3)
    q, _ = np.linalg.qr(rng.standard_normal((300, 300)))
    p, _ = np.linalg.qr(rng.standard_normal((400, 300)))
    u = ref.rounded(q @ np.diag(np.geomspace(0.02, 1, 300)) @ p.T, F32)
    out = torch.empty(300, 400, device="cuda")
    B.adatopk_muon_update(ref.on_device(u, F32), None, 0.0, False, out, 1.0, 0.0, workspace(300, 400), steps=8)
    s = np.linalg.svd(ref.host(out), compute_uv=False)
    assert s.max() < 1.2025 and s.min() > 0.63
    assert np.abs(ref.host(out) @ p - q @ (q.T @ ref.host(out) @ p) * 1.0).max() < 1e-4  # the same directions


@pytest.mark.parametrize("tile", [(4200, 4100), (1600, 6400), (2500, 1300)])
def test_large_tiles(tile):
    rows, cols = tile
    gen = torch.Generator(device="cuda").manual_seed(rows)
    g = torch.randn(rows, cols, device="cuda", generator=gen)
    out = torch.empty(rows, cols, device="cuda")
    B.adatopk_muon_update(g, None, 0.0, False, out, 1.0, 0.0, workspace(rows, cols), steps=2)
    x = g.double() if rows <= cols else g.double().t().contiguous()

    def steps(x):
        x = x / (x.double().norm() + EPS).to(x.dtype)
        for _ in range(2):
            gram = x @ x.t().contiguous()
            x = 3.4445 * x + (-4.7750 * gram + 2.0315 * (gram @ gram)) @ x
        return x if rows <= cols else x.t()

    exact, single = steps(x), steps(x.float())
    tol = 4 * float((single.double() - exact).norm() / exact.norm()) + 64 * 2.0 ** -22
    assert float((out.double() - exact).norm() / exact.norm()) <= tol
    worst = float((out.double() - exact).abs().max() / exact.pow(2).mean().sqrt())
    assert worst <= 8 * tol * 4  # no element stands out: eight standard deviations of a normal error, four for its size


@pytest.mark.parametrize("nesterov", [False, True])
@pytest.mark.parametrize("grad_dtype,dtype", [(F32, F32), (F32, BF16), (BF16, F16), (F16, BF16)])
@pytest.mark.parametrize("shape", [(70, 131), (131, 70), (260, 400)])
def test_update(nesterov, grad_dtype, dtype, shape):
    rng = np.random.default_rng(11)
    g, m = ref.rounded(gradient(rng, *shape), grad_dtype), ref.rounded(1e-2 * rng.standard_normal(shape), F32)
    w = ref.rounded(0.05 * rng.standard_normal(shape), dtype)
    wide = torch.full((shape[0], shape[1] + 8), 7.0, dtype=dtype, device="cuda")
    view, momentum = wide[:, :shape[1]], torch.from_numpy(m).float().cuda()
    view.copy_(torch.from_numpy(w).to(dtype))
    B.adatopk_muon_update(ref.on_device(g, grad_dtype, 2), momentum, 0.95, nesterov, view, -0.02, 0.998, workspace(*shape))
    mu, decay, scale = (float(np.float32(v)) for v in (0.95, 0.998, -0.02))
    after = mu * m + g
    got = ref.host(momentum).reshape(shape)
    assert (np.abs(got - after) <= ref.U * np.abs(after)).all()
    u = g + mu * got if nesterov else got
    exact = newton_schulz(u, 5)
    expected = decay * w + scale * exact
    slack = np.abs(scale) * (tolerance(u, exact, 5, dtype) + 2 * ref.U) * np.linalg.norm(exact)  # (of any one element at most that of all)
    bound = slack + 4 * ref.U * (np.abs(w) + np.abs(scale * exact)) + ref.HALF_ULP[dtype] * (np.abs(expected) + slack) + ref.SMALLEST[dtype]
    assert (np.abs(ref.host(wide)[:, :shape[1]] - expected) <= bound).all()
    assert (ref.host(wide)[:, shape[1]:] == 7.0).all()


def test_equal_calls_give_equal_bits():
    g = torch.randn(500, 333, device="cuda")
    out, ws = [torch.empty(500, 333, device="cuda") for _ in range(2)], workspace(500, 333)
    for o in out:
        B.adatopk_muon_update(g, None, 0.0, False, o, 1.0, 0.0, ws)
    assert torch.equal(*out)


def test_gradients_of_any_size():
    g = torch.randn(90, 120, device="cuda")
    outs = []
    for size in (1.0, 2.0 ** 60, 2.0 ** -60, 2.0 ** -100):
        out = torch.empty(90, 120, device="cuda")
        B.adatopk_muon_update(g * size, None, 0.0, False, out, 1.0, 0.0, workspace(90, 120), eps=0.0)
        outs.append(out)
    assert all(torch.equal(outs[0], o) for o in outs[1:])
    w = torch.randn(90, 120, device="cuda")
    kept, before = w.clone(), torch.zeros(90, 120, device="cuda")
    B.adatopk_muon_update(before, None, 0.0, False, w, -1.0, 1.0, workspace(90, 120))  # no gradient, no change
    assert torch.equal(w, kept)
    for bad in (float("nan"), float("inf")):
        g[7, 11] = bad
        B.adatopk_muon_update(g, None, 0.0, False, w, 1.0, 0.0, workspace(90, 120))
        assert torch.isnan(w).all()


def test_empty():
    ws = torch.empty(256, dtype=torch.uint8, device="cuda")
    for shape in ((0, 4), (4, 0)):
        B.adatopk_muon_update(torch.empty(shape, device="cuda"), None, 0.0, False, torch.empty(shape, device="cuda"), 1.0, 0.0, ws)
