"""The calls around projections in 8-bit floating point together: as a training step uses them, under graph capture, on streams of their own, with and without the
extension, and at the edges of what their description allows."""
import numpy as np
import pytest
import torch

import fp8_reference as fp8
import stage_reference as ref
from paper_2410_12707_amd import binding as B
from paper_2410_12707_amd import stage_example as ex

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.fixture(params=[True, False], ids=["extension", "python"])
def either_way(request, monkeypatch):
    """The calls with their arguments read by the extension, and by Python."""
    if request.param:
        assert B._load_marshal() is not None
    else:
        monkeypatch.setattr(B, "_marshal", False)


def autograd_reference(stage, xs, ds):
    """The stage's step in 64 bits with everything kept as it is: outputs, input gradients, weight gradients."""
    p = {name: getattr(stage, name).double().clone().requires_grad_() for name in stage.grad if name != "bias"}
    outs, dxs = [], []
    for x, d in zip(xs, ds):
        x = x.double().clone().requires_grad_()
        a = x / torch.sqrt((x * x).mean(1, keepdim=True) + ex.EPS) * p["weight"]
        z = a @ p["w1"].t() + p["b1"]
        g = 0.5 * z * (1 + torch.tanh((2 / np.pi) ** 0.5 * (z + 0.044715 * z ** 3)))
        out = x + g @ p["w2"].t() + p["b2"]
        out.backward(d.double())
        outs.append(out.detach())
        dxs.append(x.grad)
    return outs, dxs, {name: t.grad for name, t in p.items()}


def near(got, want, bound):
    return float((got.double() - want).norm() / want.norm()) < bound


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_a_training_step_against_autograd(dtype):
    # e4m3 holds a number to half a step of 2^-3 of its power of two: 2^-4 / sqrt 3, 3.6 percent in the root mean square at the worst place, and a product has
    # two such factors: 5.1 percent.  The longest way, to dW1 and dx, passes four of them (z, whose error the slope of GELU hands on, dg and then dW1 or da, g and
    # out beside them): 5.1 * sqrt 4 = 10.2 percent; 8-bit activations, 16-bit roundings and the links at ratio 1 add a percent or two in the root mean square: 12
    tokens, features, hidden, micro = 200, 96, 288, 3
    stage = ex.EightBitStage(features, hidden, tokens, micro, dtype, seed=1)
    gen = torch.Generator(device="cuda").manual_seed(2)
    xs = [torch.randn(tokens, features, device="cuda", generator=gen).to(dtype) for _ in range(micro)]
    ds = [(torch.randn(tokens, features, device="cuda", generator=gen) * 0.1).to(dtype) for _ in range(micro)]
    outs, dxs = ex.train_step(stage, xs, ds, ex.Link(tokens * features, 1.0, dtype), ex.Link(tokens * features, 1.0, dtype))
    want = autograd_reference(stage, xs, ds)
    for m in range(micro):
        assert near(outs[m], want[0][m], 0.12) and near(dxs[m], want[1][m], 0.12)
    for name, g in want[2].items():
        assert near(stage.grad[name], g, 0.12), name
    assert bool((stage.grad["bias"] == 0).all())
    before = {name: getattr(stage, name).double().clone() for name in stage.eight}
    stage.update(rate=0.02, decay=0.1, mu=0.9)
    for name, (straight, across) in stage.eight.items():
        w, g = getattr(stage, name), stage.grad[name]
        assert torch.equal(stage.momentum[name], g)  # which was nothing before
        u = (g.double() + float(np.float32(0.9)) * g.double())
        x = u if u.shape[0] <= u.shape[1] else u.t().contiguous()
        x = x / (x.norm() + 1e-7)
        for _ in range(5):
            gram = x @ x.t().contiguous()
            x = 3.4445 * x + (-4.7750 * gram + 2.0315 * (gram @ gram)) @ x
        step = -0.02 * (x if u.shape[0] <= u.shape[1] else x.t())
        slack = float(step.norm()) * 1e-4  # (of sides below 256 the update has some 20 bits)
        want_w = before[name] * (1 - 0.02 * 0.1) + step
        assert bool(((w.double() - want_w).abs() <= slack + (ref.HALF_ULP[dtype] + 8 * ref.U) * (want_w.abs() + step.abs() + slack)).all())
        again = B.new_fp8(*w.shape), B.new_fp8(*reversed(w.shape))
        B.adatopk_fp8_store_weight(w, *again)
        back = [torch.empty(*shape, device="cuda") for shape in (w.shape, w.shape, w.shape[::-1], w.shape[::-1])]
        for buffer, to in zip((straight, again[0], across, again[1]), back):
            B.adatopk_fp8_load(buffer, to)
        assert torch.equal(back[0], back[1]) and torch.equal(back[2], back[3]) and torch.equal(back[0].t(), back[2])


def test_the_example_runs(capsys):
    ex.main(features=192, hidden=320, tokens=130, micro_batches=2, eight_bit=True)
    ex.main(features=192, hidden=320, tokens=130, micro_batches=2)
    said = capsys.readouterr().out.splitlines()
    assert len(said) == 2 and "in 8 bits:" in said[0] and "in 8 bits:" not in said[1]


def buffers(rows, cols, hidden, dtype):
    new = lambda *s, d=dtype: torch.empty(*s, dtype=d, device="cuda")  # noqa: E731
    ws = max(B.adatopk_rmsnorm_backward_workspace_bytes(rows, cols), B.adatopk_weight_grad_workspace_bytes(rows, hidden, cols, dtype), 256,
             B.adatopk_fp8_product_workspace_bytes(rows, hidden, cols), B.adatopk_fp8_product_workspace_bytes(rows, cols, hidden), B.adatopk_muon_update_workspace_bytes(hidden, cols))
    return {"x": new(rows, cols), "r": new(rows, cols), "dz": new(rows, hidden), "weight": new(cols), "b": new(hidden), "w": new(hidden, cols), "m": new(hidden, cols, d=F32),
            "s": new(rows, cols), "y": new(rows, cols), "rstd": new(rows, d=F32), "z": new(rows, hidden), "da": new(rows, cols), "dx": new(rows, cols),
            "gweight": new(cols, d=F32), "dw": new(hidden, cols, d=F32), "db": new(hidden, d=F32), "back": new(rows, cols), "wback": new(cols, hidden),
            "h8": B.new_act8(rows, cols), "y8": B.new_fp8(rows, cols), "dz8": B.new_fp8(rows, hidden), "w8": B.new_fp8(hidden, cols), "wt8": B.new_fp8(cols, hidden),
            "ws": torch.empty(ws, dtype=torch.uint8, device="cuda")}


INPUTS, OUTPUTS = ("x", "r", "dz", "weight", "b", "w", "m"), ("s", "y", "rstd", "z", "da", "dx", "gweight", "dw", "db", "back", "wback", "w", "m")


def fill(t, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    for name in INPUTS:
        t[name].copy_(torch.randn(t[name].shape, device="cuda", generator=gen))


def everything(t):
    (rows, cols), hidden = t["x"].shape, t["w"].shape[0]
    B.adatopk_fp8_store_weight(t["w"], t["w8"], t["wt8"])
    B.adatopk_rmsnorm_forward(t["x"], t["weight"], 1e-5, t["y"], t["rstd"], residual=t["r"], sum_out=t["s"], act8=t["h8"], fp8=t["y8"])
    B.adatopk_fp8_load(t["y8"], t["back"])
    B.adatopk_fp8_product(t["y8"], t["w8"], cols, t["z"], t["ws"], bias=t["b"], add=t["dz"])
    B.adatopk_fp8_store(t["dz"], t["dz8"])
    B.adatopk_fp8_product(t["dz8"], t["wt8"], hidden, t["da"], t["ws"])
    B.adatopk_rmsnorm_backward(t["da"], None, t["h8"], t["rstd"], t["weight"], t["dx"], t["gweight"], t["ws"], dsum=t["r"])
    B.adatopk_weight_grad(t["dz"], t["h8"], t["dw"], t["db"], t["ws"], weight=t["weight"])
    B.adatopk_muon_update(t["dw"], t["m"], 0.9, True, t["w"], -0.02, 0.99, t["ws"])
    B.adatopk_fp8_store_weight(t["w"], t["w8"], t["wt8"])
    B.adatopk_fp8_load(t["wt8"], t["wback"])
    return [t[k] for k in OUTPUTS]


SHAPES = [(1, 130, 72), (35, 5256, 70), (300, 768, 516), (1500, 1601, 260)]


@pytest.mark.parametrize("rows,cols,hidden", SHAPES)
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_graph_capture_and_replay(dtype, rows, cols, hidden):
    t = buffers(rows, cols, hidden, dtype)
    wanted = []
    for seed in range(3):
        fill(t, seed)
        wanted.append([v.clone() for v in everything(t)])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = everything(t)
    for rep in range(6):  # replays with eager work and synchronisation in between
        for v in outs:
            v.fill_(7.0)
        fill(t, rep % 3)
        for name in ("ws", "y8", "dz8", "w8", "wt8", "h8"):
            t[name].fill_(0x55)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, wanted[rep % 3])), rep


def test_two_graphs_with_one_workspace():
    sets = [buffers(200, 640, 260, BF16), buffers(520, 300, 700, F32)]
    shared = max((t["ws"] for t in sets), key=torch.Tensor.numel)
    graphs, wanted = [], []
    for i, t in enumerate(sets):
        t["ws"] = shared
        fill(t, i)
        wanted.append([v.clone() for v in everything(t)])
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            everything(t)
    for _ in range(3):
        for i, t in enumerate(sets):
            fill(t, i)
        for graph in graphs:  # one behind the other on a stream
            graph.replay()
        torch.cuda.synchronize()
        for t, want in zip(sets, wanted):
            assert all(torch.equal(t[k], b) for k, b in zip(OUTPUTS, want))


def test_two_streams_with_their_own_workspaces():
    sets = [buffers(1000, 640, 260, BF16) for _ in range(2)]
    wanted = []
    for i, t in enumerate(sets):
        fill(t, i)
        wanted.append([v.clone() for v in everything(t)])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(4):
        for i, t in enumerate(sets):
            fill(t, i)
        torch.cuda.synchronize()
        for t, st in zip(sets, streams):
            with torch.cuda.stream(st):
                everything(t)
        torch.cuda.synchronize()
        for t, want in zip(sets, wanted):
            assert all(torch.equal(t[k], b) for k, b in zip(OUTPUTS, want))


def test_calls_with_and_without_the_extension(monkeypatch):
    t = buffers(257, 331, 70, F16)
    fill(t, 9)
    with_it = [v.clone() for v in everything(t)]

    def refused():
        said = []
        for call in (lambda: B.adatopk_fp8_store(t["x"], t["y8"][:-4]), lambda: B.adatopk_fp8_load(t["y8"], t["z"].new_empty(4000, 331)),
                     lambda: B.adatopk_fp8_store_weight(t["w"], t["w8"], t["wt8"][:64]), lambda: B.adatopk_fp8_product(t["y8"], t["w8"][:64], 331, t["z"], t["ws"]),
                     lambda: B.adatopk_fp8_product(t["y8"], t["w8"], 331, t["z"], t["ws"], bias=t["b"][:3]),
                     lambda: B.adatopk_fp8_product(t["y8"], t["w8"], 331, t["z"], t["ws"], add=t["x"]),
                     lambda: B.adatopk_rmsnorm_forward(t["x"], t["weight"][:5], 1e-5, t["y"], None), lambda: B.adatopk_rmsnorm_forward(t["x"], None, 1e-5, None, None),
                     lambda: B.adatopk_rmsnorm_backward(t["da"], t["x"], t["h8"], t["rstd"], None, t["dx"], None, None),
                     lambda: B.adatopk_rmsnorm_backward(t["da"], t["x"], None, t["rstd"], None, t["dx"], t["gweight"], t["ws"][1:]),
                     lambda: B.adatopk_muon_update(t["dw"], t["m"], 0.9, True, t["w"], 1.0, 0.0, t["ws"][:256]),
                     lambda: B.adatopk_muon_update(t["dw"], t["dw"], 0.9, True, t["w"].t(), 1.0, 0.0, t["ws"])):
            with pytest.raises((ValueError, B.AdaTopKError)) as e:
                call()
            said.append((type(e.value), str(e.value)))
        return said

    said = refused()
    monkeypatch.setattr(B, "_marshal", False)
    fill(t, 9)
    assert all(torch.equal(a, b) for a, b in zip(everything(t), with_it)) and refused() == said


def test_weights_that_are_parameters(either_way):
    x, y, z = torch.randn(12, 64, device="cuda"), torch.empty(12, 64, device="cuda"), torch.empty(12, 64, device="cuda")
    w = torch.nn.Parameter(torch.randn(64, device="cuda"))
    B.adatopk_rmsnorm_forward(x, w, 1e-5, y, None)
    B.adatopk_rmsnorm_forward(x, w.detach().clone(), 1e-5, z, None)
    assert torch.equal(y, z)
    p = torch.nn.Parameter(torch.randn(40, 64, device="cuda"))
    kept, g, ws = p.detach().clone(), torch.randn(40, 64, device="cuda"), torch.empty(B.adatopk_muon_update_workspace_bytes(40, 64), dtype=torch.uint8, device="cuda")
    for w in (p, kept):
        B.adatopk_muon_update(g, None, 0.0, False, w, -0.1, 1.0, ws)
    assert torch.equal(p.detach(), kept)
    buffers = [B.new_fp8(40, 64) for _ in range(2)]
    for w, buffer in zip((p, kept), buffers):
        buffer.fill_(0)
        B.adatopk_fp8_store_weight(w, buffer)
    assert torch.equal(*buffers)


def test_the_measuring_build_has_the_calls():
    t = buffers(100, 96, 40, BF16)
    fill(t, 4)
    want = [v.clone() for v in everything(t)]
    with B.measuring():
        fill(t, 4)
        assert all(torch.equal(a, b) for a, b in zip(everything(t), want))


@pytest.mark.parametrize("shape", [(0, 64), (3, 0), (3, 0, 64), (0, 3, 64), (2, 3, 0), (0, 0, 64)])
def test_tensors_without_elements(shape, either_way):
    rows, cols = int(torch.Size(shape[:-1]).numel()), shape[-1]
    for x in (torch.empty(shape, device="cuda"), torch.empty(tuple(size + 2 for size in shape), device="cuda")[tuple(slice(0, size) for size in shape)]):
        buffer, f = torch.full((16,), 7, dtype=torch.uint8, device="cuda"), torch.full((rows,), 3.0, device="cuda")
        ws = torch.empty(1 << 16, dtype=torch.uint8, device="cuda")
        B.adatopk_fp8_store(x, buffer)
        B.adatopk_fp8_load(buffer, x)
        B.adatopk_rmsnorm_forward(x, None, 1e-5, x, f, residual=x, sum_out=x, act8=buffer, fp8=buffer)
        dw = torch.full((cols,), 3.0, device="cuda")
        for source in ((x, None), (None, buffer)):
            B.adatopk_rmsnorm_backward(x, *source, f, None, x, dw, ws, accumulate=True)
            assert bool((dw == 3.0).all())
        B.adatopk_rmsnorm_backward(x, x, None, f, None, x, dw, ws)
        assert bool((dw == 0.0).all())
        if x.dim() == 2:
            B.adatopk_fp8_store_weight(x, buffer, buffer)
            B.adatopk_muon_update(x, None, 0.0, False, x, 1.0, 0.0, ws)
            B.adatopk_fp8_product(B.new_fp8(rows, 32), B.new_fp8(cols, 32), 32, x, ws)
        torch.cuda.synchronize()
        assert bool((buffer == 7).all())


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("rows", [3, 20, 100, 700])
def test_products_with_the_identity_are_what_is_held(dtype, rows):
    # one product a sum, so nothing is cut off: y is the numbers themselves, every byte there is among them, subnormals and negative zeros too, at 29 scales
    n = 260
    q = torch.arange(rows * n, device="cuda").view(rows, n) * 7 % 254
    q = torch.where(q >= 127, q + 1, q)  # (without the two that are no numbers)
    values = q.to(torch.uint8).view(torch.float8_e4m3fn).float() * torch.exp2(torch.arange(rows, device="cuda") % 29 - 14.0)[:, None]
    values[:, ::128] = 448 * torch.exp2(torch.arange(rows, device="cuda") % 29 - 14.0)[:, None]  # which fixes the scales
    x, eye, back, y = B.new_fp8(rows, n), B.new_fp8(n, n), torch.empty(rows, n, device="cuda"), torch.empty(rows, n, dtype=dtype, device="cuda")
    B.adatopk_fp8_store(values, x)
    B.adatopk_fp8_load(x, back)
    assert torch.equal(back, values)
    B.adatopk_fp8_store_weight(torch.eye(n, device="cuda"), eye)
    B.adatopk_fp8_product(x, eye, n, y, torch.empty(max(B.adatopk_fp8_product_workspace_bytes(rows, n, n), 256), dtype=torch.uint8, device="cuda"))
    assert torch.equal(y, values.to(dtype))


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("rows", [5, 40, 200, 2300])
def test_blocks_that_are_no_numbers_stay_in_their_rows(dtype, rows):
    rng = np.random.default_rng(6)
    n_out = 90 if rows < 2000 else 2049
    x, w = rng.standard_normal((rows, 300)), rng.standard_normal((n_out, 300))
    x[2, 140], x[4, 299], w[3, 5] = np.inf, np.nan, np.nan
    y = torch.empty(rows, n_out, dtype=dtype, device="cuda")
    B.adatopk_fp8_product(torch.from_numpy(fp8.fp8_buffer(ref.rounded(x, F32))).cuda(), torch.from_numpy(fp8.fp8_buffer(ref.rounded(w, F32))).cuda(), 300, y,
                          torch.empty(max(B.adatopk_fp8_product_workspace_bytes(rows, n_out, 300), 256), dtype=torch.uint8, device="cuda"))
    expected = np.zeros((rows, n_out), dtype=bool)
    expected[2], expected[4], expected[:, 3] = True, True, True
    assert np.array_equal(np.isnan(ref.host(y)), expected)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("rows", [2, 40, 150])
def test_scales_from_end_to_end(dtype, rows):
    x, w = np.zeros((rows, 256)), np.zeros((16, 256))
    x[:, 0], w[:, 0] = 2.0 ** 127, 2.0 ** -126
    x[:, 200], w[:, 200] = 2.0 ** -100, 2.0 ** 101
    w[3, 0], w[4, 200] = 2.0, 0.0
    y = torch.empty(rows, 16, dtype=dtype, device="cuda")
    B.adatopk_fp8_product(torch.from_numpy(fp8.fp8_buffer(x)).cuda(), torch.from_numpy(fp8.fp8_buffer(w)).cuda(), 256, y, torch.empty(1 << 20, dtype=torch.uint8, device="cuda"))
    expected = x @ w.T
    expected[:, 3] = np.inf
    assert np.array_equal(ref.host(y), expected)


def test_a_weight_that_is_only_written():
    # decay 0: what w held is not looked at, nor is a gradient's or a weight's neighbourhood written
    g, ws = torch.randn(70, 90, device="cuda"), torch.empty(B.adatopk_muon_update_workspace_bytes(70, 90), dtype=torch.uint8, device="cuda")
    w, plain = torch.full((70, 90), float("nan"), device="cuda"), torch.zeros(70, 90, device="cuda")
    for out in (w, plain):
        B.adatopk_muon_update(g, None, 0.0, False, out, 1.0, 0.0, ws)
    assert torch.equal(w, plain)
    kept = g.clone()
    B.adatopk_muon_update(g, None, 0.0, False, w, 0.0, 1.0, ws)  # and one that is left as it is
    assert torch.equal(w, plain) and torch.equal(g, kept)


def test_matrices_past_32_bits():
    rows, cols, some = 140000, 32768, 300
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty(rows, cols, dtype=BF16, device="cuda")
    for top in range(0, rows, 20000):
        x[top:top + 20000].copy_(torch.randn(20000, cols, device="cuda", generator=gen))
    buffer, back, y = B.new_fp8(rows, cols), torch.empty_like(x), torch.empty_like(x)
    last, few = x[-some:].clone(), B.new_fp8(some, cols)
    want = torch.empty_like(last)
    B.adatopk_fp8_store(x, buffer)
    B.adatopk_fp8_load(buffer, back)
    B.adatopk_fp8_store(last, few)
    B.adatopk_fp8_load(few, want)
    assert torch.equal(back[-some:], want)
    # its products with a few features, whose sums may be cut into other shares
    w = torch.randn(40, cols, device="cuda", generator=gen) * cols ** -0.5
    w8, held = B.new_fp8(40, cols), torch.empty(40, cols, device="cuda")
    B.adatopk_fp8_store_weight(w, w8)
    B.adatopk_fp8_load(w8, held)
    z = torch.empty(rows, 40, device="cuda")
    B.adatopk_fp8_product(buffer, w8, cols, z, torch.empty(max(B.adatopk_fp8_product_workspace_bytes(rows, 40, cols), 256), dtype=torch.uint8, device="cuda"))
    a, b = want.double(), held.double()
    bound = (a.abs() @ b.abs().t().contiguous()) * (2 * ref.U * (8 + 2 * cols ** 0.5))
    assert bool(((z[-some:].double() - a @ b.t().contiguous()).abs() <= bound).all())
    # the norm, its backward pass, and what it puts away
    rstd, act8 = torch.empty(rows, device="cuda"), B.new_act8(rows, cols)
    B.adatopk_rmsnorm_forward(x, None, 1e-5, y, rstd, act8=act8, fp8=buffer)
    B.adatopk_fp8_load(buffer, back)
    few_rstd, few_act8 = torch.empty(some, device="cuda"), B.new_act8(some, cols)
    B.adatopk_rmsnorm_forward(last, None, 1e-5, want, few_rstd, act8=few_act8, fp8=few)
    assert torch.equal(y[-some:], want) and torch.equal(rstd[-some:], few_rstd)
    B.adatopk_fp8_load(few, want)
    assert torch.equal(back[-some:], want)
    B.adatopk_rmsnorm_backward(x, None, act8, rstd, None, y, None, None)
    B.adatopk_rmsnorm_backward(last, None, few_act8, few_rstd, None, want, None, None)
    assert torch.equal(y[-some:], want)


def test_weights_past_32_bits():
    rows, cols, some = 70100, 65000, 200
    gen = torch.Generator(device="cuda").manual_seed(2)
    w = torch.empty(rows, cols, dtype=BF16, device="cuda")
    for top in range(0, rows, 10000):
        w[top:top + 10000].copy_(torch.randn(min(10000, rows - top), cols, device="cuda", generator=gen))
    first = rows // 128 * 128 - 128  # where a tile begins
    part = w[first:].clone()
    straight, across, few = B.new_fp8(rows, cols), B.new_fp8(cols, rows), B.new_fp8(*part.shape)
    B.adatopk_fp8_store_weight(w, straight, across)
    B.adatopk_fp8_store_weight(part, few)
    back, want = torch.empty_like(w), torch.empty_like(part)
    B.adatopk_fp8_load(few, want)
    B.adatopk_fp8_load(straight, back)
    assert torch.equal(back[first:], want)
    turned = back.view(cols, rows)
    B.adatopk_fp8_load(across, turned)
    assert torch.equal(turned[-some:, first:], want[:, -some:].t())


def test_an_update_past_32_bits():
    # a gradient of rank one, u v': its one singular value is the polynomial's value at 1, all else of X stays nothing
    rows, cols = 33000, 64001
    gen = torch.Generator(device="cuda").manual_seed(3)
    u, v = torch.randn(rows, 1, device="cuda", generator=gen), torch.randn(1, cols, device="cuda", generator=gen)
    w, ws = torch.empty(rows, cols, device="cuda"), torch.empty(B.adatopk_muon_update_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    B.adatopk_muon_update(u @ v, None, 0.0, False, w, 1.0, 0.0, ws, steps=1)
    factor = (3.4445 - 4.7750 + 2.0315) / (float(u.double().norm()) * float(v.double().norm()))
    # a x, b x^3 and c x^5 are off by some roundings of 2^-22 each: of 10.3 that cancel to 0.7, and of the elements' pairs, of which the smallest lose bits to
    # fp16's subnormals: 2^-25 of 2^14, the size of X's norm
    for rows_of in (slice(0, 500), slice(rows - 500, rows)):
        want = u[rows_of].double() @ v.double() * factor
        assert float((w[rows_of].double() - want).norm() / want.norm()) <= 4 * 10.3 / 0.701 * 2.0 ** -22 + float(2.0 ** -39 * (500 * cols) ** 0.5 / want.norm())
