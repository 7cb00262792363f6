"""What the calls of the orthogonalised update refuse.  Those marked gpu need a device for the extension to read the arguments."""
import pytest
import torch

from paper_2410_12707_amd import binding as B

OK, EINVAL, EWORKSPACE = 0, 1, 2
P, WS = 0x10000, 0x100000  # never dereferenced
F32, BF16 = 0, 1


class Fake:
    """What the binding looks at in a tensor on the device, from one in host memory."""

    is_cuda = True

    def __init__(self, t):
        self.shape, self.dtype, self._t = t.shape, t.dtype, t

    def __getattr__(self, name):
        return getattr(self._t, name)


def test_the_coarse_call_refuses_what_the_other_does():
    lib = B.load_library()
    names = ["g", "gs", "gdt", "m", "mu", "nesterov", "rows", "cols", "steps", "eps", "w", "ws_", "dt", "scale", "decay", "ws", "bytes", "st"]
    need = lib.adatopk_muon_update_workspace_bytes(48, 64)
    good = dict(zip(names, [P, 64, F32, P, 0.9, 1, 48, 64, 5, 1e-7, P, 64, BF16, -0.1, 0.9, WS, need, None]))

    def f(**kw):
        return lib.adatopk_muon_update_coarse(*(dict(good, **kw)[k] for k in names))

    for bad in (dict(gdt=3), dict(dt=3), dict(rows=-1), dict(cols=65537, gs=65537, ws_=65537), dict(steps=0), dict(steps=65), dict(eps=-1.0), dict(eps=float("nan")), dict(g=None),
                dict(g=P + 2), dict(gs=63), dict(w=None), dict(w=P + 1), dict(ws_=63), dict(m=P + 2), dict(ws=None), dict(ws=WS + 16)):
        assert f(**bad) == EINVAL, bad
    assert f(bytes=need - 1) == EWORKSPACE
    assert f(rows=0, g=None, w=None) == OK


# the momentum goes along with w's rows: of another shape it would be read, and written, in an order of its own
WRONG, RIGHT = [(64, 48), (48 * 64 - 1,), (48, 8, 8), (96, 32), (48, 65)], [(48, 64), (48 * 64,), (6, 8, 64)]


def test_a_momentum_of_another_shape(monkeypatch):
    monkeypatch.setattr(B, "_marshal", False)
    monkeypatch.setattr(B, "_stream", lambda: None)
    g, w, small = Fake(torch.zeros(48, 64)), Fake(torch.zeros(48, 64)), Fake(torch.zeros(16, dtype=torch.uint8))
    for shape in WRONG:
        with pytest.raises(ValueError, match="momentum must be float32 with 48 rows of 64"):
            B.adatopk_muon_update(g, Fake(torch.zeros(shape)), 0.9, True, w, 1.0, 0.0, small)
    with pytest.raises(ValueError, match="momentum must be"):
        B.adatopk_muon_update(g, Fake(torch.zeros(48, 64, dtype=torch.float64)), 0.9, True, w, 1.0, 0.0, small)
    for shape in RIGHT:  # what is refused then is the workspace
        with pytest.raises(B.AdaTopKError):
            B.adatopk_muon_update(g, Fake(torch.zeros(shape)), 0.9, True, w, 1.0, 0.0, small)


@pytest.mark.gpu
@pytest.mark.parametrize("extension", [True, False])
def test_a_momentum_of_another_shape_on_the_device(extension, monkeypatch):
    if extension:
        assert B._load_marshal() is not None
    else:
        monkeypatch.setattr(B, "_marshal", False)
    g, w = torch.randn(48, 64, device="cuda"), torch.zeros(48, 64, device="cuda")
    ws = torch.empty(B.adatopk_muon_update_workspace_bytes(48, 64), dtype=torch.uint8, device="cuda")
    for shape in WRONG:
        m = torch.zeros(shape, device="cuda")
        with pytest.raises(ValueError, match="momentum must be float32 with 48 rows of 64"):
            B.adatopk_muon_update(g, m, 0.9, True, w, 1.0, 0.0, ws)
        assert not bool(m.any()) and not bool(w.any())
    for turned in (torch.zeros(64, 48, device="cuda").t(), torch.zeros(48, 65, device="cuda")[:, :64]):  # rows of w's, but not one behind the other
        with pytest.raises(ValueError):
            B.adatopk_muon_update(g, turned, 0.9, True, w, 1.0, 0.0, ws)
    out = []
    for shape in RIGHT:
        m = torch.zeros(shape, device="cuda")
        B.adatopk_muon_update(g, m, 0.9, True, w, 1.0, 0.0, ws)
        out.append(w.clone())
        assert torch.equal(m.view(48, 64), g)
    assert torch.equal(out[0], out[1]) and torch.equal(out[0], out[2])
