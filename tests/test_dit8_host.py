"""The autograd side of the DiT's 8-bit layers on the CPU, with plain products in place of the kernels."""
import pytest
import torch

from paper_2607_05711_amd import dit

BF, F32 = torch.bfloat16, torch.float32


class Plain:
    """What the layers call, in fp32 without quantization."""
    FT_ACT_GELU, FT_PROJ_R_BY_COLS = 1, 1

    @staticmethod
    def ft_quantize_blockwise(w, block_rows):
        return w.float(), None, None

    @staticmethod
    def ft_quantize8(x, proj, proj_layout=0):
        return x.float(), None, x.float() @ (proj.float().T if proj_layout else proj.float()), None

    @staticmethod
    def ft_linear8_fwd(x, _, w, __, P, U, bias, act=0, want_z=False):
        z = x @ w.T + P @ U.float() + bias.float()
        y = torch.nn.functional.gelu(z, approximate="tanh") if act else z
        return (y.to(BF), z.to(BF)) if want_z else y.to(BF)

    @staticmethod
    def ft_linear8_bwd_input(g, _, w, __, Qp, D, z=None, act=0):
        d = g @ w + Qp @ D.float().T
        if act:
            with torch.enable_grad():
                z = z.float().requires_grad_(True)
                d = d * torch.autograd.grad(torch.nn.functional.gelu(z, approximate="tanh").sum(), z)[0]
        return d.to(BF)

    @staticmethod
    def ft_lora_grads(x, dy, P, Qp, r, col0):
        return x.float().T @ Qp[:, col0:], P[:, col0:].T @ dy.float()


@pytest.fixture(params=[dit.FourTuneLinear8, dit.FourTuneMLP8])
def layer(request, monkeypatch):
    monkeypatch.setattr(dit, "_lib", Plain)
    g = torch.Generator().manual_seed(1)
    m = request.param(32, 64, 4, 4, g, "cpu")
    with torch.no_grad():
        for p in m.parameters():
            p.normal_(0.0, 0.1, generator=g)
    m.sync()
    return m


def data(seed=2):
    return torch.randn((5, 32), generator=torch.Generator().manual_seed(seed)).to(BF).requires_grad_(True)


def test_second_derivatives_are_refused(layer):
    """The gradient is no function that can be differentiated again: a sum with it must not lose its part."""
    x = data()
    y = layer(x).float().sum()
    g, = torch.autograd.grad(y, x, create_graph=True)
    with pytest.raises(RuntimeError, match="first derivatives only"):
        (y + g.float().square().sum()).backward()


def test_first_derivatives_under_create_graph(layer):
    """create_graph alone changes nothing, with an input whose rows are out of order too."""
    x = data()
    for t in (x, x.detach().T.contiguous().T.requires_grad_(True)):
        leaves = (t,) + tuple(layer.parameters())
        want = torch.autograd.grad(layer(t).float().square().sum(), leaves)
        got = torch.autograd.grad(layer(t).float().square().sum(), leaves, create_graph=True)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        with pytest.raises(RuntimeError, match="first derivatives only"):
            got[0].float().sum().backward()


def test_factors_changed_before_the_backward(layer):
    """Gradients are those of the factors that the forward used: refreshed ones in between are refused."""
    x = data()
    y = layer(x)
    with torch.no_grad():
        for p in layer.parameters():
            p.mul_(2.0)
    layer.sync()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.float().sum().backward()
    y = layer(x)                                              # and a new forward takes the new ones
    y.float().sum().backward()
    assert all(p.grad is not None for p in layer.parameters())


def test_backward_captured_beside_an_eager_graph(layer, monkeypatch):
    """A parameter's accumulation stays on the stream of its first live graph, and the default stream cannot be captured:
    refused before any work is sent there, and only then."""
    now = {"default": True, "capturing": False}
    monkeypatch.setattr(dit, "_on_default_stream", lambda device: now["default"], raising=False)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: now["capturing"])
    x, leaves = data(), tuple(layer.parameters())

    def captured():
        now.update(default=False, capturing=True)
        try:
            return torch.autograd.grad(layer(x).float().sum(), (x,) + leaves)
        finally:
            now.update(default=True, capturing=False)

    held = layer(x).float().sum()                             # an eager step's loss, kept
    with pytest.raises(RuntimeError, match="default stream"):
        captured()
    held.backward()                                           # its graph is of use still, and lives on
    with pytest.raises(RuntimeError, match="default stream"):
        captured()
    del held
    want = captured()
    with torch.no_grad():
        kept = layer(x)                                       # has no graph
    now["default"] = False
    beside = layer(x)                                         # an eager graph on a stream of its own
    for a, b in zip(captured(), want):
        assert torch.equal(a, b)
    assert kept.shape == beside.shape
