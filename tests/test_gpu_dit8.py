"""The DiT's layers on MXFP8 activations and gradients: outputs and gradients of
the modules against the layer in 64 bits, and a training step."""
import pytest
import torch

from paper_2607_05711_amd import dit
from tests import _mx8 as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def layers64(m):
    """The layer's weight, stabilizer and adapters in 64 bits, the adapters as leaves."""
    A, B = (t.detach().to(torch.bfloat16).double().requires_grad_(True) for t in (m.A, m.B))
    return ref.values4(m.wq, m.ws), m.D[:, :m.rs].double(), m.U[:m.rs].double(), A, B, m.bias.double()


def linear64(x, p):
    W, L1, L2, A, B, b = p
    return x @ W.T + x @ L1 @ L2 + x @ A @ B + b


def rel(got, want):
    return float((got.detach().double() - want.detach()).norm() / want.detach().norm())


def filled(m, g):
    for l in m.modules():
        if isinstance(l, dit.FourTuneLinear):
            with torch.no_grad():
                l.B.normal_(0.0, 0.02, generator=g)
                l.sync()
    return m


# An E4M3 rounding is off by at most 2^-4 of a value, 0.036 root mean square, in each of a product's independent
# terms: its result by as much of itself in the 2-norm, the adapter gradients by their factors' 2^-17 and bf16 inputs.
@pytest.mark.parametrize("T", [1, 70, 512])
def test_linear(T):
    g = ref.gen(T)
    m = filled(dit.FourTuneLinear8(256, 416, 16, 16, g, DEV), g)
    x = ref.normal(g, T, 256).requires_grad_(True)
    dy = ref.normal(g, T, 416)
    y = m(x)
    y.backward(dy)
    p, x64 = layers64(m), x.detach().double().requires_grad_(True)
    y64 = linear64(x64, p)
    y64.backward(dy.double())
    assert rel(y, y64) < 0.04 and rel(x.grad, x64.grad) < 0.04
    assert rel(m.A.grad, p[3].grad) < 1e-3 and rel(m.B.grad, p[4].grad) < 1e-3


def test_mlp():
    """Two roundings in a row, and the activation's input off by the first's: sqrt(2) and twice the linear's."""
    g = ref.gen(3)
    m = filled(dit.FourTuneMLP8(256, 1024, 16, 16, g, DEV), g)
    x = ref.normal(g, 2, 75, 256).requires_grad_(True)
    dy = ref.normal(g, 2, 75, 256)
    y = m(x)
    y.backward(dy)
    p1, p2, x64 = layers64(m.fc1), layers64(m.fc2), x.detach().double().requires_grad_(True)
    y64 = linear64(torch.nn.functional.gelu(linear64(x64, p1), approximate="tanh"), p2)
    y64.backward(dy.double())
    assert y.shape == y64.shape and rel(y, y64) < 0.057
    for got, want in ((x.grad, x64.grad), (m.fc1.A.grad, p1[3].grad), (m.fc1.B.grad, p1[4].grad), (m.fc2.A.grad, p2[3].grad),
                      (m.fc2.B.grad, p2[4].grad)):
        assert rel(got, want) < 0.08


def test_step_runs():
    cfg = dit.DiTConfig(hidden=256, heads=2, mlp=1024, double_blocks=1, single_blocks=1, img_tokens=64, txt_tokens=33,
                        lora_rank=16, stab_rank=16)
    model = dit.DiT(cfg, "fp8", 1, DEV)
    trainer = dit.Trainer(model)
    batch = dit.synthetic_batch(cfg, 2, DEV)
    for _ in range(2):
        assert bool(trainer.step(*batch).isfinite())
    for p in trainer.params:
        assert p.grad is not None and bool(p.grad.isfinite().all())


def test_input_without_gradient():
    g = ref.gen(5)
    m = dit.FourTuneLinear8(64, 96, 16, 16, g, DEV)
    m(ref.normal(g, 9, 64)).sum().backward()
    assert m.A.grad is not None and m.B.grad.abs().sum() > 0


def test_no_tokens():
    g = ref.gen(6)
    m = dit.FourTuneMLP8(64, 96, 16, 16, g, DEV)
    x = torch.empty((2, 0, 64), dtype=torch.bfloat16, device=DEV, requires_grad=True)
    y = m(x)
    y.backward(torch.empty_like(y))
    assert y.shape == (2, 0, 64) and x.grad.shape == x.shape
    for p in m.parameters():
        assert bool((p.grad == 0).all())                      # sums over no tokens


def test_strided_input_and_gradient():
    g = ref.gen(7)
    m = filled(dit.FourTuneLinear8(128, 96, 16, 16, g, DEV), g)
    x, dy = ref.normal(g, 40, 3, 128), ref.normal(g, 96)
    a = x.transpose(0, 1).requires_grad_(True)                # rows out of order
    b = x.transpose(0, 1).contiguous().requires_grad_(True)
    got = torch.autograd.grad(m(a), (a, m.A, m.B), dy.expand(3, 40, 96))
    want = torch.autograd.grad(m(b), (b, m.A, m.B), dy.expand(3, 40, 96).contiguous())
    for s, t in zip(got, want):
        assert torch.equal(s, t)


def test_step_in_a_graph():
    """Forward and backward of a layer and an MLP, captured: every replay on new inputs equals the eager step."""
    g = ref.gen(8)
    m, f = filled(dit.FourTuneLinear8(256, 128, 16, 16, g, DEV), g), filled(dit.FourTuneMLP8(128, 416, 16, 16, g, DEV), g)
    leaves = tuple(p for l in (m, f) for p in l.parameters())
    x, dy = ref.normal(g, 70, 256).requires_grad_(True), ref.normal(g, 70, 128)

    def step():
        y = f(m(x))
        return (y.detach(),) + torch.autograd.grad(y, (x,) + leaves, dy)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    for _ in range(4):
        with torch.no_grad():
            x.copy_(ref.normal(g, 70, 256))
            dy.copy_(ref.normal(g, 70, 128))
        graph.replay()
        torch.cuda.synchronize()
        held = [t.clone() for t in outs]
        for got, want in zip(held, step()):
            assert torch.equal(got, want)
