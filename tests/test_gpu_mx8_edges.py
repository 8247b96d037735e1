"""The 8-bit operators at the ends of what their documentation allows."""
import gc

import pytest
import torch

from tests import _mx8 as ref
from tests._mx8 import BF, U8
from paper_2607_05711_amd import _lib as L
from paper_2607_05711_amd import dit

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def some_rows(g, M, K, runs):
    """Ones, with random values in the runs of rows that are looked at."""
    x = torch.ones((M, K), dtype=BF, device=DEV)
    for a, b in runs:
        x[a:b] = ref.normal(g, b - a, K)
    return x


@pytest.mark.parametrize("M,K", [((1 << 26) + 41, 32), ((1 << 24) + 19, 2080)])
def test_norm_of_more_rows_than_a_launch_dimension_holds(M, K):
    """A workgroup each, or one for four: 2^32 threads and more.  Every run of rows is that of a short call on it."""
    torch.cuda.empty_cache()
    g = ref.gen(K)
    runs = [(0, 70), (M // 2 - 35, M // 2 + 35), ((1 << 22) - 35, (1 << 22) + 35), ((1 << 20) - 35, (1 << 20) + 35), (M - 70, M)]
    x, w = some_rows(g, M, K, runs), ref.normal(g, K)
    _, _, c, s, r = L.ft_rmsnorm_quantize8(x, w, want_rstd=True)
    for a, b in runs:
        _, _, c2, s2, r2 = L.ft_rmsnorm_quantize8(x[a:b].clone(), w, want_rstd=True)
        assert torch.equal(c[a:b].view(U8), c2.view(U8)) and torch.equal(s[:, a:b], s2) and torch.equal(r[a:b], r2)
    del x, c, s, r
    torch.cuda.empty_cache()


def test_quantize_of_more_rows_than_a_launch_dimension_holds():
    torch.cuda.empty_cache()
    M, K = (1 << 28) + 5, 32
    g = ref.gen(1)
    runs = [(0, 70), ((1 << 24) - 35, (1 << 24) + 35), (M // 2 - 35, M // 2 + 35), (M - 70, M)]
    x = some_rows(g, M, K, runs)
    c, s, _, _ = L.ft_quantize8(x)
    for a, b in runs:
        c2, s2 = ref.mxfp8(x[a:b])
        assert torch.equal(c[a:b].view(U8), c2) and torch.equal(s[:, a:b], s2)
    del x, c, s
    torch.cuda.empty_cache()


@pytest.mark.parametrize("kind", [dit.FourTuneLinear8, dit.FourTuneMLP8])
def test_capture_beside_the_results_of_an_eager_step(kind):
    """Refused while a loss from the default stream lives, and captured once it is gone."""
    g = ref.gen(3)
    m = kind(128, 96 if kind is dit.FourTuneLinear8 else 256, 16, 16, g, DEV)
    leaves, x = tuple(m.parameters()), ref.normal(g, 33, 128).requires_grad_(True)
    held = m(x)
    dy = torch.ones_like(held)
    step = lambda: torch.autograd.grad(m(x), (x,) + leaves, dy)  # noqa: E731
    torch.cuda.synchronize()
    with pytest.raises(RuntimeError, match="default stream"):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            step()
    want = torch.autograd.grad(held, (x,) + leaves, dy)
    del held
    gc.collect()                                              # (the refusal's traceback)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    for _ in range(3):
        for t in outs:
            t.fill_(1)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
        want = step()


def test_norm_of_rows_at_the_ends_of_fp32():
    """Squares past 2^128 and below 2^-149, without an eps and with one."""
    x = torch.ones((4, 64), dtype=BF, device=DEV)
    x[0], x[1], x[2] = 2.0 ** 64, 2.0 ** -76, 2.0 ** -70
    w = torch.ones(64, dtype=BF, device=DEV)
    _, y, _, _, r = L.ft_rmsnorm_quantize8(x, w, eps=0.0, want_y=True, want_rstd=True)
    assert r.tolist() == [0.0, torch.inf, 2.0 ** 70, 1.0]     # 2^-140, a subnormal, is held exactly
    assert bool((y[0] == 0).all()) and bool(y[1].isinf().all()) and bool((y[2:] == 1).all())
    _, y, _, _, r = L.ft_rmsnorm_quantize8(x, w, eps=2.0 ** -20, want_y=True, want_rstd=True)
    assert bool((r[1:3] == 1024).all()) and bool((y[1] == 2.0 ** -66).all())
