"""Group norm with an activation on the GPU against the float64 reference.

Tolerances as in the other parity tests (largest error over largest value): 1e-5 for
fp32 (sums of at most 1e5 values around a value of the group, each in partial sums
of some hundred), 2e-2 for bf16, with 2-norms of 1e-5 and 5e-3."""
import numpy as np
import pytest
import torch

from paper_2501_12381_amd import lib as L
from paper_2501_12381_amd import ops
from tests import seq_reference as R
from tests.parity_util import np64, normwise

DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16


def close(got, ref, dtype, what, big=None):
    tol, rel = (1e-5, 1e-5) if dtype == F32 else (2e-2, 5e-3)
    g = np64(got)
    assert np.isfinite(g).all(), f"{what}: not finite"
    assert normwise(g, ref) <= (big or tol), f"{what}: {normwise(g, ref):.2e} of the largest value"
    assert np.linalg.norm(g - ref) <= (big or rel) * np.linalg.norm(ref) + 1e-30, what


def make(B, Ls, C, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(B, Ls, C, generator=g) * 1.5 + torch.randn(C, generator=g)
    w, b = 1 + 0.3 * torch.randn(C, generator=g), 0.3 * torch.randn(C, generator=g)
    dy = torch.randn(B, Ls, C, generator=g)
    return [t.to(dtype).to(DEV) for t in (x, w, b, dy)]


def check(x, w, b, dy, G, act, eps=1e-5, big=None):
    y, mean, rstd = ops.gspn_group_norm_fwd(x, G, w, b, eps=eps, act=act)
    got = (y,) + ops.gspn_group_norm_bwd(dy, x, mean, rstd, G, w, b, act=act)
    torch.cuda.synchronize()
    h = [np64(t) if t is not None else None for t in (x, w, b, dy)]
    ref = R.group_norm(h[0], G, h[1], h[2], eps, act, h[3])
    for name, g, r in zip(("y", "dx", "dw", "db"), got, ref):
        if g is not None:
            close(g, r, x.dtype, name, big)


# slabs a wave holds (with whole vectors and without), slabs that are split, single tokens
SHAPES = [(1, 1, 8, 1), (2, 7, 24, 4), (3, 49, 40, 8), (1, 196, 384, 32), (2, 50, 30, 3), (2, 1024, 64, 32),
          (1, 5000, 53, 1), (2, 3465, 96, 8), (2, 300, 1280, 1), (5, 1, 2048, 16), (700, 1, 96, 4), (1, 40, 8192, 32),
          (33, 64, 320, 32), (1, 17, 4100, 2), (9000, 1, 64, 8)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("act", ["none", "silu"])
def test_shapes(shape, act, dtype):
    B, Ls, C, G = shape
    print(f"norm {shape} {act} {dtype}", flush=True)
    check(*make(B, Ls, C, dtype, seed=C), G, act)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", [(2, 30, 48, 4), (1, 2000, 64, 4)], ids=str)
def test_gelu_and_missing_parameters(shape, dtype):
    B, Ls, C, G = shape
    x, w, b, dy = make(B, Ls, C, dtype)
    check(x, w, b, dy, G, "gelu")
    check(x, w, None, dy, G, "silu")
    check(x, None, b, dy, G, "silu")
    check(x, None, None, dy, G, "none", eps=0.1)


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(2, 64, 64, 8), (2, 4096, 64, 8)], ids=str)
def test_large_mean(shape):
    """A mean of 1000 spreads: fp32 holds the mean itself to 3e-5 of a spread, which is all that may be lost."""
    B, Ls, C, G = shape
    x, w, b, dy = make(B, Ls, C, F32)
    check(x + 1000, w, b, dy, G, "none", big=1e-4)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_constant_groups(dtype):
    """No spread: y is act(bias), and only eps keeps the gradient finite."""
    x = torch.full((2, 100, 32), 3.25, dtype=dtype, device=DEV)
    w, b = (torch.randn(32, device=DEV).to(dtype) for _ in range(2))
    for Ls in (100, 1):
        y = ops.gspn_group_norm(x[:, :Ls].contiguous(), 4, w, b)
        assert torch.equal(y, b.expand(2, Ls, 32))


@pytest.mark.gpu
@pytest.mark.parametrize("Ls", [20, 3000])
def test_groups_do_not_touch(Ls):
    x, w, b, dy = make(2, Ls, 64, BF16)
    y = ops.gspn_group_norm(x, 8, w, b, act="silu")
    x2 = x.clone()
    x2[1, Ls // 2, 20] = float("nan")
    x2[0, 3, 60] = float("inf")
    y2 = ops.gspn_group_norm(x2, 8, w, b, act="silu")
    keep = torch.ones((2, 8), dtype=torch.bool, device=DEV)
    keep[1, 2] = keep[0, 7] = False
    same = keep[:, None, :, None].expand(2, Ls, 8, 8).reshape(2, Ls, 64)
    assert torch.equal(y2[same], y[same])
    assert torch.isnan(y2[1, :, 16:24]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", [(2, 33, 64, 4), (2, 2100, 64, 4)], ids=str)
def test_layouts(shape, dtype):
    """Maps of several sides, views that start off 16 bytes, and tensors in another order of axes."""
    B, Ls, C, G = shape
    x, w, b, dy = make(B, Ls, C, dtype)
    want = ops.gspn_group_norm(x, G, w, b, act="silu")
    assert torch.equal(ops.gspn_group_norm(x.view(B, 3, Ls // 3, C), G, w, b, act="silu").view(x.shape), want)
    off = torch.empty(x.numel() + 1, dtype=dtype, device=DEV)[1:].view(x.shape)
    off.copy_(x)
    g = ops.gspn_group_norm(off, G, w, b, act="silu")
    close(g, np64(want), dtype, "off by one")
    stats = ops.gspn_group_norm_fwd(x, G, w, b, act="silu")[1:]
    close(ops.gspn_group_norm_bwd(dy, off, *stats, G, w, b, act="silu")[0],
          np64(ops.gspn_group_norm_bwd(dy, x, *stats, G, w, b, act="silu")[0]), dtype, "dx off by one")
    first = x.transpose(1, 2).contiguous().transpose(1, 2)
    assert torch.equal(ops.gspn_group_norm(first, G, w, b, act="silu"), want)


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(2, 49, 64, 8), (2, 5000, 64, 8), (6000, 1, 64, 8)], ids=str)
def test_autograd_repeats_and_graphs(shape):
    B, Ls, C, G = shape
    x, w, b, dy = make(B, Ls, C, BF16)
    for t in (x, w, b):
        t.requires_grad_(True)

    def call():
        y = ops.gspn_group_norm(x, G, w, b, act="silu")
        return (y.detach(),) + torch.autograd.grad(y, (x, w, b), dy)

    first = [t.clone() for t in call()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = call()
    for k in range(3):
        for t in held:
            t.zero_()
        graph.replay()
        again = call()
        torch.cuda.synchronize()
        for p, q, r, s in zip(first, other, held, again):
            assert torch.equal(p, q) and torch.equal(p, r) and torch.equal(p, s), k


@pytest.mark.gpu
def test_empty():
    for shape in ((0, 5, 16), (3, 0, 16)):
        x = torch.empty(shape, device=DEV, requires_grad=True)
        w, b = (torch.ones(16, device=DEV, requires_grad=True) for _ in range(2))
        y = ops.gspn_group_norm(x, 4, w, b)
        g = torch.autograd.grad(y, (x, w, b), torch.empty_like(y))
        assert y.shape == shape and not g[1].any() and not g[2].any()


@pytest.mark.gpu
def test_refusals():
    x, w, b, dy = make(2, 9, 32, F32)
    f = ops.gspn_group_norm_fwd
    with pytest.raises(RuntimeError):
        f(x.cpu(), 4)
    with pytest.raises(TypeError):
        f(x.half(), 4)
    with pytest.raises(TypeError):
        f(x, 4, w.bfloat16())
    with pytest.raises(ValueError):
        f(x, 5)
    with pytest.raises(ValueError):
        f(x, 4, w[:31])
    with pytest.raises(ValueError):
        f(x, 4, act="relu")
    with pytest.raises(ValueError):
        f(x[0, 0], 4)
    with pytest.raises(L.GSPNError):
        f(x, 4, eps=-1.0)
    with pytest.raises(L.GSPNError):
        f(torch.zeros((1, 1, 8200), device=DEV), 4)
    y, mean, rstd = f(x, 4, w, b)
    with pytest.raises(ValueError):
        ops.gspn_group_norm_bwd(dy, x, mean[:1], rstd, 4, w, b)
    with pytest.raises(ValueError):
        ops.gspn_group_norm_bwd(dy[:, :8], x, mean, rstd, 4, w, b)
