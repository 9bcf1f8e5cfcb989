"""The raster mixer on the GPU: norm, projections, linear attention and the norm of
its heads together, against the same layer in float64 on the CPU (token by token)."""
import numpy as np
import pytest
import torch

from paper_2501_12381_amd.module import RasterMixer
from tests import seq_reference as R
from tests.parity_util import np64

DEV = "cuda:0"


def reference(m, x, dy=None, cu=None):
    """Output, final states; gradients of the input and of every parameter with dy."""
    P = {k: np64(v) for k, v in m.named_parameters()}
    B, C = x.shape[0], x.shape[-1]
    xs = np64(x)
    flat = xs.reshape(B, -1, C)
    T = flat.shape[1]
    rows = flat.reshape(-1, 1, C) if m.per_token else flat
    norm = lambda dz=None: R.group_norm(rows, m.groups, P["norm_weight"], P["norm_bias"], m.eps, "silu",  # noqa: E731
                                        None if dz is None else dz.reshape(rows.shape))
    n = norm().reshape(B, T, C)
    pr = n @ P["proj.weight"].T + P["proj.bias"]
    w = np.cumsum([0] + list(m.widths))
    q, k, v, a = (pr[..., w[i]:w[i + 1]] for i in range(4))
    heads = lambda t, h: t.reshape(B, T, h, -1)  # noqa: E731
    q, k, v = heads(q, m.qk_heads), heads(k, m.qk_heads), heads(v, m.heads)
    la = -np.log1p(np.exp(-a))
    scale = m.head_dim ** -0.5
    o, sf = R.linattn(q, k, v, la, scale, cu=cu)
    ho = o.reshape(-1, 1, m.heads * m.value_dim)
    hn = R.group_norm(ho, m.heads, P["head_weight"], P["head_bias"], m.eps)
    y = flat + (hn[:, 0] @ P["out.weight"].T + P["out.bias"]).reshape(flat.shape)
    if dy is None:
        return y.reshape(xs.shape), sf
    g = np64(dy).reshape(-1, C)
    grads = {"out.weight": g.T @ hn[:, 0], "out.bias": g.sum(0)}
    _, dho, grads["head_weight"], grads["head_bias"] = R.group_norm(
        ho, m.heads, P["head_weight"], P["head_bias"], m.eps, "none", (g @ P["out.weight"])[:, None])
    _, _, dq, dk, dv, da, _ = R.linattn(q, k, v, la, scale, cu=cu, do=dho.reshape(o.shape))
    dp = np.concatenate([t.reshape(B, T, -1) for t in (dq, dk, dv, da / (1 + np.exp(a)))], -1)
    grads["proj.weight"] = dp.reshape(-1, dp.shape[-1]).T @ n.reshape(-1, C)
    grads["proj.bias"] = dp.sum((0, 1))
    _, dx, grads["norm_weight"], grads["norm_bias"] = norm(dp @ P["proj.weight"])
    grads["x"] = (dx.reshape(flat.shape) + np64(dy).reshape(flat.shape)).reshape(xs.shape)
    return y.reshape(xs.shape), sf, grads


def near(got, ref, tol, what):
    g = np64(got)
    assert g.shape == ref.shape and np.isfinite(g).all(), what
    e = np.linalg.norm(g - ref) / np.linalg.norm(ref)
    assert e <= tol, f"{what}: {e:.2e}"


# fp32: library products of some hundred terms around the kernels (1e-5 each).  bf16: about ten roundings
# of 1.7e-3 from the input to a gradient, some of them amplified by the norms
TOL = {torch.float32: 5e-5, torch.bfloat16: 3e-2}


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("per_token", [False, True])
def test_training_step(per_token, dtype):
    torch.manual_seed(1)
    m = RasterMixer(96, 4, 24, kv_heads=2, value_dim=32, groups=8, per_token=per_token).to(DEV, dtype)
    x = torch.randn(2, 9, 11, 96, device=DEV).to(dtype).requires_grad_(True)
    dy = torch.randn(2, 9, 11, 96, device=DEV).to(dtype)
    y = m(x)
    names, params = zip(*m.named_parameters())
    got = dict(zip(("x",) + names, torch.autograd.grad(y, (x,) + params, dy)))
    ry, _, rg = reference(m, x, dy)
    near(y, ry, TOL[dtype], "y")
    for name, g in got.items():
        near(g, rg[name], TOL[dtype], name)


@pytest.mark.gpu
def test_prompts_then_tokens():
    """Packed prompts, then tokens in a pool of states: the same as the whole sequences at once."""
    torch.manual_seed(2)
    m = RasterMixer(64, 4, 16, groups=8, per_token=True).to(DEV)
    lens, more = [5, 70, 33], 6
    seqs = [torch.randn(n + more, 64, device=DEV) for n in lens]
    with torch.no_grad():
        whole = [m(s[None]) for s in seqs]
        cu = torch.tensor([0, 5, 75, 108], dtype=torch.int32, device=DEV)
        y, state = m(torch.cat([s[:n] for s, n in zip(seqs, lens)])[None], return_state=True, cu_seqlens=cu)
        at = 0
        for w, n in zip(whole, lens):
            near(y[0, at:at + n], np64(w[0, :n]), 5e-5, "prompt")
            at += n
        pool, slots = m.new_state(8), torch.tensor([6, 1, 3], dtype=torch.int32, device=DEV)
        pool[slots.long()] = state
        for t in range(more):
            y = m.step(torch.stack([s[n + t] for s, n in zip(seqs, lens)]), pool, slots)
            near(y, np.stack([np64(w[0, n + t]) for w, n in zip(whole, lens)]), 5e-5, f"token {t}")
        for i in (0, 2, 4, 5, 7):
            assert not pool[i].any()


def test_refusals():
    with pytest.raises(ValueError):
        RasterMixer(64, 4, 16, kv_heads=3, groups=8)
    with pytest.raises(ValueError):
        RasterMixer(60, 4, 16, groups=32)
    with pytest.raises(ValueError):
        RasterMixer(64, 4, 16, groups=8).step(torch.zeros(1, 64), torch.zeros(1, 4, 16, 16))
