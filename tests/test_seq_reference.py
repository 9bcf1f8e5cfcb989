"""The float64 references of linear attention and group norm against differences."""
import numpy as np
import pytest

from tests import seq_reference as R


def check(f, grads, args, rng, eps=1e-6):
    """<grad, direction> against the central difference along it, for every argument."""
    for name, g in grads.items():
        d = rng.standard_normal(args[name].shape)
        hi, lo = dict(args), dict(args)
        hi[name], lo[name] = args[name] + eps * d, args[name] - eps * d
        num = (f(**hi) - f(**lo)) / (2 * eps)
        assert abs(num - (g * d).sum()) <= 1e-6 * max(1.0, abs(num)), name


@pytest.mark.parametrize("per_token", [False, True])
@pytest.mark.parametrize("cu", [None, [0, 3, 3, 4, 11]])
def test_linattn_gradients(per_token, cu):
    rng = np.random.default_rng(3)
    B, T, H, Hk, Dk, Dv = (2, 7, 4, 2, 3, 5) if cu is None else (1, 11, 4, 2, 3, 5)
    n = B if cu is None else len(cu) - 1
    args = {"q": rng.standard_normal((B, T, Hk, Dk)), "k": rng.standard_normal((B, T, Hk, Dk)),
            "v": rng.standard_normal((B, T, H, Dv)),
            "a": -rng.random((B, T, H) if per_token else (H,)), "s0": rng.standard_normal((n, H, Dk, Dv))}
    do, dsf = rng.standard_normal((B, T, H, Dv)), rng.standard_normal((n, H, Dk, Dv))

    def loss(**kw):
        o, sf = R.linattn(scale=0.7, cu=cu, **kw)
        return (o * do).sum() + (sf * dsf).sum()

    got = R.linattn(scale=0.7, cu=cu, do=do, dsf=dsf, **args)
    check(loss, dict(zip(("q", "k", "v", "a", "s0"), got[2:])), args, rng)


@pytest.mark.parametrize("act", ["none", "silu", "gelu"])
def test_group_norm_gradients(act):
    rng = np.random.default_rng(5)
    args = {"x": rng.standard_normal((2, 5, 6)), "w": rng.standard_normal(6), "b": rng.standard_normal(6)}
    dy = rng.standard_normal((2, 5, 6))
    got = R.group_norm(G=2, act=act, dy=dy, **args)
    check(lambda **kw: (R.group_norm(G=2, act=act, **kw) * dy).sum(), dict(zip(("x", "w", "b"), got[1:])), args, rng)


def test_linattn_is_the_decayed_sum():
    """o_t = scale sum_{s<=t} e^{a_{s+1} + .. + a_t} (q_t.k_s) v_s, written out."""
    rng = np.random.default_rng(7)
    q, k, v = (rng.standard_normal((1, 6, 1, 4)) for _ in range(3))
    a = -rng.random((1, 6, 1))
    o, _ = R.linattn(q, k, v, a, 0.5)
    for t in range(6):
        want = sum(np.exp(a[0, s + 1:t + 1, 0].sum()) * (q[0, t, 0] @ k[0, s, 0]) * v[0, s, 0] for s in range(t + 1))
        np.testing.assert_allclose(o[0, t, 0], 0.5 * want, rtol=1e-12)
