"""Linear attention with decay on the GPU against the float64 reference.

Tolerances (largest error over largest value of the reference, and 2-norm of the
error over that of the reference): fp32 tensors and all states 1e-5, sums of at most
some thousand fp32 products; bf16 outputs 2e-2 and 5e-3, the rounding of the
output (2-norm 1.7e-3) and of up to two operands before it.  A decay's gradient is a
difference of sums within a chunk: twice that."""
import numpy as np
import pytest
import torch

from paper_2501_12381_amd import lib as L
from paper_2501_12381_amd import ops
from tests import seq_reference as R
from tests.parity_util import np64, normwise

DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16


def close(got, ref, dtype, what, loose=1):
    big, rel = (1e-5, 1e-5) if dtype == F32 else (2e-2, 5e-3)
    g = np64(got)
    assert g.shape == ref.shape, what
    assert np.isfinite(g).all(), f"{what}: not finite"
    if not ref.size:
        return
    n = np.linalg.norm(ref)
    assert normwise(g, ref) <= loose * big, f"{what}: {normwise(g, ref):.2e} of the largest value"
    assert np.linalg.norm(g - ref) <= loose * rel * n + 1e-30, f"{what}: {np.linalg.norm(g - ref) / n:.2e} in norm"


def inputs(B, T, H, Hk, Dk, Dv, dtype, per_token, n, state, seed=0, device=DEV):
    g = torch.Generator().manual_seed(seed)
    rn = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    d = {"q": rn(B, T, Hk, Dk), "k": rn(B, T, Hk, Dk), "v": rn(B, T, H, Dv)}
    d["a"] = -torch.exp(rn(B, T, H) - 3) if per_token else -torch.exp(rn(H) - 3)
    d = {k: t.to(dtype).to(device) for k, t in d.items()}
    d["do"] = rn(B, T, H, Dv).to(dtype).to(device)
    d["s0"] = rn(n, H, Dk, Dv).to(device) if state else None
    d["dsf"] = rn(n, H, Dk, Dv).to(device) if state else None
    return d


def run_both(d, cu=None, scale=None):
    """(names, GPU results, reference results) of forward and backward."""
    cut = torch.tensor(cu, dtype=torch.int32, device=DEV) if cu is not None else None
    o, sf = ops.gspn_linattn_fwd(d["q"], d["k"], d["v"], d["a"], scale=scale, initial_state=d["s0"], return_state=True,
                                 cu_seqlens=cut)
    g = ops.gspn_linattn_bwd(d["do"], d["q"], d["k"], d["v"], d["a"], scale=scale, initial_state=d["s0"],
                             dfinal_state=d["dsf"], cu_seqlens=cut)
    torch.cuda.synchronize()
    h = {k: np64(t) if t is not None else None for k, t in d.items()}
    ref = R.linattn(h["q"], h["k"], h["v"], h["a"], d["q"].shape[-1] ** -0.5 if scale is None else scale, h["s0"], cu,
                    h["do"], h["dsf"])
    return ("o", "sf", "dq", "dk", "dv", "da", "ds0"), (o, sf) + tuple(g), ref


def check(d, cu=None, scale=None):
    dtype = d["q"].dtype
    for name, got, ref in zip(*run_both(d, cu, scale)):
        if got is not None:
            close(got, ref, F32 if name in ("sf", "ds0") else dtype, name, 2 if name == "da" else 1)


# lengths around the chunk (64 in bf16, 32 in fp32), and long enough to be cut into pieces
LENGTHS = [0, 1, 2, 31, 32, 33, 63, 64, 65, 129, 300, 1100]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("T", LENGTHS)
def test_lengths(T, dtype):
    print(f"T {T} {dtype}", flush=True)
    check(inputs(2, T, 2, 2, 32, 32, dtype, True, 2, True, seed=T))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("dims", [(1, 1), (5, 128), (16, 16), (24, 40), (33, 17), (64, 64), (65, 63), (128, 64),
                                  (64, 128), (96, 80), (128, 128)], ids=str)
def test_head_sizes(dims, dtype):
    print(f"dims {dims} {dtype}", flush=True)
    check(inputs(1, 150, 3, 1, *dims, dtype, True, 1, True, seed=sum(dims)))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("heads", [(1, 1), (6, 6), (6, 2), (8, 1)], ids=str)
@pytest.mark.parametrize("per_token", [False, True])
def test_heads_and_decays(heads, per_token, dtype):
    print(f"heads {heads} per_token {per_token} {dtype}", flush=True)
    check(inputs(2, 90, *heads, 16, 24, dtype, per_token, 2, per_token, seed=heads[0]), scale=0.3)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("lens", [[5], [0, 0], [1, 0, 1, 64, 63], [300, 1, 0, 700, 2, 65], [1] * 40, [0, 256, 256, 512]],
                         ids=str)
@pytest.mark.parametrize("per_token", [False, True])
def test_packed(lens, per_token, dtype):
    print(f"lens {lens} {dtype}", flush=True)
    cu = [sum(lens[:i]) for i in range(len(lens) + 1)]
    check(inputs(1, cu[-1], 2, 1, 32, 16, dtype, per_token, len(lens), True, seed=len(lens)), cu)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("per_token", [False, True])
def test_tokens_of_no_sequence(per_token, dtype):
    """Behind the last sequence outputs and gradients are 0, whatever stands there."""
    cu = [0, 70, 500]
    d = inputs(1, 900, 4, 2, 24, 24, dtype, per_token, 2, True)
    full = {k: (t.clone() if t is not None else None) for k, t in d.items()}
    for name in ("q", "k", "v", "do") + (("a",) if per_token else ()):
        full[name][:, 500:] = float("nan")
    cut = {k: (t[:, :500].contiguous() if k in ("q", "k", "v", "do") or (k == "a" and per_token) else t)
           for k, t in d.items()}
    names, got, _ = run_both(full, cu)
    _, want, _ = run_both(cut, cu)
    for name, x, y in zip(names, got, want):
        if x.shape != y.shape:
            assert not x[:, 500:].any(), name
            x = x[:, :500]
        close(x, np64(y), F32 if name in ("sf", "ds0") else dtype, name, 2 if name == "da" else 1)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("dims", [(32, 32), (24, 40), (64, 64), (128, 64), (128, 128)], ids=str)
@pytest.mark.parametrize("name,T", [("v", 200), ("k", 200), ("q", 200), ("a", 200), ("v", 1100)])
def test_non_finite_values_and_earlier_tokens(name, T, dims, dtype):
    """Infinities and NaN of a token reach the outputs that the formula has them in, and no earlier one."""
    print(f"{name} T {T} dims {dims} {dtype}", flush=True)
    d = inputs(1, T, 2, 2, *dims, dtype, True, 1, False, seed=T)
    at = (0, T - 10, 0) if name == "a" else (0, T - 10, 0, 3)
    d[name][at] = float("nan")
    at = (0, T - 130, 1) if name == "a" else (0, T - 130, 1, 5)
    d[name][at] = float("inf") if name == "v" else float("nan")
    o, _ = ops.gspn_linattn_fwd(d["q"], d["k"], d["v"], d["a"])
    h = {k: np64(d[k]) for k in ("q", "k", "v", "a")}
    with np.errstate(invalid="ignore"):
        ref = R.linattn(h["q"], h["k"], h["v"], h["a"], dims[0] ** -0.5, None, None, None, None)[0]
    got, fine = np64(o), np.isfinite(ref)
    assert fine[:, :T - 130].all() and not fine.all()
    np.testing.assert_array_equal(np.isfinite(got), fine)
    close(torch.from_numpy(got[fine]), ref[fine], dtype, "finite part")


@pytest.mark.gpu
def test_sequences_do_not_touch():
    """Non-finite values of one sequence stay in it."""
    cu = [0, 40, 80, 120]
    d = inputs(1, 120, 2, 2, 16, 16, BF16, True, 3, True)
    _, clean, _ = run_both(d, cu)
    for name in ("q", "k", "v", "a"):
        d[name][:, 40:80] = float("nan") if name != "v" else float("inf")
    names, got, _ = run_both(d, cu)
    for name, x, y in zip(names, got, clean):
        for part in ((slice(None), slice(0, 40)), (slice(None), slice(80, 120))) if x.dim() and x.shape[0] == 1 else (
                (0,), (2,)):
            assert torch.equal(x[part], y[part]), name


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_resets_and_no_decay(dtype):
    """-inf (and a type's lowest value) empties the state; 0 keeps it all."""
    d = inputs(1, 200, 3, 3, 32, 32, dtype, True, 1, True)
    d["a"][:, :, 0] = 0
    d["a"][:, 50, 1] = float("-inf")
    d["a"][:, 51, 1] = torch.finfo(dtype).min
    d["a"][:, ::3, 2] = -60000.0
    check(d)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_strides(dtype):
    """q, k, v as slices of one projection, aligned and not, and in another order of axes."""
    d = inputs(2, 100, 4, 2, 32, 48, dtype, True, 2, False)
    want = ops.gspn_linattn_fwd(d["q"], d["k"], d["v"], d["a"])[0]
    gw = ops.gspn_linattn_bwd(d["do"], d["q"], d["k"], d["v"], d["a"])
    for off in (0, 1):
        width = off + 2 * 32 * 2 + 4 * 48 + 7 * off
        proj = torch.full((2, 100, width), float("nan"), dtype=dtype, device=DEV)
        q = proj[..., off:off + 64].unflatten(-1, (2, 32))
        k = proj[..., off + 64:off + 128].unflatten(-1, (2, 32))
        v = proj[..., off + 128:off + 320].unflatten(-1, (4, 48))
        q.copy_(d["q"]), k.copy_(d["k"]), v.copy_(d["v"])
        assert torch.equal(ops.gspn_linattn_fwd(q, k, v, d["a"])[0], want)
        for x, y in zip(ops.gspn_linattn_bwd(d["do"], q, k, v, d["a"]), gw):
            assert (x is None and y is None) or torch.equal(x, y)
    swapped = [d[n].transpose(1, 2).contiguous().transpose(1, 2) for n in ("q", "k", "v")]
    assert torch.equal(ops.gspn_linattn_fwd(*swapped, d["a"])[0], want)
    dense = [d[n].transpose(-1, -2).contiguous().transpose(-1, -2) for n in ("q", "k", "v")]
    assert torch.equal(ops.gspn_linattn_fwd(*dense, d["a"])[0], want)
    shared = [d[n][:1].expand(2, -1, -1, -1) for n in ("q", "k", "v")]
    same = ops.gspn_linattn_fwd(*shared, d["a"][:1].expand(2, -1, -1))[0]
    assert torch.equal(same[0], want[0]) and torch.equal(same[1], want[0])


@pytest.mark.gpu
def test_offsets_past_32_bits():
    """Heads and tokens further apart than 2^31 elements."""
    d = inputs(1, 70, 2, 2, 16, 16, BF16, True, 1, False)
    step = (1 << 31) // 60
    big = torch.empty(70 * step + 64, dtype=BF16, device=DEV)
    q = big.as_strided((1, 70, 2, 16), (0, step, 16, 1))
    q.copy_(d["q"])
    assert torch.equal(ops.gspn_linattn_fwd(q, d["k"], d["v"], d["a"])[0],
                       ops.gspn_linattn_fwd(d["q"], d["k"], d["v"], d["a"])[0])
    del big, q
    H, n = 2, (1 << 31) // (2 * 128 * 128) + 3
    state = torch.empty((n, H, 128, 128), device=DEV)
    state[-1].normal_()
    old = state[-1].clone()
    s = inputs(1, 1, H, H, 128, 128, F32, True, 1, False)
    at = torch.tensor([n - 1], dtype=torch.int32, device=DEV)
    o = ops.gspn_linattn_step(s["q"][:, 0], s["k"][:, 0], s["v"][:, 0], s["a"][:, 0], state, slots=at)
    ref, sf = R.linattn(*(np64(s[n]) for n in ("q", "k", "v", "a")), 128 ** -0.5, np64(old)[None])
    close(o, ref[:, 0], F32, "o")
    close(state[-1:], sf, F32, "state")
    del state
    torch.cuda.empty_cache()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 1, 1, 16, 16), (3, 4, 2, 64, 64), (5, 6, 2, 128, 128), (2, 3, 3, 33, 17),
                                   (7, 2, 1, 128, 4), (2, 4, 4, 1, 100)], ids=str)
@pytest.mark.parametrize("per_row", [False, True])
def test_step(shape, per_row, dtype):
    B, H, Hk, Dk, Dv = shape
    print(f"step {shape} {dtype}", flush=True)
    d = inputs(B, 1, H, Hk, Dk, Dv, dtype, per_row, B, True, seed=B)
    state = d["s0"].clone()
    o = ops.gspn_linattn_step(d["q"][:, 0], d["k"][:, 0], d["v"][:, 0], d["a"][:, 0] if per_row else d["a"], state)
    ref, sf = R.linattn(*(np64(d[n]) for n in ("q", "k", "v", "a")), Dk ** -0.5, np64(d["s0"]))
    close(o, ref[:, 0], dtype, "o")
    close(state, sf, F32, "state")


@pytest.mark.gpu
def test_step_slots():
    """Rows by slot; rows whose slot is none give 0 and change no state."""
    d = inputs(5, 1, 2, 2, 32, 32, BF16, True, 8, True)
    slots = torch.tensor([6, -1, 0, 8, 3], dtype=torch.int32, device=DEV)
    state = d["s0"].clone()
    args = [d[n][:, 0] for n in ("q", "k", "v", "a")]
    o = ops.gspn_linattn_step(*args, state, slots=slots)
    assert not o[1].any() and not o[3].any()
    for i in (1, 2, 4, 5, 7):
        assert torch.equal(state[i], d["s0"][i])
    rows = torch.tensor([0, 2, 4], device=DEV)
    own = d["s0"][slots[rows].long()].clone()
    assert torch.equal(o[rows], ops.gspn_linattn_step(*(t[rows] for t in args), own))
    assert torch.equal(state[slots[rows].long()], own)
    none = ops.gspn_linattn_step(*(t[:0] for t in args), state, slots=slots[:0])
    assert none.shape == (0, 2, 32)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_prompt_then_steps(dtype):
    """A prompt in one call, in two, and token by token."""
    d = inputs(2, 130, 4, 2, 32, 64, dtype, True, 2, True)
    o, sf = ops.gspn_linattn_fwd(d["q"], d["k"], d["v"], d["a"], initial_state=d["s0"], return_state=True)
    parts = [{k: d[k][:, s] for k in ("q", "k", "v", "a")} for s in (slice(0, 77), slice(77, 130))]
    o1, s1 = ops.gspn_linattn_fwd(**_named(parts[0]), initial_state=d["s0"], return_state=True)
    o2, s2 = ops.gspn_linattn_fwd(**_named(parts[1]), initial_state=s1, return_state=True)
    close(torch.cat([o1, o2], 1), np64(o), dtype, "o in two")
    close(s2, np64(sf), F32, "state in two")
    state = s1.clone()
    steps = [ops.gspn_linattn_step(*(d[n][:, t] for n in ("q", "k", "v", "a")), state) for t in range(77, 130)]
    close(torch.stack(steps, 1), np64(o[:, 77:]), dtype, "o by steps")
    close(state, np64(sf), F32, "state by steps")


def _named(p):
    return {"q": p["q"], "k": p["k"], "v": p["v"], "log_decay": p["a"]}


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_autograd(dtype):
    d = inputs(1, 100, 4, 2, 16, 32, dtype, False, 1, True)
    t = {n: d[n].clone().requires_grad_(True) for n in ("q", "k", "v", "a", "s0")}
    o, sf = ops.gspn_linattn(t["q"], t["k"], t["v"], t["a"], initial_state=t["s0"], return_state=True)
    got = torch.autograd.grad((o, sf), list(t.values()), (d["do"], d["dsf"]))
    want = ops.gspn_linattn_bwd(d["do"], d["q"], d["k"], d["v"], d["a"], initial_state=d["s0"], dfinal_state=d["dsf"])
    for n, x, y in zip(t, got, want):
        assert torch.equal(x, y), n
    # one output used alone
    _, sf = ops.gspn_linattn(t["q"], t["k"], t["v"], t["a"], initial_state=t["s0"], return_state=True)
    got = torch.autograd.grad(sf, list(t.values()), d["dsf"], allow_unused=True)
    h = {k: np64(x) for k, x in d.items()}
    ref = R.linattn(h["q"], h["k"], h["v"], h["a"], 0.25, h["s0"], None, np.zeros_like(h["do"]), h["dsf"])[2:]
    for n, x, y in zip(t, got, ref):
        close(x, y, F32 if n == "s0" else dtype, n, 2 if n == "a" else 1)
    o = ops.gspn_linattn(t["q"], t["k"], t["v"], t["a"])
    assert torch.equal(torch.autograd.grad(o, t["v"], d["do"])[0],
                       ops.gspn_linattn_bwd(d["do"], d["q"], d["k"], d["v"], d["a"])[2])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 3000, 2, 1, 64, 64), (1, 2000, 2, 2, 128, 128), (3, 900, 4, 4, 128, 33),
                                   (2, 1500, 3, 3, 24, 100), (1, 100, 2, 2, 16, 16)], ids=str)
@pytest.mark.parametrize("packed", [False, True])
def test_states_of_the_forward(shape, packed, dtype):
    """The backward from the states that the forward left in its workspace."""
    print(f"states of the forward {shape} packed {packed} {dtype}", flush=True)
    B, T = shape[:2]
    cu = [0, 1, T // 3, T // 3, T * B - 5] if packed else None
    d = inputs(*((1, B * T) if packed else (B, T)), *shape[2:], dtype, True, 4 if packed else B, True, seed=T)
    cut = torch.tensor(cu, dtype=torch.int32, device=DEV) if packed else None
    args = (d["q"], d["k"], d["v"], d["a"])
    ws = ops.gspn_linattn_workspace(*args, cu_seqlens=cut)
    ops.gspn_linattn_fwd(*args, initial_state=d["s0"], cu_seqlens=cut, workspace=ws)
    got = ops.gspn_linattn_bwd(d["do"], *args, initial_state=d["s0"], dfinal_state=d["dsf"], cu_seqlens=cut,
                               forward_workspace=ws)
    h = {k: np64(t) for k, t in d.items()}
    ref = R.linattn(h["q"], h["k"], h["v"], h["a"], shape[4] ** -0.5, h["s0"], cu, h["do"], h["dsf"])
    for name, x, y in zip(("dq", "dk", "dv", "da", "ds0"), got, ref[2:]):
        close(x, y, F32 if name == "ds0" else dtype, name, 2 if name == "da" else 1)
    if ws.numel():
        with pytest.raises(ValueError):
            ops.gspn_linattn_bwd(d["do"], *args, cu_seqlens=cut, forward_workspace=ws[:-256])


@pytest.mark.gpu
def test_repeats_and_streams():
    """The same bits every time, on another stream, and from a replayed graph."""
    d = inputs(1, 1500, 2, 1, 64, 64, BF16, True, 1, True)

    def call():
        o, sf = ops.gspn_linattn_fwd(d["q"], d["k"], d["v"], d["a"], initial_state=d["s0"], return_state=True)
        return (o, sf) + ops.gspn_linattn_bwd(d["do"], d["q"], d["k"], d["v"], d["a"], initial_state=d["s0"],
                                              dfinal_state=d["dsf"])

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
        for x, y, z, u in zip(first, other, held, again):
            assert torch.equal(x, y) and torch.equal(x, z) and torch.equal(x, u), k


@pytest.mark.gpu
def test_empty():
    """No sequences, or none of any length."""
    d = inputs(0, 5, 2, 1, 16, 16, BF16, False, 0, True)
    o, sf = ops.gspn_linattn_fwd(d["q"], d["k"], d["v"], d["a"], initial_state=d["s0"], return_state=True)
    assert o.shape == (0, 5, 2, 16) and sf.shape == (0, 2, 16, 16)
    g = ops.gspn_linattn_bwd(d["do"], d["q"], d["k"], d["v"], d["a"])
    assert g[0].shape == d["q"].shape and not g[3].any()
    d = inputs(1, 9, 2, 1, 16, 16, F32, False, 0, False)
    cu = torch.zeros(1, dtype=torch.int32, device=DEV)
    o, sf = ops.gspn_linattn_fwd(d["q"], d["k"], d["v"], d["a"], return_state=True, cu_seqlens=cu)
    assert not o.any() and sf.shape == (0, 2, 16, 16)


@pytest.mark.gpu
def test_refusals():
    d = inputs(2, 8, 4, 2, 16, 16, F32, True, 2, True)
    q, k, v, a, s0 = (d[n] for n in ("q", "k", "v", "a", "s0"))
    f = ops.gspn_linattn_fwd
    with pytest.raises(RuntimeError):
        f(q.cpu(), k, v, a)
    with pytest.raises(TypeError):
        f(q.double(), k, v, a)
    with pytest.raises(TypeError):
        f(q, k.bfloat16(), v, a)
    with pytest.raises(ValueError):
        f(q, k[:, :7], v, a)
    with pytest.raises(ValueError):
        f(q, k, v[:, :, :3], a[:, :, :3])  # 3 value heads, 2 query heads
    with pytest.raises(ValueError):
        f(q, k, v, a[:, :7])
    with pytest.raises(ValueError):
        f(q, k, v, a, initial_state=s0[:1])
    with pytest.raises(TypeError):
        f(q, k, v, a, initial_state=s0.bfloat16())
    with pytest.raises(ValueError):
        f(q, k, v, a, cu_seqlens=torch.zeros(3, dtype=torch.int32, device=DEV))  # two batch rows
    with pytest.raises(TypeError):
        f(q[:1], k[:1], v[:1], a[:1], cu_seqlens=torch.zeros(3, device=DEV))
    with pytest.raises(ValueError):
        ops.gspn_linattn_bwd(d["do"][:, :7], q, k, v, a)
    big = torch.zeros((1, 4, 1, 129), device=DEV)
    with pytest.raises(L.GSPNError) as e:
        f(big, big, v[:1, :4], a[:1, :4])
    assert e.value.status == 7
    s = [t[:, 0] for t in (q, k, v, a)]
    with pytest.raises(ValueError):
        ops.gspn_linattn_step(*s, s0[:1])
    with pytest.raises(ValueError):
        ops.gspn_linattn_step(*s, s0.transpose(-1, -2))
    with pytest.raises(TypeError):
        ops.gspn_linattn_step(*s, s0, slots=torch.zeros(2, dtype=torch.int64, device=DEV))
    with pytest.raises(ValueError):
        ops.gspn_linattn_step(*s, s0, out=torch.empty((2, 4, 17), device=DEV))
