"""Torch-facing wrappers of the sequence operators beside the scan: linear
attention with a decay for each head, and group norm with an activation on
channels-last maps (argument marshalling only; `ops` re-exports them).

Tensors must live on a ROCm device: there is no CPU path.
"""
from __future__ import annotations

import ctypes
from functools import lru_cache

import torch

from . import lib as L

_DT = {torch.float32: L.GSPN_F32, torch.bfloat16: L.GSPN_BF16}
_ACT = {"none": L.GSPN_ACT_NONE, "silu": L.GSPN_ACT_SILU, "gelu": L.GSPN_ACT_GELU}
_I64x9, _I64x6 = ctypes.c_int64 * 9, ctypes.c_int64 * 6

# Workspace sizes depend on these numbers alone; a program calls with few of them.
_lin_fwd_bytes = lru_cache(maxsize=256)(L.gspn_linattn_fwd_workspace_bytes)
_lin_bwd_bytes = lru_cache(maxsize=256)(L.gspn_linattn_bwd_workspace_bytes)
_norm_fwd_bytes = lru_cache(maxsize=256)(L.gspn_group_norm_fwd_workspace_bytes)
_norm_bwd_bytes = lru_cache(maxsize=256)(L.gspn_group_norm_bwd_workspace_bytes)


def _call(fn, where: str, dev, *args) -> None:
    """Call the library's `fn` with the current stream of `dev` behind `args`."""
    if torch.cuda.current_device() == dev.index:
        st = fn(*args, torch._C._cuda_getCurrentRawStream(dev.index))
    else:
        with torch.cuda.device(dev):
            st = fn(*args, torch._C._cuda_getCurrentRawStream(dev.index))
    if st != 0:
        raise L.GSPNError(st, where)


def _dtype(t: torch.Tensor, what: str) -> int:
    if t.dtype not in _DT:
        raise TypeError(f"{what} supports float32 and bfloat16, got {t.dtype}")
    return _DT[t.dtype]


def _check_tensor(name, t, shape, dtype, dev, what) -> None:
    # `dev` is a GPU's; the one test that all good tensors pass comes first
    if isinstance(t, torch.Tensor) and t.dtype == dtype and t.shape == shape and t.device == dev:
        return
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a tensor")
    if not t.is_cuda:
        raise RuntimeError(f"{name} is on {t.device}: the {what} runs on the GPU only")
    if t.dtype != dtype:
        raise TypeError(f"{name} has dtype {t.dtype}, expected {dtype}")
    if t.device != dev:
        raise RuntimeError(f"{name} is on {t.device}, expected {dev}")
    raise ValueError(f"{name} must be {tuple(shape)}, got {tuple(t.shape)}")


def _ptr(t):
    return None if t is None else t.data_ptr()


def _rows(t: torch.Tensor) -> torch.Tensor:
    """A tensor whose last axis is dense (other strides are passed on)."""
    return t if t.is_contiguous() or t.stride(-1) == 1 else t.contiguous()


def _needs_grad(*tensors) -> bool:
    return torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors)


# ---------------------------------------------------------------------------
# linear attention
# ---------------------------------------------------------------------------
_LIN = "linear attention"


class _Lin:
    """Sizes of a call, checked."""

    __slots__ = ("dt", "dev", "n", "sizes", "flags", "scale", "strides", "q", "k", "v", "a", "s0", "cu", "packed")

    def __init__(self, q, k, v, log_decay, scale, initial_state, cu_seqlens):
        if not isinstance(q, torch.Tensor):
            raise TypeError("q must be a tensor")
        if not q.is_cuda:
            raise RuntimeError(f"q is on {q.device}: the {_LIN} runs on the GPU only")
        self.dt, self.dev = _dtype(q, _LIN), q.device
        if q.dim() != 4 or not isinstance(v, torch.Tensor) or v.dim() != 4:
            raise ValueError("q must be (B, T, Hk, Dk) and v (B, T, H, Dv)")
        B, T, Hk, Dk = q.shape
        H, Dv = v.shape[2:]
        _check_tensor("k", k, q.shape, q.dtype, self.dev, _LIN)
        _check_tensor("v", v, (B, T, H, Dv), q.dtype, self.dev, _LIN)
        if Hk < 1 or H < 1 or H % Hk:
            raise ValueError(f"v's {H} heads must be a multiple of q's and k's {Hk}")
        per_token = isinstance(log_decay, torch.Tensor) and log_decay.dim() != 1
        _check_tensor("log_decay", log_decay, (B, T, H) if per_token else (H,), q.dtype, self.dev, _LIN)
        self.packed = cu_seqlens is not None
        n = B
        if self.packed:
            if not isinstance(cu_seqlens, torch.Tensor) or cu_seqlens.dim() != 1 or cu_seqlens.numel() < 1:
                raise ValueError("cu_seqlens must be a tensor of the sequences' starts and the last one's end")
            if B != 1:
                raise ValueError(f"packed sequences have one batch row, got {B}")
            n = cu_seqlens.numel() - 1
            _check_tensor("cu_seqlens", cu_seqlens, (n + 1,), torch.int32, self.dev, _LIN)
            cu_seqlens = cu_seqlens.contiguous()
        if initial_state is not None:
            _check_tensor("initial_state", initial_state, (n, H, Dk, Dv), torch.float32, self.dev, _LIN)
            initial_state = initial_state.contiguous()
        self.n = n
        self.sizes = (n, B, T, H, Hk, Dk, Dv)
        self.flags = L.GSPN_LINATTN_DECAY_PER_TOKEN if per_token else 0
        self.scale = Dk ** -0.5 if scale is None else float(scale)
        q, k, v = _rows(q), _rows(k), _rows(v)
        self.q, self.k, self.v, self.a = q, k, v, log_decay.contiguous()
        self.s0, self.cu = initial_state, cu_seqlens
        dense = q.is_contiguous() and k.is_contiguous() and v.is_contiguous()
        self.strides = None if dense else _I64x9(*q.stride()[:3], *k.stride()[:3], *v.stride()[:3])

    def workspace(self, size, given):
        need = size(*self.sizes, int(self.packed), self.dt, self.flags)
        if given is not None and given.numel() >= need:
            if need and (given.device != self.dev or not given.is_contiguous() or given.dtype != torch.uint8):
                raise ValueError(f"workspace must be a contiguous uint8 tensor on {self.dev}")
            return given
        return torch.empty(need, dtype=torch.uint8, device=self.dev) if need else None


def gspn_linattn_workspace(q, k, v, log_decay, *, cu_seqlens=None) -> torch.Tensor:
    """A workspace for the forward call, for programs that hand the states it keeps
    there on to the backward (`forward_workspace`)."""
    c = _Lin(q, k, v, log_decay, None, None, cu_seqlens)
    ws = c.workspace(_lin_fwd_bytes, None)
    return torch.empty(0, dtype=torch.uint8, device=c.dev) if ws is None else ws


def _linattn_fwd(c: _Lin, return_state, workspace):
    n, B, T, H, Hk, Dk, Dv = c.sizes
    o = torch.empty((B, T, H, Dv), dtype=c.q.dtype, device=c.dev)
    sf = torch.empty((n, H, Dk, Dv), dtype=torch.float32, device=c.dev) if return_state else None
    ws = c.workspace(_lin_fwd_bytes, workspace)
    _call(L.load().gspn_linattn_fwd, "gspn_linattn_fwd", c.dev, c.q.data_ptr(), c.k.data_ptr(), c.v.data_ptr(),
          c.a.data_ptr(), _ptr(c.s0), _ptr(c.cu), o.data_ptr(), _ptr(sf), *c.sizes, c.strides, c.dt, c.flags,
          c.scale, _ptr(ws), 0 if ws is None else ws.numel())
    return o, sf, ws


def _linattn_bwd(c: _Lin, q, k, v, a, s0, cu, do, dsf, forward_workspace, workspace):
    """c: the sizes of the call that q .. cu (dense on their last axis) belong to."""
    _check_tensor("do", do, v.shape, q.dtype, c.dev, _LIN)
    do = do.contiguous()
    n, B, T, H, Hk, Dk, Dv = c.sizes
    if dsf is not None:
        _check_tensor("dfinal_state", dsf, (n, H, Dk, Dv), torch.float32, c.dev, _LIN)
        dsf = dsf.contiguous()
    if forward_workspace is not None:
        need = _lin_fwd_bytes(*c.sizes, int(c.packed), c.dt, c.flags)
        if forward_workspace.numel() < need:
            raise ValueError(f"the forward's workspace holds {forward_workspace.numel()} bytes, not {need}")
        forward_workspace = c.workspace(_lin_fwd_bytes, forward_workspace) if need else None
    new = lambda t: torch.empty(t.shape, dtype=t.dtype, device=c.dev)  # noqa: E731
    dq, dk, dv = new(q), new(k), new(v)
    da = new(a) if n else torch.zeros(a.shape, dtype=q.dtype, device=c.dev)
    ds0 = new(s0) if s0 is not None else None
    ws = c.workspace(_lin_bwd_bytes, workspace)
    _call(L.load().gspn_linattn_bwd, "gspn_linattn_bwd", c.dev, do.data_ptr(), q.data_ptr(), k.data_ptr(),
          v.data_ptr(), a.data_ptr(), _ptr(s0), _ptr(dsf), _ptr(cu), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(),
          da.data_ptr(), _ptr(ds0), *c.sizes, c.strides, c.dt, c.flags, c.scale, _ptr(forward_workspace), _ptr(ws),
          0 if ws is None else ws.numel())
    return dq, dk, dv, da, ds0


def gspn_linattn_fwd(q, k, v, log_decay, *, scale=None, initial_state=None, return_state: bool = False,
                     cu_seqlens=None, workspace=None):
    """(o, final state or None): S_t = exp(a_t) S_{t-1} + k_t v_t^T, o_t = scale q_t S_t.

    q, k: (B, T, Hk, Dk); v: (B, T, H, Dv), H a multiple of Hk; log_decay: (H,) or
    (B, T, H); scale: Dk ** -0.5 unless given.  States are float32 (n, H, Dk, Dv).
    cu_seqlens (int32, n + 1 positions, on the GPU): n sequences packed into a
    batch of one; else n = B."""
    return _linattn_fwd(_Lin(q, k, v, log_decay, scale, initial_state, cu_seqlens), return_state, workspace)[:2]


def gspn_linattn_bwd(do, q, k, v, log_decay, *, scale=None, initial_state=None, dfinal_state=None, cu_seqlens=None,
                     forward_workspace=None, workspace=None):
    """Gradients (dq, dk, dv, dlog_decay, dinitial_state or None) of <do, o> + <dfinal_state, final state>.

    forward_workspace: the workspace that the forward call on the same inputs was
    given (gspn_linattn_workspace), unchanged since: its states are used again."""
    c = _Lin(q, k, v, log_decay, scale, initial_state, cu_seqlens)
    return _linattn_bwd(c, c.q, c.k, c.v, c.a, c.s0, c.cu, do, dfinal_state, forward_workspace, workspace)


class GSPNLinAttn(torch.autograd.Function):
    """Autograd wrapper: forward and backward both run the HIP kernels."""

    @staticmethod
    def forward(ctx, q, k, v, log_decay, initial_state, scale, return_state, cu_seqlens):
        c = _Lin(q, k, v, log_decay, scale, initial_state, cu_seqlens)
        # the workspace, if there is one, carries the states of the sequences' pieces to the backward
        o, sf, ctx.ws = _linattn_fwd(c, return_state, None)
        ctx.save_for_backward(c.q, c.k, c.v, c.a, c.s0, c.cu)
        c.q = c.k = c.v = c.a = c.s0 = c.cu = None
        ctx.call = c
        ctx.set_materialize_grads(False)
        return (o, sf) if return_state else o

    @staticmethod
    def backward(ctx, do, dsf=None):
        if do is None and dsf is None:
            return (None,) * 8
        saved = ctx.saved_tensors
        if do is None:
            do = torch.zeros_like(saved[2], memory_format=torch.contiguous_format)
        return (*_linattn_bwd(ctx.call, *saved, do, dsf, ctx.ws, None), None, None, None)


def gspn_linattn(q, k, v, log_decay, *, scale=None, initial_state=None, return_state: bool = False,
                 cu_seqlens=None):
    """Differentiable linear attention with a decay for each head (arguments as in
    gspn_linattn_fwd): o, or (o, final state) with return_state."""
    if _needs_grad(q, k, v, log_decay, initial_state):
        return GSPNLinAttn.apply(q, k, v, log_decay, initial_state, scale, return_state, cu_seqlens)
    o, sf, _ = _linattn_fwd(_Lin(q, k, v, log_decay, scale, initial_state, cu_seqlens), return_state, None)
    return (o, sf) if return_state else o


def gspn_linattn_step(q, k, v, log_decay, state, *, scale=None, slots=None, out=None) -> torch.Tensor:
    """One token for each of B sequences: updates `state` in place and returns o (B, H, Dv).

    q, k: (B, Hk, Dk); v: (B, H, Dv); log_decay: (H,) or (B, H); state: float32
    (n, H, Dk, Dv), contiguous.  slots (int32 (B,), on the GPU): the state each row uses, a
    number outside [0, n) leaves the row out (its output is 0); else row b uses state b."""
    if not isinstance(q, torch.Tensor):
        raise TypeError("q must be a tensor")
    if not q.is_cuda:
        raise RuntimeError(f"q is on {q.device}: the {_LIN} runs on the GPU only")
    dt, dev = _dtype(q, _LIN), q.device
    if q.dim() != 3 or not isinstance(v, torch.Tensor) or v.dim() != 3:
        raise ValueError("q must be (B, Hk, Dk) and v (B, H, Dv)")
    B, Hk, Dk = q.shape
    H, Dv = v.shape[1:]
    _check_tensor("k", k, q.shape, q.dtype, dev, _LIN)
    _check_tensor("v", v, (B, H, Dv), q.dtype, dev, _LIN)
    if Hk < 1 or H < 1 or H % Hk:
        raise ValueError(f"v's {H} heads must be a multiple of q's and k's {Hk}")
    per_row = isinstance(log_decay, torch.Tensor) and log_decay.dim() != 1
    _check_tensor("log_decay", log_decay, (B, H) if per_row else (H,), q.dtype, dev, _LIN)
    if not isinstance(state, torch.Tensor) or state.dim() != 4:
        raise ValueError("state must be a tensor (n, H, Dk, Dv)")
    n = state.shape[0]
    _check_tensor("state", state, (n, H, Dk, Dv), torch.float32, dev, _LIN)
    if not state.is_contiguous():
        raise ValueError("state must be contiguous: it is updated in place")
    if slots is not None:
        _check_tensor("slots", slots, (B,), torch.int32, dev, _LIN)
        slots = slots.contiguous()
    elif n < B:
        raise ValueError(f"{B} rows need as many states, got {n}")
    q, k, v, log_decay = _rows(q), _rows(k), _rows(v), log_decay.contiguous()
    if out is None:
        out = torch.empty((B, H, Dv), dtype=q.dtype, device=dev)
    else:
        _check_tensor("out", out, (B, H, Dv), q.dtype, dev, _LIN)
        if not out.is_contiguous():
            raise ValueError("out must be contiguous")
    dense = q.is_contiguous() and k.is_contiguous() and v.is_contiguous()
    strides = None if dense else _I64x6(*q.stride()[:2], *k.stride()[:2], *v.stride()[:2])
    _call(L.load().gspn_linattn_step, "gspn_linattn_step", dev, q.data_ptr(), k.data_ptr(), v.data_ptr(),
          log_decay.data_ptr(), state.data_ptr(), _ptr(slots), out.data_ptr(), n, B, H, Hk, Dk, Dv, strides, dt,
          L.GSPN_LINATTN_DECAY_PER_TOKEN if per_row else 0, Dk ** -0.5 if scale is None else float(scale))
    return out


# ---------------------------------------------------------------------------
# group norm
# ---------------------------------------------------------------------------
_NORM = "group norm"


def _norm_sizes(x, groups, weight, bias, act):
    if not isinstance(x, torch.Tensor):
        raise TypeError("x must be a tensor")
    if not x.is_cuda:
        raise RuntimeError(f"x is on {x.device}: the {_NORM} runs on the GPU only")
    dt = _dtype(x, _NORM)
    if x.dim() < 2:
        raise ValueError("x must be (B, ..., C), channels last")
    if act not in _ACT:
        raise ValueError(f"act must be one of {sorted(_ACT)}, got {act!r}")
    B, C = x.shape[0], x.shape[-1]
    if groups < 1 or C < 1 or C % groups:
        raise ValueError(f"{C} channels do not make {groups} groups")
    for name, t in (("weight", weight), ("bias", bias)):
        if t is not None:
            _check_tensor(name, t, (C,), x.dtype, x.device, _NORM)
    n = x.numel()
    if n:
        return dt, B, n // (B * C), C
    length = 1
    for s in x.shape[1:-1]:
        length *= s
    return dt, B, length, C


def gspn_group_norm_fwd(x, groups: int, weight=None, bias=None, *, eps: float = 1e-5, act: str = "none"):
    """(y, mean, rstd): group norm of x (B, ..., C), channels last, then `act`
    ("none", "silu" or "gelu"); mean and rstd (B, groups) in float32."""
    dt, B, length, C = _norm_sizes(x, groups, weight, bias, act)
    dev = x.device
    x = x.contiguous()
    weight, bias = (t if t is None else t.contiguous() for t in (weight, bias))
    y = torch.empty(x.shape, dtype=x.dtype, device=dev)
    stats = torch.empty((2, B, groups), dtype=torch.float32, device=dev)
    need = _norm_fwd_bytes(B, length, C, groups, dt)
    ws = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
    mean = stats.data_ptr()
    _call(L.load().gspn_group_norm_fwd, "gspn_group_norm_fwd", dev, x.data_ptr(), _ptr(weight), _ptr(bias),
          y.data_ptr(), mean, mean + 4 * B * groups, B, length, C, groups, eps, _ACT[act], dt, _ptr(ws), need)
    return y, stats[0], stats[1]


def gspn_group_norm_bwd(dy, x, mean, rstd, groups: int, weight=None, bias=None, *, act: str = "none"):
    """Gradients (dx, dweight or None, dbias or None) of <dy, y>; mean, rstd: the forward's."""
    dt, B, length, C = _norm_sizes(x, groups, weight, bias, act)
    dev = x.device
    _check_tensor("dy", dy, x.shape, x.dtype, dev, _NORM)
    for name, t in (("mean", mean), ("rstd", rstd)):
        _check_tensor(name, t, (B, groups), torch.float32, dev, _NORM)
    x, dy, mean, rstd = x.contiguous(), dy.contiguous(), mean.contiguous(), rstd.contiguous()
    weight, bias = (t if t is None else t.contiguous() for t in (weight, bias))
    dx = torch.empty(x.shape, dtype=x.dtype, device=dev)
    new = torch.empty if x.numel() else torch.zeros  # an empty x leaves the parameters' gradients at zero
    dw, db = (None if t is None else new((C,), dtype=x.dtype, device=dev) for t in (weight, bias))
    need = _norm_bwd_bytes(B, length, C, groups, dt)
    ws = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
    _call(L.load().gspn_group_norm_bwd, "gspn_group_norm_bwd", dev, dy.data_ptr(), x.data_ptr(), _ptr(weight),
          _ptr(bias), mean.data_ptr(), rstd.data_ptr(), dx.data_ptr(), _ptr(dw), _ptr(db), B, length, C, groups,
          _ACT[act], dt, _ptr(ws), need)
    return dx, dw, db


class GSPNGroupNorm(torch.autograd.Function):
    """Autograd wrapper: forward and backward both run the HIP kernels."""

    @staticmethod
    def forward(ctx, x, weight, bias, groups, eps, act):
        y, mean, rstd = gspn_group_norm_fwd(x, groups, weight, bias, eps=eps, act=act)
        ctx.save_for_backward(x, weight, bias, mean, rstd)
        ctx.groups, ctx.act = groups, act
        return y

    @staticmethod
    def backward(ctx, dy):
        x, weight, bias, mean, rstd = ctx.saved_tensors
        dx, dw, db = gspn_group_norm_bwd(dy, x, mean, rstd, ctx.groups, weight, bias, act=ctx.act)
        return dx, dw, db, None, None, None


def gspn_group_norm(x, groups: int, weight=None, bias=None, eps: float = 1e-5, act: str = "none") -> torch.Tensor:
    """Differentiable group norm with an activation on a channels-last x (B, ..., C)."""
    if _needs_grad(x, weight, bias):
        return GSPNGroupNorm.apply(x, weight, bias, groups, eps, act)
    return gspn_group_norm_fwd(x, groups, weight, bias, eps=eps, act=act)[0]
