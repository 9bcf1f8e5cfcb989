"""Performance cases of the sequence operators beside the line scan: linear attention with a decay for
each head (prompts, training, single tokens) and group norm with an activation on channels-last maps.

The calls are those of a program that runs 1-D token mixing over the raster of a map: maps of
classification stages (14 to 28 a side) and diffusion latents (64 to 256 a side), prompts packed
without padding, one token for each running sequence, and the norms in front of such a layer (32
groups of channels) and behind it (a group for each head, every token on its own).

`run` makes the calls with the framework's operators where `own` is true; otherwise it computes the same in elementary
torch operations in 32 bits.
"""
from __future__ import annotations

import math

import torch

own = False

_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
_CHUNK = 64  # tokens of a chunk in the plain form


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------
def _prompt(B, T, H, Hk, Dk, Dv, dtype, decay, train=False, state=False, lens=""):
    """decay: "head" (one number for each head) or "token" (one for each token and head); state: an initial state
    goes in and the final one comes out; lens: lengths of packed sequences (then B = 1, T their sum)."""
    return {"kind": "train" if train else "prompt", "B": B, "T": T, "H": H, "Hk": Hk, "Dk": Dk, "Dv": Dv,
            "dtype": dtype, "decay": decay, "state": state, "lens": lens}


def _step(B, slots, H, Hk, Dk, Dv, dtype, decay):
    return {"kind": "step", "B": B, "slots": slots, "H": H, "Hk": Hk, "Dk": Dk, "Dv": Dv, "dtype": dtype,
            "decay": decay}


def _norm(B, L, C, G, dtype, act, train):
    return {"kind": "norm_train" if train else "norm", "B": B, "L": L, "C": C, "G": G, "dtype": dtype, "act": act}


def listed():
    lens = "1,1337,64,63,901,2048,300,17,1025,129,0,2307"
    return [
        # one sequence generating: the smallest call, where only latency counts
        {"name": "step_one_f32", **_step(1, 0, 4, 4, 64, 64, "f32", "head")},
        # a server's step: 256 running sequences in a pool of 320 states, four value heads for each key head
        {"name": "step_pool_bf16", **_step(256, 320, 16, 4, 128, 128, "bf16", "token")},
        # prompts of very different lengths packed into one call, final states kept for generation
        {"name": "prompt_packed_bf16", **_prompt(1, sum(map(int, lens.split(","))), 16, 16, 128, 128, "bf16", "token",
                                                 state=True, lens=lens)},
        # the raster of a 256 x 256 map as one long sequence: few heads, a long axis
        {"name": "prompt_raster256_bf16", **_prompt(1, 65536, 10, 10, 64, 64, "bf16", "token")},
        # training step on the raster of a 14 x 14 map, fp32, carried state (a sequence trained in pieces)
        {"name": "train_stage14_f32", **_prompt(2, 196, 12, 12, 32, 32, "f32", "token", train=True, state=True)},
        # training step of a classifier's 28 x 28 stage, 192 channels in six heads
        {"name": "train_stage28_bf16", **_prompt(32, 784, 6, 6, 32, 32, "bf16", "token", train=True)},
        # training step on 64 x 64 latents, shared query and key heads, one decay for each head
        {"name": "train_lat64_bf16", **_prompt(4, 4096, 16, 4, 128, 128, "bf16", "head", train=True)},
        # one small map in inference: latency
        {"name": "norm_stage14_f32", **_norm(1, 196, 384, 32, "f32", "silu", False)},
        # the norm and activation in front of a layer of a 128 x 128 latent
        {"name": "norm_lat128_bf16", **_norm(2, 16384, 640, 32, "bf16", "silu", False)},
        # fp32 training on a ragged map
        {"name": "norm_ragged45x77_f32_train", **_norm(4, 45 * 77, 96, 8, "f32", "silu", True)},
        # the same latent in fine-tuning
        {"name": "norm_lat128_bf16_train", **_norm(2, 16384, 640, 32, "bf16", "silu", True)},
        # behind linear attention: every token on its own, a group for each head
        {"name": "norm_heads_bf16_train", **_norm(16384, 1, 2048, 16, "bf16", "none", True)},
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges above."""
    dtype = "bf16" if rng.random() < 0.65 else "f32"
    r = rng.random()
    if r < 0.6:  # linear attention
        Hk = rng.choice([1, 2, 3, 4, 6, 8])
        H = Hk * rng.choice([1, 1, 2, 4])
        Dk = rng.choice([16, 24, 32, 40, 64, 64, 80, 128, 128])
        Dv = Dk if rng.random() < 0.7 else rng.choice([16, 33, 64, 96, 128])
        decay = rng.choice(["head", "token"])
        if r < 0.15:
            B = _log_uniform(rng, 1, 256)
            while B * H * Dk * Dv > 256 * 16 * 128 * 128:
                B = max(1, B // 2)
            return _step(B, B + rng.randint(0, 64) if rng.random() < 0.5 else 0, H, Hk, Dk, Dv, dtype, decay)
        train = r < 0.38
        if rng.random() < 0.3:  # packed
            lens, n = [], rng.randint(2, 24)
            for _ in range(n):
                lens.append(0 if rng.random() < 0.05 else _log_uniform(rng, 1, 2500))
            lens.append(_log_uniform(rng, 1, 2500))
            return _prompt(1, sum(lens), H, Hk, Dk, Dv, dtype, decay, train, rng.random() < 0.5,
                           ",".join(map(str, lens)))
        B, T = _log_uniform(rng, 1, 32), _log_uniform(rng, 1, 8192 if train else 65536)
        most = 1_000_000_000 if dtype == "f32" or T > 8192 else 4_000_000_000
        while B * T * H * Dk * Dv > most:
            B, T = (B // 2, T) if B > 1 else (1, T * 2 // 3)
        return _prompt(B, T, H, Hk, Dk, Dv, dtype, decay, train, rng.random() < 0.4)
    train, act = rng.random() < 0.5, rng.choice(["silu", "silu", "none", "gelu"])
    G = rng.choice([1, 4, 8, 16, 32, 32])
    C = G * _log_uniform(rng, 1 if G > 8 else 8, 1280 // G)
    if rng.random() < 0.3:  # tokens on their own
        L, B = 1, _log_uniform(rng, 1, 16384)
        C = max(C, 8 * G)  # a group of one or two values has nothing but its bias left
    else:
        L, B = _log_uniform(rng, 49, 65536), _log_uniform(rng, 1, 32)
    while B * L * C > 21_000_000:
        B, L = (B // 2, L) if B > 1 else (1, L // 2)
    if L > 1:
        L = max(L, -(-8 * G // C))
    return _norm(B, L, C, G, dtype, act, train)


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _randn(shape, seed, tid):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1_000_003 + tid * 7919 + 54321) & 0x7FFF_FFFF_FFFF)
    return torch.randn(shape, generator=g, device="cuda")


def prepare(case, seed):
    dt = _DTYPES[case["dtype"]]
    s = {"case": case}
    if case["kind"].startswith("norm"):
        B, L, C = case["B"], case["L"], case["C"]
        # maps with a mean of their own in every channel, as a convolution's bias leaves it
        s["x"] = (_randn((B, L, C), seed, 0) * 1.5 + 0.7 * _randn((C,), seed, 1)).to(dt)
        s["weight"] = (1 + 0.2 * _randn((C,), seed, 2)).to(dt)
        s["bias"] = (0.2 * _randn((C,), seed, 3)).to(dt)
        if case["kind"] == "norm_train":
            s["dy"] = _randn((B, L, C), seed, 4).to(dt)
            for name in ("x", "weight", "bias"):
                s[name].requires_grad_(True)
        return s
    B, H, Hk, Dk, Dv = (case[n] for n in ("B", "H", "Hk", "Dk", "Dv"))
    lead = (B,) if case["kind"] == "step" else (B, case["T"])
    s["q"] = _randn(lead + (Hk, Dk), seed, 0).to(dt)
    s["k"] = _randn(lead + (Hk, Dk), seed, 1).to(dt)
    s["v"] = _randn(lead + (H, Dv), seed, 2).to(dt)
    if case["decay"] == "head":  # memories of some ten to some thousand tokens
        s["log_decay"] = torch.log1p(-torch.exp2(-torch.linspace(3.5, 9.5, H, device="cuda")
                                                 + 0.2 * _randn((H,), seed, 3))).to(dt)
    else:  # input-dependent, of the same range; the gate of a trained layer is near one for most tokens
        s["log_decay"] = (-torch.exp(_randn(lead + (H,), seed, 3) - 4.0)).to(dt)
    if case["kind"] == "step":
        n = case["slots"] or B
        s["state"] = _randn((n, H, Dk, Dv), seed, 4)
        s["slots"] = torch.argsort(_randn((n,), seed, 5))[:B].to(torch.int32) if case["slots"] else None
        return s
    lens = [int(n) for n in case["lens"].split(",")] if case["lens"] else None
    s["lens"] = lens
    s["cu_seqlens"] = torch.tensor([sum(lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int32,
                                   device="cuda") if lens else None
    n = len(lens) if lens else B
    s["initial_state"] = _randn((n, H, Dk, Dv), seed, 4) if case["state"] else None
    if case["kind"] == "train":
        s["do"] = _randn(lead + (H, Dv), seed, 6).to(dt)
        s["dstate"] = _randn((n, H, Dk, Dv), seed, 7) if case["state"] else None
        for name in ("q", "k", "v", "log_decay", "initial_state"):
            if s[name] is not None:
                s[name].requires_grad_(True)
    return s


# ---------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------
def _pack_index(cu_seqlens, longest):
    """(sequences, longest) positions in the packed axis, and which of them are tokens."""
    at = torch.arange(longest, device=cu_seqlens.device)
    length = (cu_seqlens[1:] - cu_seqlens[:-1]).long()
    return cu_seqlens[:-1, None].long() + at, at < length[:, None]


def _plain_linattn(q, k, v, log_decay, scale, initial_state, cu_seqlens=None, lens=None):
    """Chunks of 64 tokens: products within a chunk, and the states between chunks as one product with the matrix of the
    chunks' decays.  Returns o and the final state, fp32."""
    H, Dv = v.shape[2:]
    q, k, v = q.float(), k.float(), v.float()
    group = H // q.shape[2]
    a = log_decay.float().expand(v.shape[:3])
    if cu_seqlens is not None:
        at, used = _pack_index(cu_seqlens, max(max(lens), 1))
        at = torch.where(used, at, torch.zeros_like(at))
        q, k, v, a = (t[0][at] * used.reshape(used.shape + (1,) * (t.dim() - 2)) for t in (q, k, v, a))
    B, T = q.shape[:2]
    C = _CHUNK
    n = -(-T // C)
    pad = n * C - T

    def chunks(t):  # (B, T, heads, D) -> (B, heads, n, C, D)
        t = torch.cat([t, t.new_zeros((B, pad) + t.shape[2:])], 1) if pad else t
        return t.unflatten(1, (n, C)).permute(0, 3, 1, 2, 4)

    q, k = (chunks(t).repeat_interleave(group, 1) for t in (q, k))
    v, a = chunks(v), chunks(a[..., None])[..., 0]
    G = a.cumsum(-1)
    lower = torch.ones((C, C), dtype=torch.bool, device=q.device).tril()
    D = torch.exp((G[..., :, None] - G[..., None, :]).masked_fill(~lower, -math.inf))
    o = (q @ k.transpose(-1, -2) * D) @ v
    total = G[..., -1]
    kv = (k * torch.exp(total[..., None] - G)[..., None]).transpose(-1, -2) @ v
    # the decay from the end of chunk j to the end of chunk i: sums that start behind j, so that long sequences keep
    # their digits; the state before chunk c is row c of the product, the final one row n
    upto = torch.ones((n, n), dtype=torch.bool, device=q.device).tril()
    between = total[..., :, None].expand(B, H, n, n).tril(-1).cumsum(-2)
    M = torch.cat([total.new_zeros((B, H, 1, n)), torch.exp(between.masked_fill(~upto, -math.inf))], -2)
    E = torch.cat([total.new_zeros((B, H, 1)), total.cumsum(-1)], -1)
    S = (M @ kv.flatten(-2)).unflatten(-1, kv.shape[-2:])
    if initial_state is not None:
        S = S + torch.exp(E)[..., None, None] * initial_state[:, :, None]
    o = scale * (o + (q * torch.exp(G)[..., None]) @ S[:, :, :n])
    o = o.permute(0, 2, 3, 1, 4).reshape(B, n * C, H, Dv)[:, :T]
    if cu_seqlens is not None:
        o = o[used][None]  # the tokens in their packed order
    return o, S[:, :, n]


def _plain_step(q, k, v, log_decay, scale, state, slots):
    group = v.shape[1] // q.shape[1]
    q, k = (t.float().repeat_interleave(group, 1) for t in (q, k))
    decay = torch.exp(log_decay.float()).expand(v.shape[:2])
    old = state if slots is None else state[slots.long()]
    new = decay[..., None, None] * old + k[..., :, None] * v.float()[..., None, :]
    if slots is None:
        state.copy_(new)
    else:
        state[slots.long()] = new
    return (scale * (q[..., None, :] @ new)[..., 0, :]).to(v.dtype)


def _plain_norm(x, groups, weight, bias, eps, act):
    B, L, C = x.shape
    t = x.float().view(B, L, groups, C // groups)
    mean = t.mean((1, 3), keepdim=True)
    t = t - mean
    rstd = torch.rsqrt((t * t).mean((1, 3), keepdim=True) + eps)
    z = (t * rstd).view(B, L, C) * weight.float() + bias.float()
    if act == "silu":
        z = z * torch.sigmoid(z)
    elif act == "gelu":
        z = 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    return z.to(x.dtype)


_EPS = 1e-5


def run(s):
    c = s["case"]
    if own:
        from paper_2501_12381_amd import ops
    if c["kind"].startswith("norm"):
        if c["kind"] == "norm":
            with torch.no_grad():
                if own:
                    return ops.gspn_group_norm(s["x"], c["G"], s["weight"], s["bias"], eps=_EPS, act=c["act"])
                return _plain_norm(s["x"], c["G"], s["weight"], s["bias"], _EPS, c["act"])
        if own:
            y = ops.gspn_group_norm(s["x"], c["G"], s["weight"], s["bias"], eps=_EPS, act=c["act"])
        else:
            y = _plain_norm(s["x"], c["G"], s["weight"], s["bias"], _EPS, c["act"])
        dx, dw, db = torch.autograd.grad(y, (s["x"], s["weight"], s["bias"]), s["dy"])
        return {"y": y, "dx": dx, "dweight": dw, "dbias": db}
    scale = c["Dk"] ** -0.5
    if c["kind"] == "step":
        if own:
            o = ops.gspn_linattn_step(s["q"], s["k"], s["v"], s["log_decay"], s["state"], slots=s["slots"])
        else:
            o = _plain_step(s["q"], s["k"], s["v"], s["log_decay"], scale, s["state"], s["slots"])
        return {"o": o, "state": s["state"]}
    if own:
        got = ops.gspn_linattn(s["q"], s["k"], s["v"], s["log_decay"], initial_state=s["initial_state"],
                               return_state=c["state"], cu_seqlens=s["cu_seqlens"])
        o, final = got if c["state"] else (got, None)
    else:
        o, final = _plain_linattn(s["q"], s["k"], s["v"], s["log_decay"], scale, s["initial_state"], s["cu_seqlens"],
                                  s["lens"])
        o = o.to(s["v"].dtype)
    if c["kind"] == "prompt":
        return {"o": o, "state": final} if c["state"] else {"o": o}
    names = ["q", "k", "v", "log_decay"] + (["initial_state"] if c["state"] else [])
    outs, grads = ((o, final), (s["do"], s["dstate"])) if c["state"] else ((o,), (s["do"],))
    got = torch.autograd.grad(outs, [s[n] for n in names], grads)
    out = {"o": o, **{"d" + n: g for n, g in zip(names, got)}}
    if c["state"]:
        out["state"] = final
    return out


def work(case):
    es = _DTYPES[case["dtype"]].itemsize
    if case["kind"].startswith("norm"):
        n = case["B"] * case["L"] * case["C"]
        # x in, y out; training: dy in and dx out too
        return {"bytes": es * n * (4 if case["kind"] == "norm_train" else 2),
                "flops": n * (30 if case["kind"] == "norm_train" else 12)}
    B, H, Hk, Dk, Dv = (case[n] for n in ("B", "H", "Hk", "Dk", "Dv"))
    n = B * (1 if case["kind"] == "step" else case["T"])  # tokens
    io = n * (2 * Hk * Dk + 2 * H * Dv + (H if case["decay"] == "token" else 0))
    if case["kind"] == "step":
        return {"bytes": es * io + 8 * B * H * Dk * Dv, "flops": 5 * n * H * Dk * Dv}
    seqs = len(case["lens"].split(",")) if case["lens"] else B
    states = 4 * seqs * H * Dk * Dv if case["state"] else 0
    # the recurrence's count: the state's update and its product with q; training: q's, k's, v's and the state's
    # gradients and the forward's states again
    if case["kind"] == "prompt":
        return {"bytes": es * io + 2 * states, "flops": 4 * n * H * Dk * Dv}
    # do in, dq, dk, dv and dlog_decay out, o out
    return {"bytes": 2 * es * io + 4 * states, "flops": 14 * n * H * Dk * Dv}


# ---------------------------------------------------------------------------
# the same in 64 bits
# ---------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    d = {k: t.detach().double() if isinstance(t, torch.Tensor) and t.is_floating_point() else t for k, t in s.items()}
    if case["kind"].startswith("norm"):
        B, L, C, G = (case[n] for n in ("B", "L", "C", "G"))
        m = L * (C // G)
        per = lambda t: t.reshape(B, L, G, C // G).sum((1, 3))[:, None, :, None].expand(  # noqa: E731
            B, L, G, C // G).reshape(B, L, C) / m
        mu = per(d["x"])
        var = per((d["x"] - mu) ** 2)
        r = (var + _EPS) ** -0.5
        xh = (d["x"] - mu) * r
        z = xh * d["weight"] + d["bias"]
        if case["act"] == "silu":
            g = torch.sigmoid(z)
            y, slope = z * g, g * (1 + z * (1 - g))
        elif case["act"] == "gelu":
            cdf = 0.5 * (1 + torch.erf(z / math.sqrt(2)))
            y, slope = z * cdf, cdf + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
        else:
            y, slope = z, torch.ones_like(z)
        if case["kind"] == "norm":
            return y
        dz = d["dy"] * slope
        dxh = dz * d["weight"]
        dx = r * (dxh - per(dxh) - xh * per(dxh * xh))
        return {"y": y, "dx": dx, "dweight": (dz * xh).sum((0, 1)), "dbias": dz.sum((0, 1))}
    H, Hk, Dk = case["H"], case["Hk"], case["Dk"]
    scale = 1 / math.sqrt(Dk)
    if case["kind"] == "step":
        rows = s["slots"].long() if s["slots"] is not None else torch.arange(case["B"], device="cuda")
        q, k = (d[n].repeat_interleave(H // Hk, 1) for n in ("q", "k"))
        state = d["state"].clone()
        decay = torch.exp(d["log_decay"]) * torch.ones((case["B"], H), dtype=torch.float64, device="cuda")
        state[rows] = state[rows] * decay[:, :, None, None] + torch.einsum("bhi,bhj->bhij", k, d["v"])
        return {"o": scale * torch.einsum("bhi,bhij->bhj", q, state[rows]), "state": state}
    # the recurrence, token by token; packed sequences side by side, the longest first
    lens = s["lens"] or [case["T"]] * case["B"]
    order = sorted(range(len(lens)), key=lambda i: -lens[i])
    starts = [sum(lens[:i]) for i in range(len(lens))]
    start = torch.tensor([starts[i] for i in order], device="cuda")
    live = [sum(n > t for n in lens) for t in range(max(lens))]
    flat = {n: d[n].reshape((-1,) + d[n].shape[2:]) for n in ("q", "k", "v")}
    q, k = (flat[n].repeat_interleave(H // Hk, 1) for n in ("q", "k"))
    v = flat["v"]
    a = (d["log_decay"] * torch.ones(d["v"].shape[:3], dtype=torch.float64, device="cuda")).reshape(-1, H)
    decay = torch.exp(a)
    rank = torch.tensor([order.index(i) for i in range(len(lens))], device="cuda")
    zero = torch.zeros((len(lens), H, Dk, case["Dv"]), dtype=torch.float64, device="cuda")
    S = d["initial_state"][torch.tensor(order, device="cuda")].clone() if case["state"] else zero.clone()
    train = case["kind"] == "train"
    o, dq = torch.zeros_like(v), torch.zeros_like(q)
    do = d["do"].reshape(v.shape) if train else None
    for t in range(max(lens)):
        i, m = start[:live[t]] + t, live[t]
        S[:m] = S[:m] * decay[i][..., None, None] + k[i][..., :, None] * v[i][..., None, :]
        o[i] = scale * torch.matmul(q[i][..., None, :], S[:m])[..., 0, :]
        if train:
            dq[i] = scale * torch.matmul(S[:m], do[i][..., :, None])[..., 0]
    final = S[rank]
    out = {"o": o.reshape(s["v"].shape)}
    if case["state"]:
        out["state"] = final
    if not train:
        return out
    dk, dv = torch.zeros_like(k), torch.zeros_like(v)
    dS = d["dstate"][torch.tensor(order, device="cuda")].clone() if case["state"] else zero.clone()
    # the decay's gradient: d/dG_t = q_t . dq_t - k_t . dk_t, summed from the end, where the final state adds <S, dS>
    run_sum = (S * dS).sum((2, 3))
    da = torch.zeros_like(a)
    for t in range(max(lens) - 1, -1, -1):
        i, m = start[:live[t]] + t, live[t]
        dS[:m] += scale * q[i][..., :, None] * do[i][..., None, :]
        dk[i] = torch.matmul(dS[:m], v[i][..., :, None])[..., 0]
        dv[i] = torch.matmul(k[i][..., None, :], dS[:m])[..., 0, :]
        run_sum[:m] += (q[i] * dq[i]).sum(-1) - (k[i] * dk[i]).sum(-1)
        da[i] = run_sum[:m]
        dS[:m] *= decay[i][..., None, None]
    share = lambda g: g.unflatten(1, (Hk, H // Hk)).sum(2).reshape(s["q"].shape)  # noqa: E731
    out.update(dq=share(dq), dk=share(dk), dv=dv.reshape(s["v"].shape),
               dlog_decay=da.sum(0) if case["decay"] == "head" else da.reshape(s["log_decay"].shape))
    if case["state"]:
        out["dinitial_state"] = dS[rank]
    return out
