"""The gated delta rule and the block norm from their definitions, in 64 bits on the
CPU (token by token; gradients by autograd), and seeded inputs for both."""
import numpy as np
import torch


def gdr_tokens(q, k, v, g, beta, S, scale):
    """One sequence batch, token by token: q, k [B,T,Hk,Dk], v [B,T,Hv,Dv], g, beta
    [B,T,Hv], S [B,Hv,Dv,Dk]; all float64.  Returns (o, S_T)."""
    rep = v.shape[2] // q.shape[2]
    q, k = q.repeat_interleave(rep, 2), k.repeat_interleave(rep, 2)
    o = []
    for t in range(q.shape[1]):
        S = S * torch.exp(g[:, t])[..., None, None]
        u = beta[:, t, :, None] * (v[:, t] - torch.einsum("bhvk,bhk->bhv", S, k[:, t]))
        S = S + u[..., :, None] * k[:, t, :, None, :]
        o.append(scale * torch.einsum("bhvk,bhk->bhv", S, q[:, t]))
    return (torch.stack(o, 1) if o else v[:, :0] * 0), S


def gdr_reference(x, lens=None, grads=True):
    """x: dict of CPU tensors (q, k, v, g, beta, S0 or None, dO, dS_T or None, scale).
    lens: packed sequences.  Returns a dict of float64 outputs and gradients (rows of
    no sequence are zero)."""
    names = ("q", "k", "v", "g", "beta")
    d = {n: x[n].double().requires_grad_(grads) for n in names}
    B, T, Hv, Dv = x["v"].shape
    Dk = x["q"].shape[3]
    seqs = B if lens is None else len(lens)
    S0 = (x["S0"].double() if x.get("S0") is not None else torch.zeros(seqs, Hv, Dv, Dk, dtype=torch.float64))
    S0 = S0.clone().requires_grad_(grads)
    if lens is None:
        o, S_T = gdr_tokens(*(d[n] for n in names), S0, x["scale"])
    else:
        parts, states, at = [], [], x.get("first", 0)
        parts.append(torch.zeros(1, at, Hv, Dv, dtype=torch.float64))
        for i, n in enumerate(lens):
            oi, si = gdr_tokens(*(d[m][:, at:at + n] for m in names), S0[i:i + 1], x["scale"])
            parts.append(oi)
            states.append(si)
            at += n
        parts.append(torch.zeros(1, T - at, Hv, Dv, dtype=torch.float64))
        o, S_T = torch.cat(parts, 1), torch.cat(states, 0)
    out = {"o": o.detach(), "S_T": S_T.detach()}
    if grads:
        loss = (o * x["dO"].double()).sum()
        if x.get("dS_T") is not None:
            loss = loss + (S_T * x["dS_T"].double()).sum()
        got = torch.autograd.grad(loss, [*(d[n] for n in names), S0], allow_unused=True)
        for n, t, like in zip((*names, "S0"), got, [*(d[n] for n in names), S0]):
            out["d" + n] = torch.zeros_like(like) if t is None else t
    return out


def gdr_inputs(B, T, Hk, Hv, Dk, Dv, dtype, seed, *, seqs=None, state=True, decay=-3.0, scale=None, dst=True):
    """Unit keys and queries, decays exp(-softplus(1.5 n + decay)), write strengths in
    (0, 1); rounded to dtype, on the CPU."""
    gen = torch.Generator().manual_seed(seed)

    def randn(*shape):
        return torch.randn(shape, generator=gen)

    seqs = B if seqs is None else seqs
    x = {n: torch.nn.functional.normalize(randn(B, T, Hk, Dk), dim=-1).to(dtype) for n in ("q", "k")}
    x["v"] = randn(B, T, Hv, Dv).to(dtype)
    x["g"] = -torch.nn.functional.softplus(1.5 * randn(B, T, Hv) + decay)
    x["beta"] = torch.sigmoid(randn(B, T, Hv)).to(dtype)
    x["S0"] = 0.3 * randn(seqs, Hv, Dv, Dk) if state else None
    x["dO"] = randn(B, T, Hv, Dv).to(dtype)
    x["dS_T"] = 0.3 * randn(seqs, Hv, Dv, Dk) if dst else None
    x["scale"] = Dk ** -0.5 if scale is None else scale
    return x


def cuda(x):
    return {n: (t.cuda() if isinstance(t, torch.Tensor) else t) for n, t in x.items()}


def rel(a, b):
    """2-norm of the difference over the 2-norm of b (0 where both are zero)."""
    a, b = a.detach().cpu().double(), b.detach().double()
    n = float(torch.linalg.vector_norm(b))
    d = float(torch.linalg.vector_norm(a - b))
    return d / n if n else d


def norm_reference(x):
    """The block norm of a dict of CPU tensors in 64 bits: x, h and the gradients."""
    names = ("y", "weight", "gate", "residual", "scale", "next_weight")
    d = {n: None if x.get(n) is None else x[n].double().requires_grad_() for n in names}
    rows, N = x["y"].shape
    y = d["y"].reshape(rows, x["groups"], -1)
    t = (y / torch.sqrt(y.square().mean(-1, keepdim=True) + x["eps"])).reshape(rows, N) * d["weight"]
    if d["gate"] is not None:
        s = torch.sigmoid(d["gate"])
        t = t * (d["gate"] * s if x["gate_act"] == "silu" else s)
    if d["scale"] is not None:
        t = t * d["scale"]
    X = t if d["residual"] is None else x["alpha"] * d["residual"] + t
    h = None
    if d["next_weight"] is not None:
        h = X / torch.sqrt(X.square().mean(-1, keepdim=True) + x["eps"]) * d["next_weight"]
    loss = 0.0
    if x.get("dx") is not None:
        loss = loss + (X * x["dx"].double()).sum()
    if h is not None:
        loss = loss + (h * x["dh"].double()).sum()
    have = [n for n in names if d[n] is not None]
    out = {"d" + n: t for n, t in zip(have, torch.autograd.grad(loss, [d[n] for n in have]))}
    out["x"] = X.detach()
    if h is not None:
        out["h"] = h.detach()
    return out


def norm_inputs(rows, N, dtype, seed, *, groups=1, gate="silu", residual=True, scale=True, next=True, dx=True, eps=1e-6,
                alpha=0.75):
    rng = np.random.Generator(np.random.PCG64(seed))

    def randn(*shape):
        return torch.from_numpy(rng.standard_normal(shape, dtype=np.float32))

    x = {"y": (randn(rows, N) * torch.exp(randn(rows, 1))).to(dtype), "weight": 1 + 0.1 * randn(N), "groups": groups,
         "gate": randn(rows, N).to(dtype) if gate else None, "gate_act": gate or "silu", "alpha": alpha, "eps": eps,
         "residual": (2 * randn(rows, N)).to(dtype) if residual else None,
         "scale": 0.5 + 0.2 * randn(N) if scale else None, "next_weight": 1 + 0.1 * randn(N) if next else None,
         "dx": randn(rows, N).to(dtype) if dx else None, "dh": randn(rows, N).to(dtype) if next else None}
    return x
