"""The short causal convolution, rotary positions and the selective state space scan from
their definitions, in 64 bits on the CPU (row by row; gradients by autograd), and seeded
inputs for them."""
import torch

# A bf16 result is off by half a step, 2^-8 of itself at most, and by what was left out of
# its operands (2^-16).  An f32 result: sums of at most 256 terms, each rounded to 2^-24,
# leave 16 * 2^-24 at random, times 4 for terms that are larger than their sum.
TOL = {torch.bfloat16: 2.0 ** -8 + 2.0 ** -14, torch.float32: 4 * 16 * 2.0 ** -24}


def spans(x, lens, first=0):
    """(batch, first row, rows) of every sequence of rows x [B, T, ...]."""
    if lens is None:
        return [(b, 0, x.shape[1]) for b in range(x.shape[0])]
    out = []
    for n in lens:
        out.append((0, first, n))
        first += n
    return out


def randn(gen, *shape):
    return torch.randn(shape, generator=gen)


def grads_of(loss, leaves):
    have = {n: t for n, t in leaves.items() if t is not None}
    got = torch.autograd.grad(loss, list(have.values()), allow_unused=True)
    return {"d" + n: torch.zeros_like(t) if g is None else g for (n, t), g in zip(have.items(), got)}


def conv_inputs(B, T, C, W, dtype, seed, *, seqs=None, state=True, bias=True, act="silu"):
    gen = torch.Generator().manual_seed(seed)
    seqs = B if seqs is None else seqs
    return {"x": randn(gen, B, T, C).to(dtype), "weight": randn(gen, C, W) * W ** -0.5,
            "bias": 0.3 * randn(gen, C) if bias else None, "x0": randn(gen, seqs, W - 1, C).to(dtype) if state else None,
            "dy": randn(gen, B, T, C).to(dtype), "dx_T": randn(gen, seqs, W - 1, C).to(dtype) if state else None, "act": act}


def conv_reference(x, lens=None, first=0):
    """Outputs and gradients of a dict of conv_inputs; rows of no sequence are zero."""
    d = {n: None if x[n] is None else x[n].double().requires_grad_() for n in ("x", "weight", "bias", "x0")}
    C, W = d["weight"].shape
    y, last, loss = torch.zeros_like(d["x"]), [], 0.0
    for i, (b, at, n) in enumerate(spans(x["x"], lens, first)):
        past = torch.zeros(W - 1, C, dtype=torch.float64) if d["x0"] is None else d["x0"][i]
        z = torch.cat([past, d["x"][b, at:at + n]])
        p = torch.stack([(z[t:t + W] * d["weight"].T).sum(0) for t in range(n)]) if n else z[:0]
        if d["bias"] is not None:
            p = p + d["bias"]
        o = p * torch.sigmoid(p) if x["act"] else p
        loss = loss + (o * x["dy"][b, at:at + n].double()).sum()
        last.append(z[n:])
        if x["dx_T"] is not None:
            loss = loss + (z[n:] * x["dx_T"][i].double()).sum()
        y = y.index_put((torch.tensor(b), torch.arange(at, at + n)), o.detach())
    return {"y": y.detach(), "x_T": torch.stack(last).detach(), **grads_of(loss, d)}


def rotary_reference(x, freq, pos, interleaved, amplitude, sign=1):
    """x [B, T, H, D] turned by pos [B, T] * freq."""
    half = freq.numel()
    z = pos.double()[:, :, None, None] * freq.double()
    x = x.double()
    at = torch.arange(half)
    ia, ib = (2 * at, 2 * at + 1) if interleaved else (at, at + half)
    a, b = x[..., ia], x[..., ib]
    out = x.clone()
    out[..., ia] = amplitude * (a * torch.cos(z) - sign * b * torch.sin(z))
    out[..., ib] = amplitude * (b * torch.cos(z) + sign * a * torch.sin(z))
    return out


def ssm_inputs(B, T, G, H, P, N, dtype, seed, *, seqs=None, state=True, skip=True, bias=True, decay=1.0, dst=True, softplus=True):
    """Steps of about 0.001 to 1, decays of `decay` times 1 to 16 of them."""
    gen = torch.Generator().manual_seed(seed)
    seqs = B if seqs is None else seqs
    x = {"x": randn(gen, B, T, H, P).to(dtype), "Bm": randn(gen, B, T, G, N).to(dtype), "Cm": randn(gen, B, T, G, N).to(dtype)}
    raw = 1.5 * randn(gen, B, T, H) - (3 if not bias else 0)
    x["dt"] = (raw if softplus else torch.nn.functional.softplus(raw - 2)).to(dtype)
    x["dt_bias"] = (randn(gen, H) - 3 if softplus else 0.01 * torch.rand(H, generator=gen)) if bias else None
    x["A"] = -decay * (1 + 15 * torch.rand(H, generator=gen))
    x["D"] = randn(gen, H) if skip else None
    x["S0"] = 0.3 * randn(gen, seqs, H, P, N) if state else None
    x["dy"] = randn(gen, B, T, H, P).to(dtype)
    x["dS_T"] = 0.3 * randn(gen, seqs, H, P, N) if dst else None
    x["softplus"] = softplus
    return x


SSM_LEAVES = ("x", "dt", "A", "Bm", "Cm", "D", "dt_bias", "S0")


def ssm_tokens(x, dt, A, Bm, Cm, D, dt_bias, S, softplus):
    """One sequence, token by token: x [T, H, P], S [H, P, N]; all float64.  (y, S_T)."""
    rep = x.shape[1] // Bm.shape[1]
    Bm, Cm = Bm.repeat_interleave(rep, 1), Cm.repeat_interleave(rep, 1)
    step = dt if dt_bias is None else dt + dt_bias
    if softplus:
        step = torch.nn.functional.softplus(step, threshold=1e9)
    y = []
    for t in range(x.shape[0]):
        S = torch.exp(step[t] * A)[:, None, None] * S + (step[t, :, None] * x[t])[..., None] * Bm[t, :, None]
        y.append((S * Cm[t, :, None]).sum(-1))
    y = torch.stack(y) if y else x[:0]
    return (y if D is None else y + D[:, None] * x), S


def ssm_decay_terms(x):
    """sum_t |d_t da_t| of every head, the magnitudes of the terms of dA (one dense sequence)."""
    d = {n: None if x[n] is None else x[n].double() for n in SSM_LEAVES}
    T = x["x"].shape[1]
    A = d["A"].expand(T, -1).clone().requires_grad_()
    S, rows = d["S0"][0], []
    for t in range(T):
        o, S = ssm_tokens(d["x"][0, t:t + 1], d["dt"][0, t:t + 1], A[t], d["Bm"][0, t:t + 1], d["Cm"][0, t:t + 1], d["D"], d["dt_bias"],
                          S, x["softplus"])
        rows.append(o)
    loss = (torch.cat(rows) * x["dy"][0].double()).sum() + (S * x["dS_T"][0].double()).sum()
    return torch.autograd.grad(loss, A)[0].abs().sum(0)


def ssm_reference(x, lens=None, first=0, grads=True):
    """Outputs and gradients of a dict of ssm_inputs; rows of no sequence are zero."""
    d = {n: None if x[n] is None else x[n].double().requires_grad_(grads) for n in SSM_LEAVES}
    H, P, N = x["x"].shape[2], x["x"].shape[3], x["Bm"].shape[3]
    y, last, loss = torch.zeros_like(d["x"]).detach(), [], 0.0
    for i, (b, at, n) in enumerate(spans(x["x"], lens, first)):
        rows = slice(at, at + n)
        S = torch.zeros(H, P, N, dtype=torch.float64) if d["S0"] is None else d["S0"][i]
        o, S = ssm_tokens(d["x"][b, rows], d["dt"][b, rows], d["A"], d["Bm"][b, rows], d["Cm"][b, rows], d["D"], d["dt_bias"], S,
                          x["softplus"])
        loss = loss + (o * x["dy"][b, rows].double()).sum()
        if x["dS_T"] is not None:
            loss = loss + (S * x["dS_T"][i].double()).sum()
        last.append(S.detach())
        y[b, rows] = o.detach()
    out = {"y": y, "S_T": torch.stack(last)}
    return out | grads_of(loss, d) if grads else out
