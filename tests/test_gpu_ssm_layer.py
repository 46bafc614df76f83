"""The operators together, as a layer uses them: one projection, of whose rows a slice goes
through the short convolution and becomes x, B and C, B and C take rotary positions, the
state space scan, the gated norm of its heads, the output projection and the residual;
forward, backward, packed prompts, and decoding on the states and inputs they left.

f32 throughout, against the same layer in 64 bits.  Each operator is within 3.8e-6 of its
inputs' exact result (norms 1e-5), the projections sum up to 388 terms (20 * 4 * 2^-24 =
4.7e-6), and a gradient passes each of the six stages twice: 2 * 6 * 1e-5 = 1.2e-4.
"""
import pytest
import torch

from gdr_util import rel
from paper_2606_27229_amd import carve
from ssm_util import rotary_reference, ssm_tokens

pytestmark = pytest.mark.gpu

B, T, G, H, P, N, W, C = 2, 150, 2, 4, 32, 32, 4, 96
TOL = 1.2e-4
INNER, CONV = H * P, H * P + 2 * G * N
CUTS = [INNER, CONV, H]   # gate | convolution's inputs | steps


def weights():
    gen = torch.Generator().manual_seed(1)
    r = lambda *s: torch.randn(s, generator=gen)
    width = -(-sum(CUTS) // 4) * 4
    return {"x": r(B, T, C), "in": r(C, width) / C ** 0.5, "taps": r(CONV, W) / 2, "bias": 0.1 * r(CONV), "A": -1 - 15 * r(H).abs(),
            "D": r(H), "dt_bias": r(H) - 3, "heads": 1 + 0.1 * r(INNER), "out": r(INNER, C) / INNER ** 0.5, "dX": r(B, T, C)}


LEAVES = ("x", "in", "taps", "bias", "A", "D", "dt_bias", "heads", "out")
FREQ = carve.rotary_frequencies(N, device="cpu")


class Turned(torch.autograd.Function):
    """The rotary map in 64 bits and its transpose."""

    @staticmethod
    def forward(ctx, x, pos):
        ctx.pos = pos
        return rotary_reference(x, FREQ, pos, False, 1.0)

    @staticmethod
    def backward(ctx, g):
        return rotary_reference(g, FREQ, ctx.pos, False, 1.0, -1), None


def exact(w, lens=None):
    """lens: T rows of batch element 0 are packed sequences."""
    w = {n: t.double().requires_grad_(n in LEAVES) for n, t in w.items()}
    spans = [(b, 0, T) for b in range(B)] if lens is None else [(0, sum(lens[:i]), n) for i, n in enumerate(lens)]
    X, states, loss = [], [], 0.0
    for b, at, n in spans:
        x = w["x"][b, at:at + n]
        z, xbc, dt = (x @ w["in"])[:, :sum(CUTS)].split(CUTS, -1)
        past = torch.cat([torch.zeros(W - 1, CONV, dtype=torch.float64), xbc])
        p = torch.stack([(past[t:t + W] * w["taps"].T).sum(0) for t in range(n)]) + w["bias"]
        xs, Bm, Cm = (p * torch.sigmoid(p)).split([INNER, G * N, G * N], -1)
        pos = torch.arange(n)[None]
        Bm, Cm = (Turned.apply(t.unflatten(-1, (G, N))[None], pos)[0] for t in (Bm, Cm))
        y, S = ssm_tokens(xs.unflatten(-1, (H, P)), dt, w["A"], Bm, Cm, w["D"], w["dt_bias"], torch.zeros(H, P, N, dtype=torch.float64), True)
        y = y / torch.sqrt(y.square().mean(-1, keepdim=True) + 1e-6)
        y = y.flatten(1) * w["heads"] * z * torch.sigmoid(z)
        X.append(x + y @ w["out"])
        states.append(S)
        loss = loss + (X[-1] * w["dX"][b, at:at + n]).sum()
    grads = torch.autograd.grad(loss, [w[n] for n in LEAVES])
    return torch.cat(X).detach(), torch.stack(states).detach(), dict(zip(LEAVES, grads))


def parts(u):
    """Gate, convolution's inputs and steps: slices of the projection's rows."""
    return u[..., :INNER], u[..., INNER:INNER + CONV], u[..., INNER + CONV:sum(CUTS)]


def split(xbc):
    return (xbc[..., :INNER].unflatten(-1, (H, P)), xbc[..., INNER:INNER + G * N].unflatten(-1, (G, N)),
            xbc[..., INNER + G * N:].unflatten(-1, (G, N)))


def forward(w, x, freq, off=None):
    z, xbc, dt = parts(x @ w["in"])
    act, x_T = carve.short_conv_fwd(xbc, w["taps"], bias=w["bias"], offsets=off)
    xs, Bm, Cm = split(act)
    # (in place: B and C are slices of the convolution's outputs)
    carve.rotary_fwd(Cm, Bm, freq, offsets=off, out={"q": Cm, "k": Bm})
    scan = (xs, dt, w["A"], Bm, Cm)
    y, S, S_c = carve.ssm_chunk_fwd(*scan, D=w["D"], dt_bias=w["dt_bias"], offsets=off)
    z = z.contiguous()
    h, _ = carve.block_norm_fwd(y.flatten(2), w["heads"], groups=H, gate=z)
    X = x + h @ w["out"]
    return X, S, x_T, (z, xbc, scan, y, S_c, h)


def backward(w, x, freq, kept, dX, off=None):
    z, xbc, scan, y, S_c, h = kept
    r = carve.block_norm_bwd(y.flatten(2), w["heads"], dX @ w["out"].T, groups=H, gate=z)
    g = carve.ssm_chunk_bwd(*scan, S_c, r["dy"].unflatten(2, (H, P)), D=w["D"], dt_bias=w["dt_bias"], offsets=off, want_dS0=False)
    dC, dB = carve.rotary_bwd(g["dCm"], g["dBm"], freq, offsets=off)
    dact = torch.cat([g["dx"].flatten(2), dB.flatten(2), dC.flatten(2)], -1)
    c = carve.short_conv_bwd(xbc, w["taps"], dact, bias=w["bias"], offsets=off)
    du = torch.zeros(*x.shape[:2], w["in"].shape[1], device="cuda")
    for to, t in zip(parts(du), (r["dgate"], c["dx"], g["ddt"])):
        to.copy_(t)
    return {"x": dX + du @ w["in"].T, "in": x.flatten(0, 1).T @ du.flatten(0, 1), "taps": c["dweight"], "bias": c["dbias"], "A": g["dA"],
            "D": g["dD"], "dt_bias": g["ddt_bias"], "heads": r["dweight"], "out": h.flatten(0, 1).T @ dX.flatten(0, 1)}


@pytest.mark.parametrize("lens", [None, [70, 1, 79]])
def test_layer_forward_backward(lens):
    w0 = weights()
    X0, S0, g0 = exact(w0, lens)
    w, freq = {n: t.cuda() for n, t in w0.items()}, FREQ.cuda()
    seqs = slice(None) if lens is None else slice(0, 1)
    off = None if lens is None else torch.tensor([0] + lens).cumsum(0).int().cuda()
    x, dX = w["x"][seqs].contiguous(), w["dX"][seqs].contiguous()
    X, S, _, kept = forward(w, x, freq, off)
    assert rel(X.flatten(0, 1), X0) <= TOL and rel(S, S0) <= TOL
    grads = backward(w, x, freq, kept, dX, off)
    want = dict(g0, x=g0["x"][seqs])
    errs = {n: rel(grads[n], want[n]) for n in LEAVES}
    print({n: float("%.2g" % e) for n, e in errs.items()}, flush=True)
    assert max(errs.values()) <= TOL, errs


def test_layer_decodes_on_from_a_prompt():
    """130 tokens at once, then 20 one by one through the same layer."""
    w0 = weights()
    X0, S0, _ = exact(w0)
    w, freq = {n: t.cuda() for n, t in w0.items()}, FREQ.cuda()
    slots = torch.tensor([3, 1], dtype=torch.int32, device="cuda")
    states, inputs = torch.zeros(5, H, P, N, device="cuda"), torch.zeros(5, W - 1, CONV, device="cuda")
    X, S, x_T, _ = forward(w, w["x"][:, :130].contiguous(), freq)
    states[slots.long()], inputs[slots.long()] = S, x_T
    out = [X]
    for t in range(130, T):
        x = w["x"][:, t:t + 1]
        z, xbc, dt = parts(x @ w["in"])
        xs, Bm, Cm = split(carve.short_conv_step(xbc, w["taps"], inputs, slots, bias=w["bias"]))
        Cm, Bm = carve.rotary_fwd(Cm, Bm, freq, start=torch.full((B,), t, dtype=torch.int32, device="cuda"))
        y = carve.ssm_step(xs, dt, w["A"], Bm, Cm, states, slots, D=w["D"], dt_bias=w["dt_bias"])
        h, _ = carve.block_norm_fwd(y.flatten(2), w["heads"], groups=H, gate=z.contiguous())
        out.append(x + h @ w["out"])
    assert rel(torch.cat(out, 1).flatten(0, 1), X0) <= TOL
    assert rel(states[slots.long()], S0) <= TOL
    assert not states[[0, 2, 4]].any() and not inputs[[0, 2, 4]].any()
