"""The operators together, as a layer uses them: projections, the gated delta rule, the
gated norm of every head, the output projection, then the norm / residual / next norm
around the block; forward, backward, and decoding on the state the forward left.

f32 throughout, against the same layer in 64 bits.  Each operator is within 1.2e-5 (the
rule) and 1e-5 (norms) of its inputs' exact result, the projections sum up to 256 terms
(1.6e-5), and a gradient passes each of the five stages twice: 2 * 5 * 1.6e-5 = 1.6e-4.
"""
import pytest
import torch

from paper_2606_27229_amd import carve
from tests.gdr_util import gdr_tokens, rel

pytestmark = pytest.mark.gpu

B, T, H, D, C = 2, 150, 4, 64, 256
TOL = 1.6e-4


def weights():
    gen = torch.Generator().manual_seed(1)
    r = lambda *s: torch.randn(s, generator=gen)
    w = {n: r(C, H * D) / C ** 0.5 for n in ("q", "k", "v", "z", "o")}
    w.update(ga=r(C, H) / C ** 0.5, gb=r(C, H) / C ** 0.5, heads=1 + 0.1 * r(H * D), post=1 + 0.1 * r(C), scale=0.5 + 0.1 * r(C),
             next=1 + 0.1 * r(C), x=r(B, T, C), dx=r(B, T, C), dh=r(B, T, C))
    return w


def inputs(x, w):
    """Projections and activations before the rule (torch)."""
    unit = lambda t: torch.nn.functional.normalize(t.unflatten(-1, (H, D)), dim=-1)
    q, k = unit(x @ w["q"]), unit(x @ w["k"])
    v, z = (x @ w["v"]).unflatten(-1, (H, D)), x @ w["z"]
    return q, k, v, -torch.nn.functional.softplus(x @ w["ga"] - 3), torch.sigmoid(x @ w["gb"]), z


def exact(w):
    w = {n: t.double().requires_grad_(n not in ("dx", "dh")) for n, t in w.items()}
    q, k, v, g, beta, z = inputs(w["x"], w)
    o, S = gdr_tokens(q, k, v, g, beta, torch.zeros(B, H, D, D, dtype=torch.float64), D ** -0.5)
    y = o / torch.sqrt(o.square().mean(-1, keepdim=True) + 1e-6)
    y = y.flatten(2) * w["heads"] * z * torch.sigmoid(z)
    y = y @ w["o"].T
    y = y / torch.sqrt(y.square().mean(-1, keepdim=True) + 1e-6) * w["post"]
    X = w["x"] + w["scale"] * y
    h = X / torch.sqrt(X.square().mean(-1, keepdim=True) + 1e-6) * w["next"]
    names = [n for n in w if n not in ("dx", "dh")]
    grads = torch.autograd.grad((X * w["dx"]).sum() + (h * w["dh"]).sum(), [w[n] for n in names])
    return X.detach(), h.detach(), S.detach(), dict(zip(names, grads))


def test_layer_forward_backward():
    w0 = weights()
    X0, h0, S0, g0 = exact(w0)
    w = {n: t.cuda().requires_grad_(n not in ("dx", "dh")) for n, t in w0.items()}
    pre = inputs(w["x"], w)
    q, k, v, g, beta, z = (t.detach().contiguous() for t in pre)
    o, S, S_c = carve.gdr_chunk_fwd(q, k, v, g, beta)
    d = {n: t.detach() for n, t in w.items()}
    kw = {"groups": H, "gate": z}
    y1, _ = carve.block_norm_fwd(o.flatten(2), d["heads"], **kw)
    y2 = y1 @ d["o"].T
    kw2 = {"residual": d["x"], "scale": d["scale"], "next_weight": d["next"]}
    X, h = carve.block_norm_fwd(y2, d["post"], **kw2)
    assert rel(X, X0) <= TOL and rel(h, h0) <= TOL and rel(S, S0) <= TOL

    r2 = carve.block_norm_bwd(y2, d["post"], d["dx"], d["dh"], **kw2)
    r1 = carve.block_norm_bwd(o.flatten(2), d["heads"], r2["dy"] @ d["o"], **kw)
    gr = carve.gdr_chunk_bwd(q, k, v, g, beta, S_c, r1["dy"].unflatten(2, (H, D)), want_dS0=False)
    dz = r1["dgate"]
    names = ("x", "q", "k", "v", "z", "ga", "gb")
    grads = dict(zip(names, torch.autograd.grad(pre, [w[n] for n in names], [gr["dq"], gr["dk"], gr["dv"], gr["dg"], gr["dbeta"], dz])))
    grads["x"] = grads["x"] + r2["dresidual"]
    grads.update(post=r2["dweight"], scale=r2["dscale"], next=r2["dnext_weight"], heads=r1["dweight"],
                 o=r2["dy"].flatten(0, 1).T @ y1.flatten(0, 1))
    errs = {n: rel(grads[n], g0[n]) for n in g0}
    print({n: float("%.2g" % e) for n, e in errs.items()}, flush=True)
    assert set(grads) == set(g0)
    assert max(errs.values()) <= TOL, errs


def test_layer_decodes_on_from_a_prompt():
    """130 tokens at once, then 20 one by one through the same layer."""
    w0 = weights()
    X0, h0, _, _ = exact(w0)
    d = {n: t.cuda() for n, t in w0.items()}
    pool = torch.zeros(5, H, D, D, device="cuda")
    slots = torch.tensor([3, 1], dtype=torch.int32, device="cuda")

    def block(x, rule):
        q, k, v, g, beta, z = (t.contiguous() for t in inputs(x, d))
        y, _ = carve.block_norm_fwd(rule(q, k, v, g, beta).flatten(2), d["heads"], groups=H, gate=z)
        return carve.block_norm_fwd(y @ d["o"].T, d["post"], residual=x.contiguous(), scale=d["scale"], next_weight=d["next"])

    def prompt(*a):
        o, S, _ = carve.gdr_chunk_fwd(*a, want_chunks=False)
        pool[slots.long()] = S
        return o

    parts = [block(d["x"][:, :130], prompt)]
    for t in range(130, T):
        parts.append(block(d["x"][:, t:t + 1], lambda *a: carve.gdr_step(*a, pool, slots)))
    assert rel(torch.cat([p[0] for p in parts], 1), X0) <= TOL
    assert rel(torch.cat([p[1] for p in parts], 1), h0) <= TOL
