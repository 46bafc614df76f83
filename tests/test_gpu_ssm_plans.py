"""The ways of working that large calls of the scan and the convolution choose, at sizes that the
definition in 64 bits can follow: spans of more than two chunks, several heads a workgroup of
the gradients, and the convolution's runs of 16 rows.  What was chosen is asserted.

References run on the card in 64 bits, by elementwise operations and sums alone."""
import ctypes

import pytest
import torch

from gdr_util import cuda, rel
from paper_2606_27229_amd import carve
from ssm_util import TOL, conv_inputs, ssm_inputs
from test_gpu_ssm_use import recorded

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32


def up(n):
    return (n + 255) // 256 * 256


def check_plan(x, N, span, splits):
    """The workspaces have room for exactly these spans and shares of a group's heads."""
    B, T, H, P = x["x"].shape
    G, S = x["Bm"].shape[2:]
    code = carve.CARVE_BF16 if x["x"].dtype == BF else carve.CARVE_F32
    d = carve.SsmDims(B, T, N, G, H, P, S, code, 1, *(s for n in ("x", "Bm", "Cm") for s in x[n].stride()[:3]), *x["dt"].stride()[:2])
    lib, r = carve.load_library(), ctypes.byref(d)
    L, state = 64 * span, H * P * S * 4
    chunks = T // 64 + N if N else B * -(-T // 64)
    spans = T // L + N if N else B * -(-T // L)
    token, tiles = 64 * 4, 10 * 1024   # a scalar of every token; C B^T of a chunk
    z = up(spans * state) + up(spans * H * 4) if T > L else 0
    assert lib.carve_ssm_chunk_count(r) == chunks
    assert lib.carve_ssm_workspace_size(r, 0) == up(chunks * H * 8 * token) + up(chunks * G * tiles) + z
    shares = up(splits * 2 * B * T * G * S * 4) if splits > 1 else 0
    assert lib.carve_ssm_workspace_size(r, 1) == (up(chunks * H * 12 * token) + up(chunks * G * 2 * tiles) + z + up(chunks * state)
                                                  + up(chunks * H * 16) + shares)


def scan_reference(x, lens=None):
    """Outputs and gradients; with them, of what is summed over tokens, the sum of the terms'
    magnitudes.  x: on the card; a dense batch's elements as further heads of one sequence."""
    d = {n: x[n].double() for n in ("x", "dt", "Bm", "Cm", "dy")}
    B, T, H, P = d["x"].shape
    G = d["Bm"].shape[2]
    fold = lambda t: t.transpose(0, 1).reshape(T, -1, *t.shape[3:])
    leaf = lambda t: t.clone().requires_grad_()
    xs, dt, Bm, Cm, dy = (fold(d[n]) for n in ("x", "dt", "Bm", "Cm", "dy"))
    xs, dt, Bm, Cm = (leaf(t) for t in (xs, dt, Bm, Cm))
    each = {n: leaf(x[n].double().repeat(B).expand(T, -1)) for n in ("A", "D", "dt_bias")}   # (of every token)
    S0 = leaf(x["S0"].double())
    rep, loss, y, last, at = H // G, 0.0, [], [], 0
    for n, rows in enumerate([T] if lens is None else lens):
        S = S0.flatten(0, 1) if lens is None else S0[n]
        for t in range(at, at + rows):
            step = torch.nn.functional.softplus(dt[t] + each["dt_bias"][t], threshold=1e9)
            S = (torch.exp(step * each["A"][t])[:, None, None] * S
                 + (step[:, None] * xs[t])[..., None] * Bm[t].repeat_interleave(rep, 0)[:, None])
            y.append((S * Cm[t].repeat_interleave(rep, 0)[:, None]).sum(-1) + each["D"][t, :, None] * xs[t])
            loss = loss + (y[-1] * dy[t]).sum()
        at += rows
        last.append(S)
        loss = loss + (S * (x["dS_T"].double().flatten(0, 1) if lens is None else x["dS_T"][n].double())).sum()
    leaves = {"x": xs, "dt": dt, "Bm": Bm, "Cm": Cm, **each, "S0": S0}
    g = dict(zip(leaves, torch.autograd.grad(loss, list(leaves.values()))))
    unfold = lambda t, like: t.reshape(T, B, *like.shape[2:]).transpose(0, 1)
    out = {"y": unfold(torch.stack(y).detach(), x["x"]), "S_T": torch.cat([s.detach() for s in last]).reshape(x["dS_T"].shape), "dS0": g["S0"]}
    out.update({"d" + n: unfold(g[n], x[n]) for n in ("x", "dt", "Bm", "Cm")})
    heads = {n: g[n].reshape(T, B, H) for n in each}
    out.update({"d" + n: t.sum((0, 1)) for n, t in heads.items()})
    return out, {"d" + n: t.abs().sum((0, 1)) for n, t in heads.items()}


def check_scan(x, launches, lens=None):
    off = None if lens is None else torch.tensor([0] + lens).cumsum(0).int().cuda()
    args, kw = [x[n] for n in ("x", "dt", "A", "Bm", "Cm")], {"D": x["D"], "dt_bias": x["dt_bias"], "offsets": off}
    got = {}

    def forward():
        got["y"], got["S_T"], got["S_chunks"] = carve.ssm_chunk_fwd(*args, x["S0"], **kw)

    def backward():
        got.update(carve.ssm_chunk_bwd(*args, got["S_chunks"], x["dy"], x["dS_T"], **kw))

    assert (recorded(forward) - 1, recorded(backward) - 1) == launches
    ref, terms = scan_reference(x, lens)
    bad = {}
    for n, r in ref.items():
        if n in terms:
            # sums over tokens, their terms each as exact as TOL says: measured by the terms
            e = float(torch.linalg.vector_norm(got[n].double() - r) / torch.linalg.vector_norm(terms[n]))
        else:
            e = rel(got[n], r.cpu())
        if not e <= TOL[got[n].dtype]:
            bad[n] = (e, TOL[got[n].dtype])
    assert not bad, bad


@pytest.mark.parametrize("dtype", [BF, F])
def test_spans_of_three_chunks(dtype):
    """32 sequences of 640 tokens: four spans of three chunks, the last one of one."""
    x = cuda(ssm_inputs(32, 640, 4, 4, 32, 32, dtype, 41))
    check_plan(x, 0, 3, 1)
    check_scan(x, (4, 6))


@pytest.mark.parametrize("dtype", [BF, F])
def test_packed_spans_of_three_chunks(dtype):
    """Sequences that end within a span and within a chunk, 32 heads of 256 rows."""
    lens = [700, 0, 1, 835]
    x = cuda(ssm_inputs(1, sum(lens), 1, 32, 256, 32, dtype, 42, seqs=len(lens)))
    assert x["x"].shape[1] == 1536
    check_plan(x, len(lens), 3, 8)
    check_scan(x, (4, 7), lens)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("N", [32, 128])
def test_four_heads_a_workgroup(N, dtype):
    """512 sequences of 9 tokens, four heads of two turns of 32 value columns each: one workgroup
    of the gradients has all four."""
    x = cuda(ssm_inputs(512, 9, 1, 4, 64, N, dtype, 43))
    check_plan(x, 0, 1, 1)
    check_scan(x, (2, 4))


@pytest.mark.parametrize("dtype", [BF, F])
def test_eight_heads_a_workgroup_of_packed_sequences(dtype):
    """498 packed sequences of up to three tokens, empty ones among them, and one of three
    chunks: eight heads of one turn each."""
    lens = [(2, 0, 1, 3)[i % 4] for i in range(497)]
    lens.insert(200, 150)
    x = cuda(ssm_inputs(1, sum(lens), 1, 8, 32, 32, dtype, 44, seqs=len(lens)))
    check_plan(x, len(lens), 2, 1)
    check_scan(x, (4, 6), lens)


def conv_reference(x, lens=None):
    """x: on the card."""
    d = {n: x[n].double().requires_grad_() for n in ("x", "weight", "bias", "x0")}
    B, T, C = x["x"].shape
    W = d["weight"].shape[1]
    ys, last, loss, at = [], [], 0.0, 0
    for n, rows in enumerate([T] * B if lens is None else lens):
        b, first = (n, 0) if lens is None else (0, at)
        z = torch.cat([d["x0"][n], d["x"][b, first:first + rows]])
        p = d["bias"] + sum(z[j:j + rows] * d["weight"][:, j] for j in range(W))
        o = p * torch.sigmoid(p)
        loss = loss + (o * x["dy"][b, first:first + rows].double()).sum() + (z[rows:] * x["dx_T"][n].double()).sum()
        ys.append(o.detach())
        last.append(z[rows:].detach())
        at += rows
    g = torch.autograd.grad(loss, list(d.values()))
    return {"y": torch.cat(ys).reshape(B, T, C), "x_T": torch.stack(last), **{"d" + n: t for n, t in zip(d, g)}}


@pytest.mark.parametrize("dtype,C", [(BF, 16384), (F, 8192)])
@pytest.mark.parametrize("W", [3, 4])
@pytest.mark.parametrize("B,T,lens", [(1, 600, None), (3, 257, None), (1, 612, [5, 0, 300, 1, 16, 16, 2, 272])])
def test_runs_of_sixteen_rows(B, T, lens, W, dtype, C):
    # 16 threads of 16 bytes side by side, 16 runs of 16 rows a workgroup: 256 of them and more
    # than that take such runs (fewer take runs of 4)
    wide = 16 * 16 // (2 if dtype == BF else 4)
    assert -(-T // 256) * B * (C // wide) >= 256
    x = cuda(conv_inputs(B, T, C, W, dtype, T + W, seqs=B if lens is None else len(lens)))
    off = None if lens is None else torch.tensor([0] + lens).cumsum(0).int().cuda()
    kw = {"bias": x["bias"], "activation": x["act"], "offsets": off}
    y, x_T = carve.short_conv_fwd(x["x"], x["weight"], x["x0"], **kw)
    got = {"y": y, "x_T": x_T, **carve.short_conv_bwd(x["x"], x["weight"], x["dy"], x["x0"], x["dx_T"], **kw)}
    ref = conv_reference(x, lens)
    assert torch.equal(got["x_T"].double(), ref.pop("x_T"))
    for n, r in ref.items():
        assert rel(got[n], r.cpu()) <= TOL[got[n].dtype], (n, rel(got[n], r.cpu()))
