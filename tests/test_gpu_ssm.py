"""The selective state space scan on the GPU against its definition in 64 bits."""
import pytest
import torch

from gdr_util import cuda, rel
from paper_2606_27229_amd import carve
from ssm_util import SSM_LEAVES, TOL, ssm_decay_terms, ssm_inputs, ssm_reference

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32


def run(x, offsets=None, **kw):
    """Outputs and gradients of the chunk calls on a dict of ssm_inputs."""
    d = cuda(x)
    args = [d[n] for n in ("x", "dt", "A", "Bm", "Cm")]
    opt = {"D": d["D"], "dt_bias": d["dt_bias"], "softplus": x["softplus"], "offsets": offsets}
    y, S_T, S_chunks = carve.ssm_chunk_fwd(*args, d["S0"], **opt, **kw)
    out = {"y": y, "S_T": S_T}
    out.update(carve.ssm_chunk_bwd(*args, S_chunks, d["dy"], d["dS_T"], **opt, **kw))
    return out


def check(got, ref, x, rows=None):
    bad = {}
    for n, r in ref.items():
        if n not in got:
            assert n == "dS0" or x[n[1:]] is None, n
            continue
        t = got[n]
        if rows is not None and t.shape[:2] == x["x"].shape[:2]:
            t, r = t[:, rows], r[:, rows]
        e = rel(t, r)
        if not e <= TOL[t.dtype]:
            bad[n] = (e, TOL[t.dtype])
    assert not bad, bad


CASES = [  # B, T, G, H, P, N, dtype, options
    (1, 1, 1, 1, 32, 32, BF, {}),
    (2, 63, 1, 2, 64, 64, BF, {}),
    (1, 64, 2, 2, 32, 128, BF, dict(state=False)),
    (1, 65, 1, 4, 64, 128, BF, dict(skip=False)),
    (2, 130, 2, 4, 96, 32, BF, dict(bias=False)),
    (1, 300, 1, 3, 64, 64, BF, dict(dst=False)),
    (1, 700, 1, 2, 32, 32, BF, {}),
    (3, 97, 1, 2, 128, 128, BF, dict(softplus=False)),
    (1, 1, 1, 2, 64, 64, F, {}),
    (2, 65, 1, 2, 32, 32, F, {}),
    (1, 130, 2, 4, 64, 128, F, dict(state=False, skip=False)),
    (1, 333, 1, 3, 96, 64, F, dict(bias=False)),
    (1, 600, 1, 1, 32, 128, F, {}),
    (1, 80, 1, 2, 256, 32, F, dict(softplus=False)),
]


@pytest.mark.parametrize("B,T,G,H,P,N,dtype,opt", CASES)
def test_chunks(B, T, G, H, P, N, dtype, opt):
    x = ssm_inputs(B, T, G, H, P, N, dtype, 17 * T + H, **opt)
    check(run(x), ssm_reference(x), x)


@pytest.mark.parametrize("dtype,N,P", [(BF, 128, 64), (F, 64, 32)])
@pytest.mark.parametrize("lens,first,T", [([5, 0, 70, 1, 64], 0, 140), ([200, 300, 1], 3, 520), ([0, 0], 0, 10), ([1] * 40, 1, 45)])
def test_packed(lens, first, T, dtype, N, P):
    x = ssm_inputs(1, T, 1, 2, P, N, dtype, 5, seqs=len(lens))
    ends = torch.tensor([first] + lens).cumsum(0).int().cuda()
    out = {"y": torch.full_like(x["x"], 7.0).cuda()}
    d = cuda(x)
    args, opt = [d[n] for n in ("x", "dt", "A", "Bm", "Cm")], {"D": d["D"], "dt_bias": d["dt_bias"], "offsets": ends}
    y, S_T, S_chunks = carve.ssm_chunk_fwd(*args, d["S0"], out=out, **opt)
    mark = {n: torch.full_like(d[n[1:]], 7.0) for n in ("dx", "ddt", "dBm", "dCm")}
    g = carve.ssm_chunk_bwd(*args, S_chunks, d["dy"], d["dS_T"], out=dict(mark), **opt)
    ref = ssm_reference(x, lens, first)
    rows = slice(first, first + sum(lens))
    check({"y": y, "S_T": S_T, **g}, ref, x, rows)
    for t in (y, *(g[n] for n in mark)):   # rows of no sequence are left as they were
        assert (t[:, :first] == 7).all() and (t[:, first + sum(lens):] == 7).all()


@pytest.mark.parametrize("dtype", [BF, F])
def test_hard_decays_and_resets(dtype):
    """Decays of e^-30 a token and more, steps of 0 (dt = -inf) and a small ddt beside
    large ones: what decays hide does not leave its rounding."""
    x = ssm_inputs(1, 150, 1, 2, 32, 32, dtype, 3, decay=20.0)
    x["dt"][0, 20:24] = 3.0
    x["dt"][0, 70] = 30.0
    x["dt"][0, 90:95] = float("-inf")
    ref, got = ssm_reference(x), run(x)
    # dA is a sum of terms 160 times as large as itself here (9.3 and 161 of the two heads),
    # each of which is as exact as TOL says: its error is measured by theirs
    terms = ssm_decay_terms(x)
    assert float(torch.linalg.vector_norm(got["dA"].cpu().double() - ref.pop("dA"))) <= TOL[F] * float(torch.linalg.vector_norm(terms))
    check(got, ref, x)
    assert (got["ddt"][0, 90:95] == 0).all()
    for t in (20, 22, 70, 71):   # each token by itself
        assert rel(got["ddt"][0, t], ref["ddt"][0, t]) <= 4 * TOL[dtype], t


def test_no_decay():
    """A = 0: sums of everything before."""
    x = ssm_inputs(1, 400, 1, 2, 32, 64, F, 9)
    x["A"] = torch.zeros(2)
    check(run(x), ssm_reference(x), x)


@pytest.mark.parametrize("dtype", [BF, F])
def test_gradients_against_differences(dtype):
    """The loss's change along a direction, of the definition in 64 bits."""
    x = ssm_inputs(1, 70, 1, 2, 32, 32, dtype, 21)
    got = run(x)
    gen = torch.Generator().manual_seed(2)
    for n in SSM_LEAVES:
        v = torch.randn(x[n].shape, generator=gen, dtype=torch.float64)

        def loss(e):
            z = dict(x) | {n: x[n].double() + e * v}
            r = ssm_reference(z, grads=False)
            return (r["y"] * x["dy"].double()).sum() + (r["S_T"] * x["dS_T"].double()).sum()

        diff = float((loss(1e-4) - loss(-1e-4)) / 2e-4)
        g = got["d" + n].double().cpu()
        # the gradient's own error, along a random direction, and the differences'
        tol = 4 * TOL[got["d" + n].dtype] * float(torch.linalg.vector_norm(g)) + 1e-6 * abs(diff) + 1e-6
        assert abs(diff - float((g * v).sum())) <= tol, n


@pytest.mark.parametrize("dtype", [BF, F])
def test_slices_of_a_projection(dtype):
    """x, B, C and dt as slices of wider rows, at odd offsets of dt."""
    B, T, G, H, P, N = 2, 90, 2, 4, 32, 32
    x = ssm_inputs(B, T, G, H, P, N, dtype, 4)
    d = cuda(x)
    wide = torch.randn(B, T, 8 + H * P + 2 * G * N + 3 + H + 5, device="cuda").to(dtype)
    at, parts = 8, {}
    for n in ("x", "Bm", "Cm", "dt"):
        size = d[n][0, 0].numel()
        at += 3 if n == "dt" else 0
        view = wide[..., at:at + size]
        view = view if n == "dt" else view.unflatten(-1, d[n].shape[2:])
        view.copy_(d[n])
        parts[n] = view
        at += size
    if wide.stride(1) * wide.element_size() % 16:
        pad = 16 // wide.element_size()
        rows = torch.zeros(B, T, -(-wide.shape[2] // pad) * pad, device="cuda", dtype=dtype)
        rows[..., :wide.shape[2]] = wide
        wide, at = rows, 8
        for n in ("x", "Bm", "Cm", "dt"):
            size = d[n][0, 0].numel()
            at += 3 if n == "dt" else 0
            view = wide[..., at:at + size]
            parts[n] = view if n == "dt" else view.unflatten(-1, d[n].shape[2:])
            at += size
    got = run(x | parts)
    ref = run(x)
    for n in ref:
        assert torch.equal(got[n], ref[n]), n


def test_shared_inputs():
    """B expanded over groups, x over heads (stride 0): gradients are written per element."""
    x = ssm_inputs(1, 40, 2, 4, 32, 32, F, 8)
    x["Bm"] = x["Bm"][:, :, :1].expand(-1, -1, 2, -1)
    x["x"] = x["x"][:, :, :1].expand(-1, -1, 4, -1)
    d = cuda({n: (t.contiguous() if isinstance(t, torch.Tensor) else t) for n, t in x.items()})
    d["Bm"], d["x"] = d["Bm"][:, :, :1].expand(-1, -1, 2, -1), d["x"][:, :, :1].expand(-1, -1, 4, -1)
    args, opt = [d[n] for n in ("x", "dt", "A", "Bm", "Cm")], {"D": d["D"], "dt_bias": d["dt_bias"]}
    y, S_T, S_chunks = carve.ssm_chunk_fwd(*args, d["S0"], **opt)
    g = carve.ssm_chunk_bwd(*args, S_chunks, d["dy"], d["dS_T"], **opt)
    check({"y": y, "S_T": S_T, **g}, ssm_reference({n: (t.contiguous() if isinstance(t, torch.Tensor) else t) for n, t in x.items()}), x)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("T", [1, 3])
@pytest.mark.parametrize("G,H,P,N", [(1, 2, 32, 32), (2, 4, 64, 128), (1, 3, 96, 64)])
def test_step(dtype, T, G, H, P, N):
    B, pool = 5, 8
    x = ssm_inputs(B, T, G, H, P, N, dtype, 31, dst=False)
    slots = torch.tensor([6, -1, 0, 7, 3], dtype=torch.int32)
    states = torch.randn(pool, H, P, N, generator=torch.Generator().manual_seed(1))
    d = cuda(x)
    state, out = states.cuda(), torch.full_like(d["x"], 7.0)
    y = carve.ssm_step(*(d[n] for n in ("x", "dt", "A", "Bm", "Cm")), state, slots.cuda(), D=d["D"], dt_bias=d["dt_bias"], out=out)
    assert y is out and (y[1] == 7).all()
    keep = [0, 2, 3, 4]
    x["S0"] = states[slots.clamp(min=0).long()]
    ref = ssm_reference(x, grads=False)
    assert rel(y[keep], ref["y"][keep]) <= TOL[dtype]
    for b in keep:
        assert rel(state[slots[b]], ref["S_T"][b]) <= TOL[F]
    for s in (1, 2, 4, 5):
        assert torch.equal(state[s].cpu(), states[s])


@pytest.mark.parametrize("dtype", [BF, F])
def test_steps_continue_a_prompt(dtype):
    """A prompt by chunks, then tokens one by one, as the whole by the definition."""
    x = ssm_inputs(2, 75, 1, 2, 64, 64, dtype, 12)
    d = cuda(x)
    cut = lambda a, b: [d[n][:, a:b] if n not in ("A",) else d[n] for n in ("x", "dt", "A", "Bm", "Cm")]
    opt = {"D": d["D"], "dt_bias": d["dt_bias"]}
    y, S, _ = carve.ssm_chunk_fwd(*cut(0, 70), d["S0"], want_chunks=False, **opt)
    parts = [y] + [carve.ssm_step(*cut(t, t + 1), S, **opt) for t in range(70, 75)]
    ref = ssm_reference(x, grads=False)
    assert rel(torch.cat(parts, 1), ref["y"]) <= TOL[dtype]
    assert rel(S, ref["S_T"]) <= 2 * TOL[F]


def test_reruns_are_equal():
    x = ssm_inputs(1, 500, 1, 8, 64, 128, BF, 2)
    one, two = run(x), run(x)
    for n in one:
        assert torch.equal(one[n], two[n]), n
