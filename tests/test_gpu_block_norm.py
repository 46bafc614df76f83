"""The norms around a block with its gate and residual scale, against their definition in
64 bits.

Tolerances (relative 2-norms): f32 arithmetic; sums of N <= 8192 squares or products in
partial sums of at most 32 terms a thread, 6 steps of a wave and 4 waves: 42 * 2^-24 =
2.5e-6 of a sum, and a dozen roundings of 2^-24 on the way: 4e-6 for f32 results.  The
parameters' gradients add up to 17 rows a workgroup at these sizes and the workgroups' sums
in 16 chains of at most 64: 1e-5.  bf16 results: their rounding, 2^-8, on top.
"""
import pytest
import torch

from paper_2606_27229_amd import carve
from tests.gdr_util import cuda, norm_inputs, norm_reference, rel

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


def kw_of(x):
    return {n: x[n] for n in ("groups", "gate", "gate_act", "residual", "alpha", "scale", "next_weight", "eps")}


def run(x, **more):
    X, h = carve.block_norm_fwd(x["y"], x["weight"], **kw_of(x), **more)
    got = {"x": X}
    if h is not None:
        got["h"] = h
    got.update(carve.block_norm_bwd(x["y"], x["weight"], x["dx"], x["dh"], **kw_of(x), **more))
    return got


def compare(got, ref, dtype):
    errs = {n: rel(got[n], ref[n]) for n in ref}
    print("rel errors:", {n: float("%.2g" % e) for n, e in errs.items()}, flush=True)
    assert set(got) == set(ref)
    for n, e in errs.items():
        assert torch.isfinite(got[n].float()).all(), n
        params = n in ("dweight", "dscale", "dnext_weight")
        assert e <= (1e-5 if params else 4e-6 + (2.0 ** -8 if dtype == BF else 0)), (n, e)


@pytest.mark.parametrize("rows,N,dtype", [
    (1, 4, F32), (3, 252, F32), (5, 256, F32), (70, 260, F32), (9, 512, F32), (7, 516, F32), (33, 1024, F32), (3, 1028, F32),
    (5, 2048, F32), (3, 4096, F32), (2, 8192, F32),
    (1, 8, BF), (5, 504, BF), (66, 512, BF), (7, 520, BF), (9, 1024, BF), (5, 1032, BF), (1030, 2048, BF), (3, 2056, BF),
    (4, 4096, BF), (3, 4104, BF), (2, 8192, BF),
])
def test_rows_of_every_size(rows, N, dtype):
    print(f"case block norm {rows}x{N} {dtype}", flush=True)
    x = norm_inputs(rows, N, dtype, seed=rows + N, gate="sigmoid")
    compare(run(cuda(x)), norm_reference(x), dtype)


@pytest.mark.parametrize("rows,N", [((1 << 26) + 1024, 8), ((1 << 22) + 1024, 1032)])
def test_more_rows_than_one_grid_dimension(rows, N):
    """The rows repeat after 1024, so every part of the result equals the first."""
    print(f"case block norm {rows}x{N}", flush=True)
    x = cuda(norm_inputs(1024, N, BF, seed=N, gate="", residual=False, scale=False, next=False))
    first, _ = carve.block_norm_fwd(x["y"], x["weight"], eps=x["eps"])
    many, _ = carve.block_norm_fwd(x["y"].repeat(rows // 1024, 1), x["weight"], eps=x["eps"])
    for part in many.view(-1, 1024, N).split(1024):
        assert torch.equal(part, first.expand_as(part))


def test_numbers_given_as_tensors_are_read_at_every_call():
    x = cuda(norm_inputs(4, 64, F32, seed=5, gate="", residual=True, scale=False, next=False))
    alpha = torch.tensor(1.0)
    for value in (1.0, 0.5):
        alpha.fill_(value)
        got, _ = carve.block_norm_fwd(x["y"], x["weight"], residual=x["residual"], alpha=alpha)
        want, _ = carve.block_norm_fwd(x["y"], x["weight"], residual=x["residual"], alpha=value)
        assert torch.equal(got, want)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("gate", ["", "silu", "sigmoid"])
@pytest.mark.parametrize("residual,scale,next", [(False, False, False), (True, False, False), (False, True, True), (True, True, True)])
def test_every_combination(dtype, gate, residual, scale, next):
    print(f"case block norm {dtype} gate={gate} residual={residual} scale={scale} next={next}", flush=True)
    x = norm_inputs(19, 640, dtype, seed=7, gate=gate, residual=residual, scale=scale, next=next)
    compare(run(cuda(x)), norm_reference(x), dtype)


@pytest.mark.parametrize("N,groups,dtype", [(64, 16, F32), (512, 4, F32), (1024, 4, F32), (4096, 32, F32), (8192, 64, F32),
                                            (64, 8, BF), (128, 2, BF), (2048, 16, BF), (2048, 4, BF), (6144, 96, BF),
                                            (8192, 16, BF), (192, 3, BF)])
def test_groups(N, groups, dtype):
    """Norms over the heads of a row."""
    print(f"case block norm groups {N}/{groups} {dtype}", flush=True)
    x = norm_inputs(13, N, dtype, seed=N + groups, groups=groups, residual=N == 2048)
    compare(run(cuda(x)), norm_reference(x), dtype)


def test_without_the_streams_own_gradient():
    x = norm_inputs(21, 1024, BF, seed=3, dx=False)
    compare(run(cuda(x)), norm_reference(x), BF)


@pytest.mark.parametrize("dtype", [F32, BF])
def test_strided_rows(dtype):
    """y, gate and residual as slices of wider rows, three dimensions, one row's stride 0."""
    x = norm_inputs(24, 256, dtype, seed=5)
    x["residual"] = x["residual"][:1].expand(24, 256).clone()
    ref = norm_reference(x)
    d = cuda(x)
    wide = torch.cat([d["y"], d["gate"]], -1)
    d["y"], d["gate"] = wide[:, :256], wide[:, 256:]
    d["residual"] = d["residual"][:1].expand(24, 256)
    compare(run(d), ref, dtype)
    d3 = dict(d, y=wide.view(4, 6, 512)[..., :256], gate=wide.view(4, 6, 512)[..., 256:], residual=d["residual"].view(4, 6, 256),
              dx=d["dx"].view(4, 6, 256), dh=d["dh"].view(4, 6, 256))
    got = run(d3)
    assert got["x"].shape == (4, 6, 256)
    compare({n: t.reshape(-1, 256) if t.dim() == 3 else t for n, t in got.items()}, ref, dtype)


def test_zero_rows_and_large_values():
    """Rows of zeros with eps, gates far out, and values near the ends of the range."""
    x = norm_inputs(12, 512, F32, seed=9, alpha=1.0)
    x["y"][2] = 0
    x["y"][3] *= 1e15
    x["y"][4] *= 1e-12
    x["gate"][5] = 200.0
    x["gate"][6] = -200.0
    compare(run(cuda(x)), norm_reference(x), F32)


@pytest.mark.parametrize("N", [512, 2048])
def test_reruns_and_preallocated_outputs(N):
    x = cuda(norm_inputs(3000, N, BF, seed=15))
    first = run(x)
    out = {n: torch.full_like(t, float("nan")) for n, t in first.items()}
    X, h = carve.block_norm_fwd(x["y"], x["weight"], **kw_of(x), out={n: out[n] for n in ("x", "h")})
    ws = torch.full((1 << 25,), 255, dtype=torch.uint8, device="cuda")
    again = carve.block_norm_bwd(x["y"], x["weight"], x["dx"], x["dh"], **kw_of(x), workspace=ws,
                                 out={n: t for n, t in out.items() if n not in ("x", "h")})
    again.update(x=X, h=h)
    for n in first:
        assert again[n].data_ptr() == out[n].data_ptr() and torch.equal(first[n], again[n]), n


@pytest.mark.parametrize("name", ["y", "weight", "gate", "residual", "scale", "next_weight"])
def test_gradients_against_differences(name):
    """<gradient, d> against central differences of the f32 forward along d (the bounds of
    the same test of the gated delta rule)."""
    x = cuda(norm_inputs(11, 256, F32, seed=17))
    got = run(x)
    gen = torch.Generator(device="cuda").manual_seed(18)
    slopes = []
    for _ in range(4):
        d = torch.randn(x[name].shape, generator=gen, device="cuda")
        d = d / d.norm() * max(1.0, float(x[name].norm()) / 16)
        if name == "y":   # rows differ in size: each by its own
            d = d * x["y"].norm(dim=1, keepdim=True) / x["y"].norm() * 3
        loss = []
        for sign in (1, -1):
            z = dict(x)
            z[name] = x[name] + sign * 2.0 ** -7 * d
            X, h = carve.block_norm_fwd(z["y"], z["weight"], **kw_of(z))
            loss.append((X.double() * x["dx"]).sum() + (h.double() * x["dh"]).sum())
        slopes.append((float((loss[0] - loss[1]) / 2.0 ** -6), float((got["d" + name].double() * d).sum())))
    print(name, slopes, flush=True)
    most = max(abs(b) for _, b in slopes)
    for a, b in slopes:
        assert abs(a - b) <= 5e-3 * most, (name, slopes)


def test_streams_and_graph():
    x = cuda(norm_inputs(100, 2048, BF, seed=19))
    ref = run(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = run(x, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    for n in ref:
        assert torch.equal(got[n], ref[n]), n
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        res = run(x)
    for turn in range(4):
        src = cuda(norm_inputs(100, 2048, BF, seed=20 + turn))
        for n in ("y", "gate", "residual", "dx", "dh"):
            x[n].copy_(src[n])
        graph.replay()
        torch.cuda.synchronize()
        got = {n: t.clone() for n, t in res.items()}
        want = run(x)
        for n in want:
            assert torch.equal(got[n], want[n]), (turn, n)


def test_agrees_with_rmsnorm():
    """With nothing but the weight it is the output norm."""
    x = cuda(norm_inputs(37, 1024, F32, seed=23, gate="", residual=False, scale=False, next=False))
    X, _ = carve.block_norm_fwd(x["y"], x["weight"])
    want = carve.rmsnorm_fwd(x["y"].view(1, 37, 8, 128), x["weight"]).view(37, 1024)
    assert rel(X, want.cpu()) <= 4e-6
