"""The short causal convolution on the GPU against its definition in 64 bits."""
import pytest
import torch

from gdr_util import cuda, rel
from paper_2606_27229_amd import carve
from ssm_util import TOL, conv_inputs, conv_reference

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32


def run(x, offsets=None, out=None, grads=None):
    d = cuda(x)
    kw = {"bias": d["bias"], "activation": x["act"], "offsets": offsets}
    y, x_T = carve.short_conv_fwd(d["x"], d["weight"], d["x0"], out=out, **kw)
    return {"y": y, "x_T": x_T, **carve.short_conv_bwd(d["x"], d["weight"], d["dy"], d["x0"], d["dx_T"], out=grads, want_dx0=True, **kw)}


def check(got, ref, rows=None, T=None):
    for n, r in ref.items():
        t = got[n]
        if n == "x_T":
            assert torch.equal(t.double().cpu(), r)
            continue
        if rows is not None and n in ("y", "dx"):
            t, r = t[:, rows], r[:, rows]
        # (a weight's sum runs over every row: its terms' magnitude goes with their root)
        assert rel(t, r) <= TOL[t.dtype], (n, rel(t, r))


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("B,T,C,W,opt", [
    (1, 1, 8, 2, {}), (2, 2, 32, 4, {}), (1, 3, 40, 4, dict(state=False)), (3, 17, 24, 3, dict(bias=False)),
    (1, 64, 136, 4, dict(act=None)), (2, 300, 264, 4, {}), (1, 1000, 16, 3, dict(act=None, bias=False)), (1, 515, 2304, 2, {})])
def test_conv(B, T, C, W, opt, dtype):
    x = conv_inputs(B, T, C, W, dtype, 7 * T + C, **opt)
    ref = conv_reference(x)
    got = run(x)
    if x["x0"] is None:
        assert got.pop("dx0").shape == (B, W - 1, C)
    check(got, ref)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("W", [2, 3, 4])
@pytest.mark.parametrize("lens,first,T", [([5, 0, 70, 1, 1, 64], 0, 150), ([2, 300, 1], 3, 320), ([0, 0], 2, 10), ([1] * 40, 1, 45), ([17, 16, 15], 0, 48)])
def test_packed(lens, first, T, W, dtype):
    x = conv_inputs(1, T, 72, W, dtype, 5, seqs=len(lens))
    ends = torch.tensor([first] + lens).cumsum(0).int().cuda()
    mark = torch.full_like(x["x"], 7.0).cuda()
    got = run(x, ends, {"y": mark.clone()}, {"dx": mark.clone()})
    check(got, conv_reference(x, lens, first), slice(first, first + sum(lens)))
    for n in ("y", "dx"):   # rows of no sequence are left as they were
        assert (got[n][:, :first] == 7).all() and (got[n][:, first + sum(lens):] == 7).all()


def test_rows_of_no_sequence_are_not_read():
    """NaN before, behind and in no sequence reach nothing."""
    x = conv_inputs(1, 40, 16, 4, F, 5, seqs=2)
    ends = torch.tensor([4, 9, 30], dtype=torch.int32).cuda()
    ref = run(x, ends, {"y": torch.zeros_like(x["x"]).cuda()}, {"dx": torch.zeros_like(x["x"]).cuda()})
    for n in ("x", "dy"):
        x[n][:, :4] = x[n][:, 30:] = float("nan")
    got = run(x, ends, {"y": torch.zeros_like(x["x"]).cuda()}, {"dx": torch.zeros_like(x["x"]).cuda()})
    for n in ref:
        assert torch.equal(got[n], ref[n]), n


@pytest.mark.parametrize("dtype", [BF, F])
def test_strided_rows(dtype):
    x = conv_inputs(2, 50, 64, 4, dtype, 6)
    wide = torch.randn(2, 50, 128, device="cuda").to(dtype)
    wide[..., 32:96] = x["x"].cuda()
    got, ref = run(x | {"x": wide[..., 32:96]}), run(x)
    for n in ref:
        assert torch.equal(got[n], ref[n]), n


def test_gradients_against_differences():
    x = conv_inputs(1, 20, 8, 4, F, 3)
    got = run(x)
    gen = torch.Generator().manual_seed(2)
    for n in ("x", "weight", "bias", "x0"):
        v = torch.randn(x[n].shape, generator=gen, dtype=torch.float64)

        def loss(e):
            r = conv_reference(dict(x) | {n: x[n].double() + e * v})
            return float((r["y"] * x["dy"].double()).sum() + (r["x_T"] * x["dx_T"].double()).sum())

        g = got["d" + n].double().cpu()
        diff = (loss(1e-4) - loss(-1e-4)) / 2e-4
        assert abs(diff - float((g * v).sum())) <= 4 * TOL[F] * float(torch.linalg.vector_norm(g)) + 1e-6 * abs(diff) + 1e-6


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("W", [2, 3, 4])
@pytest.mark.parametrize("T", [1, 2, 6])
def test_step(dtype, W, T):
    B, pool, C = 4, 6, 520
    x = conv_inputs(B, T, C, W, dtype, 8)
    slots = torch.tensor([5, -1, 0, 2], dtype=torch.int32)
    kept = torch.randn(pool, W - 1, C, generator=torch.Generator().manual_seed(1)).to(dtype)
    d, state = cuda(x), kept.cuda()
    out = torch.full_like(d["x"], 7.0)
    y = carve.short_conv_step(d["x"], d["weight"], state, slots.cuda(), bias=d["bias"], out=out)
    assert y is out and (y[1] == 7).all()
    x["x0"] = kept[slots.clamp(min=0).long()]
    ref = conv_reference(x)
    keep = [0, 2, 3]
    assert rel(y[keep], ref["y"][keep]) <= TOL[dtype]
    for b in keep:
        assert torch.equal(state[slots[b]].double().cpu(), ref["x_T"][b])
    for s in (1, 3, 4):
        assert torch.equal(state[s].cpu(), kept[s])
