"""The block norm over the range of its types, row by row: a row of 1e36 and one of 1e-30
are as exact as any other, and a small row is not hidden behind a large one.

Tolerances: those of the rows' results in the same form's other tests, f32 arithmetic over
N <= 4096 values a row (4e-6, and 2^-8 for results in bf16), here relative to each row's own
2-norm; the parameters' gradients as there (1e-5).  Factors of a power of two round nothing.
"""
import pytest
import torch

from paper_2606_27229_amd import carve
from tests.gdr_util import cuda, norm_inputs, norm_reference, rel

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
PARAMS = ("dweight", "dscale", "dnext_weight")


def run(x):
    kw = {n: x[n] for n in ("groups", "gate", "gate_act", "residual", "alpha", "scale", "next_weight", "eps")}
    X, h = carve.block_norm_fwd(x["y"], x["weight"], **kw)
    got = {"x": X, **({} if h is None else {"h": h})}
    got.update(carve.block_norm_bwd(x["y"], x["weight"], x["dx"], x["dh"], **kw))
    return got


def compare(x, dtype):
    ref, got = norm_reference(x), run(cuda(x))
    assert set(got) == set(ref)
    for n, want in ref.items():
        have = got[n].cpu()
        assert torch.isfinite(have.float()).all(), n
        if n in PARAMS:
            assert rel(have, want) <= 1e-5, (n, rel(have, want))
            continue
        for r in range(want.shape[0]):
            if float(want[r].abs().max()) < 2.0 ** -149:   # (below the types' smallest value)
                assert not have[r].any(), (n, r)
            else:
                e = rel(have[r], want[r])
                assert e <= 4e-6 + (2.0 ** -8 if dtype == BF else 0), (n, r, e)


@pytest.mark.parametrize("N,groups,dtype", [(512, 1, F32), (2048, 1, F32), (4096, 1, F32), (512, 8, F32), (2048, 32, F32),
                                            (512, 1, BF), (1024, 8, BF), (4096, 1, BF), (2048, 16, BF)])
def test_rows_of_every_magnitude(N, groups, dtype):
    """Rows of y from the smallest to the largest, zeros and gates far out among them; the
    streams they are added to are of the usual size."""
    print(f"case block norm range {N}/{groups} {dtype}", flush=True)
    sizes = [1.0, 0.0, 1e-30, 1e-12, 1e-3, 1e6, 1e15, 1e18, 3e18, 1e19, 1e25, 1e36, 1.0, 1.0, 1.0]
    x = norm_inputs(len(sizes), N, dtype, seed=N + groups, groups=groups, gate="silu")
    gen = torch.Generator().manual_seed(N)
    x["y"] = (torch.tensor(sizes)[:, None] * torch.randn(len(sizes), N, generator=gen)).to(dtype)
    x["gate"][-2], x["gate"][-1] = 200.0, -200.0
    compare(x, dtype)


@pytest.mark.parametrize("N,dtype", [(512, F32), (2048, F32), (1024, BF), (4096, BF)])
def test_streams_of_every_magnitude(N, dtype):
    """Rows of the residual stream, and so of x, as large; the rows' gradients reach both
    norms, or the next one alone."""
    for dx in (True, False):
        sizes = [1.0, 0.0, 1e15, 1e18, 1e19, 1e25]
        x = norm_inputs(len(sizes), N, dtype, seed=N, gate="sigmoid", dx=dx)
        gen = torch.Generator().manual_seed(N)
        x["residual"] = (torch.tensor(sizes)[:, None] * torch.randn(len(sizes), N, generator=gen)).to(dtype)
        compare(x, dtype)


@pytest.mark.parametrize("N,groups,dtype", [(512, 1, F32), (2048, 1, F32), (1024, 16, BF), (2048, 1, BF), (512, 4, F32)])
def test_small_rows_without_eps(N, groups, dtype):
    """With eps = 0 every row that is not zero has the norm of its own size."""
    sizes = [1.0, 1e-10, 1e-19, 1e-23, 1e-30]
    x = norm_inputs(len(sizes), N, dtype, seed=N, groups=groups, residual=False, eps=0.0)
    gen = torch.Generator().manual_seed(N)
    x["y"] = (torch.tensor(sizes)[:, None] * torch.randn(len(sizes), N, generator=gen)).to(dtype)
    x["scale"] *= 1e-20   # (and so has x)
    x["dx"] = (1e18 * x["dx"].float()).to(dtype)
    compare(x, dtype)


@pytest.mark.parametrize("dtype", [F32, BF])
def test_groups_of_one_row_far_apart(dtype):
    """Groups of a row, each of its own size: group by group."""
    N, groups, rows = 1024, 8, 5
    x = norm_inputs(rows, N, dtype, seed=4, groups=groups, gate="silu", residual=False, next=False, scale=False)
    size = torch.tensor([1.0, 1e20, 1e-3, 1e35, 1e6, 1e17, 1e-9, 1e30]).repeat_interleave(N // groups)
    x["y"] = (torch.randn(rows, N, generator=torch.Generator().manual_seed(2)) * size).to(dtype)
    ref, got = norm_reference(x), run(cuda(x))
    for n in ("x", "dy", "dgate"):
        a, b = got[n].cpu().view(rows, groups, -1), ref[n].view(rows, groups, -1)
        for i in range(groups):
            e = rel(a[:, i], b[:, i])
            assert e <= 4e-6 + (2.0 ** -8 if dtype == BF else 0), (n, i, e)
    assert rel(got["dweight"], ref["dweight"]) <= 1e-5
