"""The gated delta rule (chunked forward and backward, recurrent step) against its
token-by-token definition in 64 bits.

Tolerances (relative 2-norms), from the arithmetic:
  bf16 outputs (o, dq, dk, dv, dbeta): one rounding, at most eps / 2 = 2^-8 of every
    value, and f32 intermediates as below, far smaller: 2^-8.
  f32 outputs of bf16 tokens (S_T, dS0, dg): each f32 intermediate enters the matrix
    cores as two bf16 values, leaving out at most 2^-18 of it on each side of a
    product and 2^-18 for the product of the low parts, so 3 * 2^-18 = 1.2e-5 a
    product at the very most and a third of that in the mean.  A state or gradient
    takes at most four such products in a row: 5e-5.
  f32 tokens: f32 products, sums of up to 64 + 128 terms and the triangular inverse
    of 64 steps, all errors 2^-24 of a term: 192 * 2^-24 = 1.2e-5.
dg and dbeta are sums of terms that cancel: their error is measured against the
2-norm of the result as well, with a factor 4 for the cancellation.
"""
import pytest
import torch

from paper_2606_27229_amd import carve
from tests.gdr_util import cuda, gdr_inputs, gdr_reference, rel

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


def tolerance(name, dtype):
    cancel = 4 if name in ("dg", "dbeta") else 1
    if dtype == F32:
        return 1.2e-5 * cancel
    return 5e-5 * cancel if name in ("S_T", "dS0", "dg") else 2.0 ** -8


def compare(got, ref, dtype, names):
    errs = {n: rel(got[n], ref[n]) for n in names}
    print("rel errors:", {n: float("%.2g" % e) for n, e in errs.items()}, flush=True)
    for n in names:
        assert torch.isfinite(got[n].float()).all(), n
        assert errs[n] <= tolerance(n, dtype), (n, errs[n])


def run(x, offsets=None, backward=True, **kw):
    o, S_T, S_c = carve.gdr_chunk_fwd(x["q"], x["k"], x["v"], x["g"], x["beta"], x["S0"], scale=x["scale"],
                                      offsets=offsets, **kw)
    got = {"o": o, "S_T": S_T}
    if backward:
        got.update(carve.gdr_chunk_bwd(x["q"], x["k"], x["v"], x["g"], x["beta"], S_c, x["dO"], x["dS_T"],
                                       scale=x["scale"], offsets=offsets))
    torch.cuda.synchronize()
    return got


FWD = ("o", "S_T")
ALL = ("o", "S_T", "dq", "dk", "dv", "dg", "dbeta", "dS0")


@pytest.mark.parametrize("B,T,Hk,Hv,Dk,Dv,dtype", [
    (1, 1, 1, 1, 32, 32, F32), (1, 64, 1, 1, 64, 64, F32), (2, 65, 2, 4, 32, 64, F32), (1, 130, 1, 2, 128, 128, F32),
    (2, 200, 4, 4, 64, 32, F32), (1, 100, 1, 3, 64, 256, F32),
    (1, 1, 1, 1, 32, 32, BF), (1, 15, 1, 1, 128, 128, BF), (1, 64, 1, 1, 128, 128, BF), (2, 63, 2, 2, 64, 64, BF),
    (2, 129, 2, 6, 128, 64, BF), (3, 190, 3, 3, 32, 128, BF), (1, 321, 1, 4, 128, 256, BF), (1, 257, 9, 9, 64, 128, BF),
])
def test_chunks(B, T, Hk, Hv, Dk, Dv, dtype):
    print(f"case chunks B={B} T={T} Hk={Hk} Hv={Hv} Dk={Dk} Dv={Dv} {dtype}", flush=True)
    x = gdr_inputs(B, T, Hk, Hv, Dk, Dv, dtype, seed=B + T + Hk + Hv + Dk + Dv)
    compare(run(cuda(x)), gdr_reference(x), dtype, ALL)
