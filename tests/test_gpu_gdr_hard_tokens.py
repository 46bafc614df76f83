"""Decay gradients of single tokens that decay hard among soft ones, each against its own
exact value.

dg_t is a sum of what the decay at t multiplies, so every term of it holds e^{g_t}: at a
token with g = -16 it is 1e-7 of its neighbours', and a rounding of theirs that reached it
would be all that is left.  Tolerance, relative to the exact dg of the token alone: the
terms' f32 bound of 192 * 2^-24 (sums of up to 64 + 128 products and the inverse of 64
steps), and of the decay factor the roundings of its exponent x and of x log2(e), 2^-25 |x|
each and 2^-26 |x| of the constant, so less than 2 * 2^-24 |x| with |x| <= |g| + 16 (the soft
decays of a chunk); times 4, as terms of both signs are added up.
"""
import pytest
import torch

from paper_2606_27229_amd import carve
from tests.gdr_util import cuda, gdr_inputs, gdr_reference, rel

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


def dg_of(x, offsets=None):
    d = cuda(x)
    _, _, S_c = carve.gdr_chunk_fwd(d["q"], d["k"], d["v"], d["g"], d["beta"], d["S0"], scale=x["scale"], offsets=offsets)
    r = carve.gdr_chunk_bwd(d["q"], d["k"], d["v"], d["g"], d["beta"], S_c, d["dO"], d["dS_T"], scale=x["scale"],
                            offsets=offsets)
    return r["dg"]


# in every tile of 16 tokens, at their borders, in the second chunk and in the short last one
AT = (0, 1, 7, 15, 16, 30, 33, 47, 48, 62, 63, 64, 85, 127, 130, 139)


@pytest.mark.parametrize("Hk,Hv,Dk,Dv,dtype", [(4, 8, 64, 64, F32), (8, 8, 32, 32, F32), (4, 8, 128, 64, BF), (8, 8, 64, 256, BF)])
@pytest.mark.parametrize("hard", [-4.0, -8.0, -12.0, -16.0, -30.0])
def test_one_hard_token(hard, Hk, Hv, Dk, Dv, dtype):
    """A sequence for every place, one hard token each."""
    print(f"case hard token {hard} Hk={Hk} Hv={Hv} Dk={Dk} Dv={Dv} {dtype}", flush=True)
    x = gdr_inputs(len(AT), 140, Hk, Hv, Dk, Dv, dtype, seed=Dk + Dv)
    for n, t in enumerate(AT):
        x["g"][n, t] = hard
    ref = gdr_reference(x)["dg"]
    got = dg_of(x)
    tol = 4 * (192 + 2 * (16 - hard)) * 2.0 ** -24
    errs = {t: rel(got[n, t], ref[n, t]) for n, t in enumerate(AT)}
    print("rel errors:", {t: float("%.2g" % e) for t, e in errs.items()}, f"of {tol:.2g}", flush=True)
    assert max(errs.values()) <= tol, errs


@pytest.mark.parametrize("dtype", [F32, BF])
def test_hard_tokens_of_packed_sequences(dtype):
    """Two hard tokens of a sequence, a few tokens apart and in different chunks."""
    lens = [100, 1, 0, 90, 70]
    x = gdr_inputs(1, sum(lens), 4, 8, 64, 64, dtype, seed=9, seqs=len(lens))
    at = (20, 29, 70, 100, 101 + 33, 101 + 80, 191 + 66)
    for t in at:
        x["g"][:, t] = -11.0
    ref = gdr_reference(x, lens)["dg"]
    off = torch.tensor([0] + lens).cumsum(0).to(torch.int32).cuda()
    got = dg_of(x, off)
    # (one or two hard decays within a factor)
    tol = 4 * (192 + 2 * (16 + 22)) * 2.0 ** -24
    errs = {t: rel(got[0, t], ref[0, t]) for t in at}
    print("rel errors:", {t: float("%.2g" % e) for t, e in errs.items()}, f"of {tol:.2g}", flush=True)
    assert max(errs.values()) <= tol, errs


@pytest.mark.parametrize("Dk,Dv,dtype", [(64, 64, F32), (128, 128, BF), (32, 64, BF)])
def test_resets_have_no_gradient(Dk, Dv, dtype):
    """With g = -inf every term of a token's dg has a factor 0: it is 0, not a rounding of
    its neighbours'."""
    x = gdr_inputs(len(AT), 140, 2, 4, Dk, Dv, dtype, seed=13)
    for n, t in enumerate(AT):
        x["g"][n, t] = float("-inf")
    got = dg_of(x)
    for n, t in enumerate(AT):
        assert (got[n, t] == 0).all(), (t, got[n, t])
