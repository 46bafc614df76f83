"""What the gated delta rule's calls keep apart: sequences, states and runs of one pool."""
import pytest
import torch

from paper_2606_27229_amd import carve
from tests.gdr_util import cuda, gdr_inputs, gdr_reference, rel

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
TOKENS = ("q", "k", "v", "g", "beta", "dO")


def run(x, offsets=None):
    o, S_T, S_c = carve.gdr_chunk_fwd(x["q"], x["k"], x["v"], x["g"], x["beta"], x["S0"], scale=x["scale"], offsets=offsets)
    got = carve.gdr_chunk_bwd(x["q"], x["k"], x["v"], x["g"], x["beta"], S_c, x["dO"], x["dS_T"], scale=x["scale"],
                              offsets=offsets)
    return dict(got, o=o, S_T=S_T)


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("Hk,Hv,Dk,Dv,dtype", [(1, 2, 64, 64, BF), (2, 2, 32, 64, F32), (2, 4, 128, 128, BF)])
def test_a_broken_sequence_breaks_no_other(value, Hk, Hv, Dk, Dv, dtype):
    """NaN or infinities in every tensor of one packed sequence, inside chunks that its
    neighbours' rows lie next to: all other rows and states are bitwise those of a sound run."""
    lens = [70, 1, 45, 130, 0, 20]
    x = cuda(gdr_inputs(1, sum(lens), Hk, Hv, Dk, Dv, dtype, seed=17, seqs=len(lens)))
    off = torch.tensor([0] + lens).cumsum(0)
    offsets = off.to(torch.int32).cuda()
    sound = run(x, offsets)
    for bad in (2, 3):
        y = {n: t.clone() if isinstance(t, torch.Tensor) else t for n, t in x.items()}
        a, b = int(off[bad]), int(off[bad + 1])
        for n in TOKENS:
            y[n][:, a:b] = -value if n == "g" else value
        for n in ("S0", "dS_T"):
            y[n][bad] = value
        got = run(y, offsets)
        others = [i for i in range(len(lens)) if i != bad]
        for n in ("o", "dq", "dk", "dv", "dg", "dbeta"):
            assert torch.equal(got[n][:, :a], sound[n][:, :a]) and torch.equal(got[n][:, b:], sound[n][:, b:]), (n, bad)
        for n in ("S_T", "dS0"):
            assert torch.equal(got[n][others], sound[n][others]), (n, bad)
        assert not torch.isfinite(got["o"][:, a:b].float()).any()


@pytest.mark.parametrize("Hk,Hv,Dk,Dv", [(2, 2, 128, 256), (3, 12, 128, 256), (1, 4, 32, 256), (2, 4, 128, 32)])
def test_f32_packed(Hk, Hv, Dk, Dv):
    """Wide f32 heads in packed sequences, value heads sharing key heads (the tolerances of the
    other tests of the rule in f32: 192 * 2^-24 of a result, 4 times that of dg and dbeta)."""
    print(f"case f32 packed Hk={Hk} Hv={Hv} Dk={Dk} Dv={Dv}", flush=True)
    lens = [100, 0, 1, 77, 64]
    x = gdr_inputs(1, sum(lens), Hk, Hv, Dk, Dv, F32, seed=Hv + Dk, seqs=len(lens))
    offsets = torch.tensor([0] + lens).cumsum(0).to(torch.int32).cuda()
    ref, got = gdr_reference(x, lens), run(cuda(x), offsets)
    for n in ref:
        assert rel(got[n], ref[n]) <= 1.2e-5 * (4 if n in ("dg", "dbeta") else 1), (n, rel(got[n], ref[n]))


def test_two_of_four_proposed_tokens_are_kept():
    """A call of several tokens leaves the state behind the last one.  Where only some of them
    are kept, the states from before the call are put back and the kept tokens run again."""
    x = gdr_inputs(2, 6, 2, 4, 64, 64, BF, seed=23)
    d = cuda(x)
    part = lambda a, b: [d[n][:, a:b].contiguous() for n in ("q", "k", "v", "g", "beta")]
    pool = torch.zeros(4, 4, 64, 64, device="cuda")
    slots = torch.tensor([3, 0], dtype=torch.int32, device="cuda")
    pool[slots.long()] = d["S0"]
    before = pool[slots.long()]
    four = carve.gdr_step(*part(0, 4), pool, slots, scale=x["scale"])
    pool[slots.long()] = before
    two = carve.gdr_step(*part(0, 2), pool, slots, scale=x["scale"])
    assert torch.equal(two, four[:, :2])
    rest = carve.gdr_step(*part(2, 6), pool, slots, scale=x["scale"])
    ref = gdr_reference(x, grads=False)
    assert rel(torch.cat([two, rest], 1), ref["o"]) <= 2.0 ** -8 + 128 * 6 * 2.0 ** -24
    assert rel(pool[slots.long()], ref["S_T"]) <= 128 * 6 * 2.0 ** -24


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_a_broken_state_of_the_pool_breaks_no_other(value):
    x = cuda(gdr_inputs(3, 2, 1, 2, 128, 64, F32, seed=29))
    args = [x[n] for n in ("q", "k", "v", "g", "beta")]
    slots = torch.tensor([2, 0, 1], dtype=torch.int32, device="cuda")
    pools = [x["S0"].clone(), x["S0"].clone()]
    pools[1][0] = value
    o, p = (carve.gdr_step(*args, pool, slots) for pool in pools)
    for b, s in ((0, 2), (2, 1)):
        assert torch.equal(o[b], p[b]) and torch.equal(pools[0][s], pools[1][s])
    assert not torch.isfinite(p[1]).any()
