"""Rotary positions on the GPU against their definition in 64 bits."""
import pytest
import torch

from gdr_util import rel
from paper_2606_27229_amd import carve
from ssm_util import TOL, rotary_reference

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32


def tensors(B, T, Hq, Hk, D, dtype, seed=1):
    gen = torch.Generator().manual_seed(seed)
    return [torch.randn(B, T, h, D, generator=gen).to(dtype) if h else None for h in (Hq, Hk)]


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("B,T,Hq,Hk,D,rot", [
    (1, 1, 1, 0, 32, 32), (2, 5, 4, 2, 64, 64), (1, 300, 3, 1, 128, 64), (3, 33, 16, 4, 96, 32), (1, 7, 2, 2, 1024, 512),
    (1, 3000, 16, 16, 128, 128), (2, 40, 9, 3, 72, 16)])
def test_positions(B, T, Hq, Hk, D, rot, interleaved, dtype):
    q, k = tensors(B, T, Hq, Hk, D, dtype)
    freq = carve.rotary_frequencies(rot, stretch=2.0)
    start = torch.tensor([0, 700000, 123][:B], dtype=torch.int32)
    pos = start[:, None] + torch.arange(T)
    kw = {"start": start.cuda(), "interleaved": interleaved, "amplitude": 1.25}
    qo, ko = carve.rotary_fwd(q.cuda(), None if k is None else k.cuda(), freq, **kw)
    bq, bk = carve.rotary_bwd(q.cuda(), None if k is None else k.cuda(), freq, **kw)
    by = carve.rotary_fwd(q.cuda(), None if k is None else k.cuda(), freq, positions=pos.int().cuda(), interleaved=interleaved, amplitude=1.25)
    for x, got, back, same in ((q, qo, bq, by[0]), (k, ko, bk, by[1])):
        if x is None:
            assert got is None and back is None
            continue
        for t, sign in ((got, 1), (back, -1)):
            ref = rotary_reference(x, freq.cpu(), pos, interleaved, 1.25, sign)
            assert rel(t, ref) <= TOL[dtype]
            assert torch.equal(t[..., rot:].cpu(), x[..., rot:])
        assert torch.equal(got, same)


@pytest.mark.parametrize("lens,first,T", [([5, 0, 70, 1], 0, 80), ([9, 20], 3, 40), ([0], 1, 4)])
def test_packed(lens, first, T):
    q, k = tensors(1, T, 4, 2, 64, F)
    ends = torch.tensor([first] + lens).cumsum(0).int().cuda()
    start = torch.arange(len(lens), dtype=torch.int32) * 1000
    freq = carve.rotary_frequencies(64)
    out = {"q": torch.full_like(q, 7.0).cuda(), "k": torch.full_like(k, 7.0).cuda()}
    qo, ko = carve.rotary_fwd(q.cuda(), k.cuda(), freq, start=start.cuda(), offsets=ends, out=out)
    assert qo is out["q"] and ko is out["k"]
    pos = torch.cat([torch.zeros(first)] + [int(start[i]) + torch.arange(n) for i, n in enumerate(lens)])
    pos = torch.cat([pos, torch.zeros(T - pos.numel())])[None]
    rows = slice(first, first + sum(lens))
    for x, t in ((q, qo), (k, ko)):
        assert rel(t[:, rows], rotary_reference(x, freq.cpu(), pos, False, 1.0)[:, rows]) <= TOL[F]
        assert (t[:, :first] == 7).all() and (t[:, first + sum(lens):] == 7).all()


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("rot", [32, 64])
def test_in_place_on_slices(dtype, rot):
    """Queries and keys turned where they lie in one projection; the rest of it is kept."""
    B, T, Hq, Hk, D = 2, 30, 4, 2, 64
    wide = torch.randn(B, T, (Hq + 2 * Hk) * D + 32, device="cuda").to(dtype)
    was = wide.clone()
    cut = lambda t: (t[..., :Hq * D].unflatten(-1, (Hq, D)), t[..., Hq * D:(Hq + Hk) * D].unflatten(-1, (Hk, D)))
    q, k = cut(wide)
    freq = carve.rotary_frequencies(rot)
    ref = carve.rotary_fwd(*(t.clone() for t in cut(was)), freq)
    got = carve.rotary_fwd(q, k, freq, out={"q": q, "k": k})
    assert got[0] is q and got[1] is k
    assert torch.equal(q, ref[0]) and torch.equal(k, ref[1])
    assert torch.equal(wide[..., (Hq + Hk) * D:], was[..., (Hq + Hk) * D:])
    # into slices of another tensor, heads before tokens
    other = torch.zeros(B, Hq, T, D, device="cuda", dtype=dtype).transpose(1, 2)
    a, b = cut(was)
    carve.rotary_fwd(a, b, freq, out={"q": other})
    assert torch.equal(other, ref[0])


def test_backward_is_the_transposed_map():
    q, k = tensors(1, 50, 2, 1, 64, F)
    dq, dk = tensors(1, 50, 2, 1, 64, F, seed=2)
    freq = carve.rotary_frequencies(48)
    qo, ko = carve.rotary_fwd(q.cuda(), k.cuda(), freq, amplitude=0.7)
    bq, bk = carve.rotary_bwd(dq.cuda(), dk.cuda(), freq, amplitude=0.7)
    for x, y, d, b in ((q, qo, dq, bq), (k, ko, dk, bk)):
        one, two = float((y.cpu().double() * d.double()).sum()), float((x.double() * b.cpu().double()).sum())
        # 2^-23 of each of the terms, at random
        assert abs(one - two) <= 2.0 ** -22 * float((y.cpu().double() * d.double()).square().sum().sqrt()) * 4


def test_far_positions_keep_their_angles():
    """The largest position: angles of 2^31, of which f32 would keep none."""
    q, _ = tensors(1, 1, 1, 0, 32, F)
    freq = carve.rotary_frequencies(32)
    pos = torch.tensor([[2 ** 31 - 1]], dtype=torch.int32)
    got, _ = carve.rotary_fwd(q.cuda(), None, freq, positions=pos.cuda())
    assert rel(got, rotary_reference(q, freq.cpu(), pos, False, 1.0)) <= TOL[F]
