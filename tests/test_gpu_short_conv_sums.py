"""The short convolution's weight gradients of batches of many short sequences, whose sums run
over every element of the batch."""
import pytest
import torch

from paper_2606_27229_amd import carve

pytestmark = pytest.mark.gpu

# Values of one sign, one row a sequence, no activation.  A sequence's term is a product,
# rounded once (2^-24 of it); the f32 sum over its workgroup's runs adds zeros to it, which
# rounds nothing; the sum over workgroups is in 64 bits (2^18 * 2^-53 of it at most) and is
# rounded once to f32: 2^-24.
TOL = 2 * 2.0 ** -24


@pytest.mark.parametrize("B", [1 << 14, 1 << 18])
@pytest.mark.parametrize("W", [2, 4])
def test_many_sequences_of_one_token(B, W):
    C = 8
    gen = torch.Generator().manual_seed(B + W)
    x, dy = 0.5 + torch.rand(B, 1, C, generator=gen), torch.full((B, 1, C), 0.3)
    x0 = 0.5 + torch.rand(B, W - 1, C, generator=gen)
    x[..., 0], x0[..., 0] = 0.7, 1.1    # a channel of equal terms: their roundings do not even out
    weight, bias = torch.rand(C, W, generator=gen), torch.zeros(C)
    got = carve.short_conv_bwd(x.cuda(), weight.cuda(), dy.cuda(), x0.cuda(), bias=bias.cuda(), activation=None)
    d, z = dy.double(), torch.cat([x0, x], 1).double()
    for n, ref in (("dweight", (d * z).sum(0).T), ("dbias", d.sum((0, 1)))):
        off = ((got[n].cpu().double() - ref) / ref).abs().max()
        assert off <= TOL, (n, float(off))
