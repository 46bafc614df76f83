"""Offsets outside the contract (decreasing, negative, too large): the calls return, and every
output and workspace is written within its bounds, for every chain kernel."""
import ctypes

import pytest
import torch

from paper_2606_27229_amd import carve
from tests.gdr_util import cuda, gdr_inputs

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
PAD = 1 << 16     # elements on either side, more than a chunk's state of any head here


class Guarded:
    """Tensors that lie between values nothing may change."""

    def __init__(self):
        self.whole = []

    def __call__(self, shape, dtype, fill=5):
        n = 1
        for s in shape:
            n *= s
        flat = torch.full((n + 2 * PAD,), fill, dtype=dtype, device="cuda")
        self.whole.append((flat, n, fill))
        return flat[PAD:PAD + n].view(shape)

    def check(self):
        for i, (flat, n, fill) in enumerate(self.whole):
            assert (flat[:PAD] == fill).all() and (flat[PAD + n:] == fill).all(), i


OFFSETS = [[0, 150, 50, 500, -7], [300, 10, 0, 0, 200], [-5, -4, 1 << 30, 3, 2], [200, 200, 199, 63, 64],
           [-(1 << 31), (1 << 31) - 1, -1, (1 << 31) - 1, 0]]


# one wave a tile; pairs, a tile a workgroup and two; four tiles a workgroup backward
@pytest.mark.parametrize("Hk,Hv,Dk,Dv,dtype,many", [
    (1, 2, 32, 64, BF, 1), (2, 2, 32, 32, F32, 1), (1, 2, 64, 64, BF, 1), (2, 4, 128, 128, F32, 1), (5, 10, 128, 128, BF, 1),
    (5, 10, 64, 128, F32, 1), (4, 8, 64, 128, BF, 20)])
def test_every_output_stays_in_its_bounds(Hk, Hv, Dk, Dv, dtype, many):
    T = 200
    for offs in OFFSETS:
        off = [offs[0]] + offs[1:] * many
        n = len(off) - 1
        print(f"case bad offsets {offs} x{many} Hk={Hk} Hv={Hv} Dk={Dk} Dv={Dv} {dtype}", flush=True)
        x = cuda(gdr_inputs(1, T, Hk, Hv, Dk, Dv, dtype, seed=3, seqs=n))
        d = carve.GdrDims(1, T, n, Hk, Hv, Dk, Dv, carve.CARVE_BF16 if dtype == BF else carve.CARVE_F32, 1.0,
                          *[s for t in "qkv" for s in x[t].stride()[:3]])
        lib = carve.load_library()
        chunks = lib.carve_gdr_chunk_count(ctypes.byref(d))
        g = Guarded()
        ws = [g((lib.carve_gdr_workspace_size(ctypes.byref(d), b),), torch.uint8) for b in (0, 1)]
        out = {"o": g((1, T, Hv, Dv), dtype), "S_T": g((n, Hv, Dv, Dk), F32), "S_chunks": g((chunks, Hv, Dv, Dk), F32)}
        back = {"dq": g((1, T, Hk, Dk), dtype), "dk": g((1, T, Hk, Dk), dtype), "dv": g((1, T, Hv, Dv), dtype),
                "dg": g((1, T, Hv), F32), "dbeta": g((1, T, Hv), dtype), "dS0": g((n, Hv, Dv, Dk), F32)}
        o = torch.tensor(off, dtype=torch.int64).to(torch.int32).cuda()
        a = (x["q"], x["k"], x["v"], x["g"], x["beta"])
        carve.gdr_chunk_fwd(*a, x["S0"], offsets=o, out=out, workspace=ws[0])
        carve.gdr_chunk_bwd(*a, out["S_chunks"], x["dO"], x["dS_T"], offsets=o, out=back, workspace=ws[1])
        torch.cuda.synchronize()
        g.check()
