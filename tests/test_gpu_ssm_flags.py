"""What the scan's flags say is read at every call, also from a tensor that has changed since."""
import pytest
import torch

from gdr_util import cuda
from paper_2606_27229_amd import carve
from ssm_util import ssm_inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("device", ["cpu", "cuda"])
def test_softplus_of_a_tensor_that_changes(device):
    x = cuda(ssm_inputs(1, 70, 1, 2, 32, 32, torch.float32, 3, softplus=False))   # (steps that either flag takes)
    args, kw = [x[n] for n in ("x", "dt", "A", "Bm", "Cm")], {"D": x["D"], "dt_bias": x["dt_bias"]}

    def results(flag):
        y, S_T, S_c = carve.ssm_chunk_fwd(*args, x["S0"], softplus=flag, **kw)
        back = carve.ssm_chunk_bwd(*args, S_c, x["dy"], x["dS_T"], softplus=flag, **kw)
        pool = x["S0"].clone()
        return {"y": y, "S_T": S_T, **back, "step": carve.ssm_step(*args, pool, softplus=flag, **kw), "pool": pool}

    want = {value: results(value) for value in (True, False)}
    assert not torch.equal(want[True]["y"], want[False]["y"])
    flag = torch.tensor(True, device=device)
    for value in (True, False, True):
        flag.fill_(value)
        got = results(flag)
        for n, t in want[value].items():
            assert torch.equal(got[n], t), (value, n)
