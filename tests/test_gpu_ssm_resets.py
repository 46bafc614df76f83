"""Decays of -inf: the state begins anew at every token, in both directions."""
import pytest
import torch

from gdr_util import cuda, rel
from paper_2606_27229_amd import carve
from ssm_util import TOL, ssm_inputs, ssm_reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("A", [float("-inf"), -3e38])
def test_a_head_that_keeps_nothing(A, dtype):
    """A head whose A is -inf (its steps are not 0) beside one that keeps its state."""
    x = ssm_inputs(1, 150, 1, 2, 32, 32, dtype, 9)
    x["A"][0] = -1e30   # (the definition's derivative has -inf times 0 else; every decay is 0 with either)
    ref = ssm_reference(x)
    x["A"][0] = A
    d = cuda(x)
    args, kw = [d[n] for n in ("x", "dt", "A", "Bm", "Cm")], {"D": d["D"], "dt_bias": d["dt_bias"]}
    y, S_T, S_c = carve.ssm_chunk_fwd(*args, d["S0"], **kw)
    got = {"y": y, "S_T": S_T, **carve.ssm_chunk_bwd(*args, S_c, d["dy"], d["dS_T"], **kw)}
    for n, r in ref.items():
        assert torch.isfinite(got[n]).all(), n
        assert rel(got[n], r) <= TOL[got[n].dtype], n
    assert got["dA"][0] == 0 and (got["dS0"][:, 0] == 0).all()
    state, steps = d["S0"].clone(), []
    for t in range(3):
        cut = [a if a is d["A"] else a[:, t:t + 1] for a in args]
        steps.append(carve.ssm_step(*cut, state, **kw))
    assert rel(torch.cat(steps, 1), ref["y"][:, :3]) <= TOL[dtype]
