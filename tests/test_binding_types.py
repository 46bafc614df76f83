"""What is no tensor is refused by name, wherever a tensor is expected."""
import pytest
import torch

from paper_2606_27229_amd import carve


@pytest.mark.parametrize("value", [[0, 4], (0, 4), 3.0, "offsets"])
def test_not_a_tensor(value):
    with pytest.raises(TypeError, match="offsets must be a GPU tensor"):
        carve._same_device(torch.device("cpu"), offsets=value)
    carve._same_device(torch.device("cpu"), offsets=None, S0=torch.zeros(2))


@pytest.mark.gpu
def test_every_optional_tensor_of_the_entry_points():
    z = lambda *s, dt=torch.float32: torch.zeros(s, dtype=dt, device="cuda")
    q, g = z(1, 4, 1, 32), z(1, 4, 1)
    args, state = (q, q, q, g, g), z(1, 1, 32, 32)
    ws = z(1 << 20)
    y, w = z(2, 64), z(64)
    calls = {
        "offsets": lambda: carve.gdr_chunk_fwd(*args, offsets=[0, 4]),
        "S0": lambda: carve.gdr_chunk_fwd(*args, [0.0]),
        "workspace": lambda: carve.gdr_chunk_fwd(*args, workspace=1 << 20),
        "o": lambda: carve.gdr_chunk_fwd(*args, out={"o": [0.0]}),
        "dO": lambda: carve.gdr_chunk_bwd(*args, state, [0.0]),
        "dS_T": lambda: carve.gdr_chunk_bwd(*args, state, q, [0.0]),
        "dq": lambda: carve.gdr_chunk_bwd(*args, state, q, out={"dq": [0.0]}),
        "slots": lambda: carve.gdr_step(*args, state, [0]),
        "out": lambda: carve.gdr_step(*args, state, out=[0]),
        "weight": lambda: carve.block_norm_fwd(y, [1.0] * 64),
        "gate": lambda: carve.block_norm_fwd(y, w, gate=[0.0]),
        "scale": lambda: carve.block_norm_fwd(y, w, scale=2.0),
        "next_weight": lambda: carve.block_norm_fwd(y, w, next_weight=[1.0]),
        "x": lambda: carve.block_norm_fwd(y, w, out={"x": [0.0]}),
        "dx": lambda: carve.block_norm_bwd(y, w, [0.0]),
        "dy": lambda: carve.block_norm_bwd(y, w, y, out={"dy": [0.0]}),
    }
    for name, call in calls.items():
        with pytest.raises(TypeError, match=f"^{name} must be a GPU tensor"):
            call()
    carve.gdr_chunk_fwd(*args, state, workspace=ws)
