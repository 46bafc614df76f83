"""Queries' and keys' outputs that share a tensor: every element has a place of its own, in
the rows behind the first one too (no GPU needed: refused before any HIP call)."""
import ctypes

import pytest

from test_abi_ssm_host import UNSUPPORTED, far, rdims, rot


def places(first, strides, counts, D):
    return [first + b * strides[0] + t * strides[1] + h * strides[2] + e
            for b in range(counts[0]) for t in range(counts[1]) for h in range(counts[2]) for e in range(D)]


# B, T, heads, strides of batch, token and head, elements from the queries' to the keys'
COLLIDING = [
    (2, 5, 1, (144, 32, 16), 16),    # the key of (0, 4) is the query of (1, 0)
    (2, 2, 1, (96, 64, 16), 32),     # the key of (0, 1) is the query of (1, 0)
    (3, 2, 1, (48, 128, 16), 32),    # batches within a token: the key of (2, 0) is the query of (0, 1)
    (2, 3, 1, (16, 64, 16), 16),     # a batch's query is the other one's key
]


@pytest.mark.parametrize("swapped", [False, True])
@pytest.mark.parametrize("B,T,H,strides,off", COLLIDING)
def test_outputs_that_meet_in_later_rows(B, T, H, strides, off, swapped):
    q, k = places(0, strides, (B, T, H), 16), places(off, strides, (B, T, H), 16)
    assert len(set(q)) == len(q) and len(set(k)) == len(k)   # (each by itself has its places)
    assert set(q) & set(k)
    d = rdims(B=B, T=T, Hq=H, Hk=H, D=16, rot=16,
              **{f"{n}_{w}": s for n in ("qo", "ko") for w, s in zip(("batch", "token", "head"), strides)})
    a = far(8)
    a[3] = a[5] = None
    a[7] = ctypes.c_void_p(a[6].value + 2 * off)
    if swapped:
        a[6], a[7] = a[7], a[6]
    assert rot(d, a) == UNSUPPORTED
