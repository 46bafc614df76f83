"""Host-side refusals of the gated delta rule and the block norm (no GPU needed): sizes,
strides, alignment, missing and conflicting arguments, workspaces and overlapping tensors
are rejected before any HIP call."""
import ctypes

import pytest
import torch

from paper_2606_27229_amd import carve

OK, NULL, SHAPE, UNSUPPORTED, ALIGN, WORKSPACE, ARG = 0, -1, -2, -3, -4, -5, -7


def gdims(**kw):
    d = dict(B=2, T=100, N=0, Hk=2, Hv=4, Dk=64, Dv=64, dtype=carve.CARVE_BF16, scale=0.125)
    d.update({k: v for k, v in kw.items() if k in d})
    H = {"q": d["Hk"], "k": d["Hk"], "v": d["Hv"]}
    D = {"q": d["Dk"], "k": d["Dk"], "v": d["Dv"]}
    for n in "qkv":
        d[n + "_batch"], d[n + "_token"], d[n + "_head"] = d["T"] * H[n] * D[n], H[n] * D[n], D[n]
    d.update({k: v for k, v in kw.items() if k[:2] in ("q_", "k_", "v_")})
    return carve.GdrDims(*(d[f] for f, _ in carve.GdrDims._fields_))


def far(n):
    """Distinct addresses far apart; never dereferenced."""
    return [ctypes.c_void_p(1 << 40 | i << 32) for i in range(n)]


def fwd(d, args=None, ws=1 << 31):
    lib = carve.load_library()
    a = args or far(11)   # q k v g beta S0 offsets o S_T S_chunks workspace
    if args is None and d.N == 0:
        a[6] = None
    return lib.carve_gdr_chunk_fwd(ctypes.byref(d), *a, ws, None)


BAD_DIMS = [
    (dict(B=0), SHAPE), (dict(T=0), SHAPE), (dict(N=-1), SHAPE), (dict(N=3), SHAPE), (dict(Hk=0), SHAPE), (dict(Dv=0), SHAPE),
    (dict(Dk=48), UNSUPPORTED), (dict(Dk=256), UNSUPPORTED), (dict(Dv=96), UNSUPPORTED), (dict(Hk=3), UNSUPPORTED),
    (dict(dtype=5), UNSUPPORTED), (dict(Hk=1, Hv=65536), UNSUPPORTED), (dict(B=1 << 15, T=1 << 16), UNSUPPORTED),
    (dict(scale=float("nan")), ARG), (dict(scale=float("inf")), ARG), (dict(q_token=-128), ARG),
    (dict(k_token=130), ALIGN), (dict(v_head=4), ALIGN), (dict(q_token=1 << 23), UNSUPPORTED),
    (dict(q_batch=1 << 46), UNSUPPORTED),
]


@pytest.mark.parametrize("kw,status", BAD_DIMS)
def test_gdr_dims(kw, status):
    lib = carve.load_library()
    d = gdims(**kw)
    assert fwd(d) == status
    assert lib.carve_gdr_chunk_count(ctypes.byref(d)) == 0
    assert lib.carve_gdr_workspace_size(ctypes.byref(d), 0) == 0 and lib.carve_gdr_workspace_size(ctypes.byref(d), 1) == 0
    ptrs = far(17)
    assert lib.carve_gdr_chunk_bwd(ctypes.byref(d), *ptrs[:16], 1 << 40, None) == status
    assert lib.carve_gdr_step(ctypes.byref(d), *ptrs[:6], 8, *ptrs[6:8], None) == status


@pytest.mark.parametrize("kw", [dict(B=1 << 15, T=1, Hk=64, Hv=64, Dv=128), dict(B=1, N=1 << 20, T=64, Hk=2, Hv=4, Dv=64),
                                dict(B=1 << 15, T=64 * 256, Hk=1, Hv=1, Dv=32), dict(B=1, N=1 << 23, T=1, Hk=1, Hv=1, Dv=32)])
def test_chunk_calls_beyond_a_launch(kw):
    """2^32 threads or more of a kernel are refused, not left to the launch; the step, which
    spreads them over three dimensions, has no such bound."""
    lib = carve.load_library()
    d = gdims(**kw)
    assert fwd(d, ws=1 << 62) == UNSUPPORTED
    assert lib.carve_gdr_chunk_bwd(ctypes.byref(d), *far(16), 1 << 62, None) == UNSUPPORTED
    assert lib.carve_gdr_chunk_count(ctypes.byref(d)) == 0 and lib.carve_gdr_workspace_size(ctypes.byref(d), 0) == 0
    if not d.N:   # (past the sizes' checks: the missing tensors are what is refused)
        assert lib.carve_gdr_step(ctypes.byref(d), *[None] * 6, 1 << 16, None, None, None) == NULL


def test_gdr_sizes():
    lib = carve.load_library()
    count = lambda **kw: lib.carve_gdr_chunk_count(ctypes.byref(gdims(**kw)))
    assert count() == 2 * 2 and count(T=64) == 2 and count(T=1) == 2
    assert count(B=1, N=3) == 1 + 3 and count(B=1, N=1, T=64) == 2
    d = gdims()
    state = 4 * 64 * 64 * 4
    assert lib.carve_gdr_workspace_size(ctypes.byref(d), 1) >= lib.carve_gdr_workspace_size(ctypes.byref(d), 0) + 4 * state
    assert lib.carve_gdr_chunk_count(None) == 0 and lib.carve_gdr_workspace_size(None, 0) == 0


def test_gdr_forward_arguments():
    lib = carve.load_library()
    d = gdims()
    need = lib.carve_gdr_workspace_size(ctypes.byref(d), 0)
    base = far(11)
    base[6] = None
    for i in (0, 1, 2, 3, 4, 7):      # q k v g beta o
        a = list(base)
        a[i] = None
        assert fwd(d, a) == NULL, i
    for i in (0, 1, 2, 3, 4, 5, 7, 8, 9, 10):
        a = list(base)
        a[i] = ctypes.c_void_p(a[i].value + 8)
        assert fwd(d, a) == ALIGN, i
    assert fwd(d, base, need - 1) == WORKSPACE
    a = list(base)
    a[10] = None
    assert fwd(d, a) == WORKSPACE
    assert fwd(d, far(11)) == ARG                       # offsets without packed sequences
    packed = gdims(B=1, N=3)
    assert fwd(packed, base) == NULL                    # and packed sequences without offsets
    for out in (7, 8, 9, 10):
        for other in (0, 2, 5, 7):
            if out == other:
                continue
            a = list(base)
            a[out] = a[other]
            assert fwd(d, a) == UNSUPPORTED, (out, other)
    a = list(base)
    a[7] = ctypes.c_void_p(a[2].value + (2 * 100 * 4 * 64 - 8) * 2)   # o begins in v's last 16 bytes
    assert fwd(d, a) == UNSUPPORTED


def test_gdr_backward_arguments():
    lib = carve.load_library()
    d = gdims()
    need = lib.carve_gdr_workspace_size(ctypes.byref(d), 1)
    base = far(16)   # q k v g beta S_chunks offsets dO dS_T dq dk dv dg dbeta dS0 workspace
    base[6] = None
    call = lambda a, ws=need: lib.carve_gdr_chunk_bwd(ctypes.byref(d), *a, ws, None)
    for i in (0, 1, 2, 3, 4, 5, 7, 9, 10, 11, 12, 13):
        a = list(base)
        a[i] = None
        assert call(a) == NULL, i
    for i in [i for i in range(16) if i != 6]:
        a = list(base)
        a[i] = ctypes.c_void_p(a[i].value + 4)
        assert call(a) == ALIGN, i
    assert call(base, need - 1) == WORKSPACE
    for out in (9, 10, 11, 12, 13, 14, 15):
        for other in (0, 5, 7, 9):
            if out != other:
                a = list(base)
                a[out] = a[other]
                assert call(a) == UNSUPPORTED, (out, other)
    assert call(far(16)) == ARG


def test_gdr_step_arguments():
    lib = carve.load_library()
    base = far(8)    # q k v g beta slots | pool | state o
    call = lambda a, pool=8, d=gdims(T=1): lib.carve_gdr_step(ctypes.byref(d), *a[:6], pool, *a[6:], None)
    for i in (0, 1, 2, 3, 4, 6, 7):
        a = list(base)
        a[i] = None
        assert call(a) == NULL, i
    assert call(base, 0) == SHAPE
    a = list(base)
    a[5] = None
    assert call(a, 1) == SHAPE                          # no slots: a state for every sequence
    assert call(base, d=gdims(B=1, N=1, T=1)) == SHAPE  # packed sequences: not here
    assert call(base, d=gdims(B=65536, T=1)) == UNSUPPORTED
    a = list(base)
    a[5] = ctypes.c_void_p(a[5].value + 2)
    assert call(a) == ALIGN
    a = list(base)
    a[7] = a[2]
    assert call(a) == UNSUPPORTED


def ndims(**kw):
    d = dict(rows=10, N=256, groups=1, dtype=carve.CARVE_BF16, gate_act=1, eps=1e-6, alpha=1.0, y_stride=256, gate_stride=256,
             residual_stride=256)
    d.update(kw)
    return carve.BlockNormDims(*(d[f] for f, _ in carve.BlockNormDims._fields_))


NORM_BAD = [
    (dict(rows=0), SHAPE), (dict(N=0), SHAPE), (dict(groups=0), SHAPE), (dict(groups=3), SHAPE),
    (dict(N=252), UNSUPPORTED), (dict(N=8200), UNSUPPORTED), (dict(dtype=3), UNSUPPORTED), (dict(rows=1 << 31), UNSUPPORTED),
    (dict(N=96, groups=4), UNSUPPORTED), (dict(N=2048, groups=2), UNSUPPORTED), (dict(N=32, groups=8), UNSUPPORTED),
    (dict(eps=-1.0), ARG), (dict(eps=float("nan")), ARG),
]


@pytest.mark.parametrize("kw,status", NORM_BAD)
def test_norm_dims(kw, status):
    lib = carve.load_library()
    d = ndims(**kw)
    assert lib.carve_block_norm_workspace_size(ctypes.byref(d)) == 0
    assert lib.carve_block_norm_fwd(ctypes.byref(d), *far(8), None) == status
    assert lib.carve_block_norm_bwd(ctypes.byref(d), *far(15), 1 << 30, None) == status


def test_norm_arguments():
    lib = carve.load_library()
    d = ndims()
    call = lambda a, d=d: lib.carve_block_norm_fwd(ctypes.byref(d), *a, None)
    base = far(8)   # y weight gate residual scale next_weight x h
    for i, st in ((0, NULL), (1, NULL), (6, NULL), (5, ARG), (7, ARG)):
        a = list(base)
        a[i] = None
        assert call(a) == st, i
    for i in range(8):
        a = list(base)
        a[i] = ctypes.c_void_p(a[i].value + 4)
        assert call(a) == ALIGN, i
    assert call(base, ndims(gate_act=0)) == ARG and call(base, ndims(gate_act=9)) == ARG
    assert call(base, ndims(alpha=float("inf"))) == ARG
    assert call(base, ndims(y_stride=-256)) == ARG and call(base, ndims(gate_stride=260)) == ALIGN
    assert call(base, ndims(residual_stride=1 << 44)) == UNSUPPORTED
    for out, other in ((6, 0), (7, 3), (7, 6), (6, 1)):
        a = list(base)
        a[out] = a[other]
        assert call(a) == UNSUPPORTED, (out, other)
    need = lib.carve_block_norm_workspace_size(ctypes.byref(d))
    base = far(15)  # y weight gate residual scale next_weight dx dh dy dgate dresidual dweight dscale dnext_weight workspace
    back = lambda a, ws=need: lib.carve_block_norm_bwd(ctypes.byref(d), *a, ws, None)
    for i in (0, 1, 8, 11):
        a = list(base)
        a[i] = None
        assert back(a) == NULL, i
    a = list(base)
    a[6] = a[7] = a[5] = a[13] = None
    assert back(a) == NULL                               # neither dx nor dh
    for i in (2, 3, 4, 5, 7, 9, 10, 12, 13):             # an input without its gradient, or the other way round
        a = list(base)
        a[i] = None
        assert back(a) == ARG, i
    assert back(base, need - 1) == WORKSPACE
    for i in range(15):
        a = list(base)
        a[i] = ctypes.c_void_p(a[i].value + 4)
        assert back(a) == ALIGN, i
    for out, other in ((8, 0), (9, 2), (10, 7), (11, 1), (14, 6), (12, 11)):
        a = list(base)
        a[out] = a[other]
        assert back(a) == UNSUPPORTED, (out, other)


def test_hook_is_cleared_by_refused_calls():
    lib = carve.load_library()
    arr = (ctypes.c_void_p * 2)(4096, 4096)
    for call in (lambda: fwd(gdims(B=0)), lambda: lib.carve_block_norm_fwd(ctypes.byref(ndims(rows=0)), *far(8), None)):
        assert lib.carve_profile_events(arr, 2) == 0
        assert call() == SHAPE
        assert lib.carve_profile_events(None, 0) == 0


def test_binding_refuses_host_tensors():
    x = torch.zeros(1, 4, 1, 32)
    g = torch.zeros(1, 4, 1)
    with pytest.raises(TypeError):
        carve.gdr_chunk_fwd(x, x, x, g, g)
    with pytest.raises(TypeError):
        carve.gdr_step(x, x, x, g, g, torch.zeros(1, 1, 32, 32))
    with pytest.raises(TypeError):
        carve.block_norm_fwd(torch.zeros(2, 64), torch.ones(64))
