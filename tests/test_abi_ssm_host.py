"""Host-side refusals of the short convolution, rotary positions and the state space scan (no
GPU needed): sizes, strides, alignment, missing and conflicting arguments, workspaces and
overlapping tensors are rejected before any HIP call."""
import ctypes

import pytest
import torch

from paper_2606_27229_amd import carve

OK, NULL, SHAPE, UNSUPPORTED, ALIGN, WORKSPACE, ARG = 0, -1, -2, -3, -4, -5, -7
BIG = 1 << 62


def far(n):
    """Distinct addresses far apart; never dereferenced."""
    return [ctypes.c_void_p(1 << 40 | i << 34) for i in range(n)]


# ---- the short convolution ----


def cdims(**kw):
    d = dict(B=2, T=100, N=0, C=64, W=4, dtype=carve.CARVE_BF16, activation=1)
    d.update({k: v for k, v in kw.items() if k in d})
    d["x_batch"], d["x_token"] = kw.get("x_batch", d["T"] * d["C"]), kw.get("x_token", d["C"])
    return carve.ShortConvDims(*(d[f] for f, _ in carve.ShortConvDims._fields_))


def conv(d, which="fwd", args=None, ws=BIG, pool=8):
    lib = carve.load_library()
    if which == "fwd":     # x weight bias x0 offsets y x_T
        a = args or far(7)
        if args is None and d.N == 0:
            a[4] = None
        return lib.carve_short_conv_fwd(ctypes.byref(d), *a, None)
    if which == "bwd":     # x weight bias x0 offsets dy dx_T dx dweight dbias dx0 workspace
        a = args or far(12)
        if args is None and d.N == 0:
            a[4] = None
        return lib.carve_short_conv_bwd(ctypes.byref(d), *a, ws, None)
    a = args or far(6)     # x weight bias slots | state y
    return lib.carve_short_conv_step(ctypes.byref(d), *a[:4], pool, *a[4:], None)


@pytest.mark.parametrize("kw,status", [
    (dict(B=0), SHAPE), (dict(T=0), SHAPE), (dict(N=-1), SHAPE), (dict(N=3), SHAPE), (dict(C=0), SHAPE), (dict(W=0), SHAPE),
    (dict(W=1), UNSUPPORTED), (dict(W=5), UNSUPPORTED), (dict(C=60), UNSUPPORTED), (dict(C=1 << 20), UNSUPPORTED),
    (dict(dtype=7), UNSUPPORTED), (dict(activation=2), ARG), (dict(activation=-1), ARG), (dict(x_token=-64), ARG),
    (dict(x_token=66), ALIGN), (dict(x_batch=4), ALIGN), (dict(x_batch=1 << 46), UNSUPPORTED),
    (dict(B=1 << 15, T=1 << 16), UNSUPPORTED)])
def test_conv_dims(kw, status):
    d = cdims(**kw)
    for which in ("fwd", "bwd", "step"):
        assert conv(d, which) == status
    assert carve.load_library().carve_short_conv_workspace_size(ctypes.byref(d)) == 0


def test_conv_arguments():
    d, p = cdims(), cdims(B=1, N=3)
    for which, count, needed in (("fwd", 7, (0, 1, 5)), ("bwd", 12, (0, 1, 5, 7, 8)), ("step", 6, (0, 1, 4, 5))):
        for i in needed:
            a = far(count)
            if which != "step":
                a[4] = None
            a[i] = None
            assert conv(d, which, a) == NULL, (which, i)
        for i in range(count):
            if which == "step" and i == 3:
                continue   # (slots: four bytes)
            a = far(count)
            if which != "step":
                a[4] = None if i != 4 else a[4]
            a[i] = ctypes.c_void_p((1 << 41) + 8)
            assert conv(p if i == 4 and which != "step" else d, which, a) in (ALIGN, ARG), (which, i)
    a = far(7)
    assert conv(d, "fwd", a) == ARG                       # offsets without N
    a[4] = None
    assert conv(p, "fwd", a) == NULL                      # N without offsets
    a = far(12)
    a[4] = a[9] = None
    assert conv(d, "bwd", a) == ARG                       # bias without dbias
    a = far(12)
    a[4] = a[11] = None
    assert conv(d, "bwd", a) == WORKSPACE
    a = far(12)
    a[4] = None
    need = carve.load_library().carve_short_conv_workspace_size(ctypes.byref(d))
    assert need > 0 and conv(d, "bwd", a, need - 1) == WORKSPACE
    assert conv(cdims(B=1, N=2), "step") == SHAPE and conv(d, "step", pool=0) == SHAPE
    a = far(6)
    a[3] = None
    assert conv(d, "step", a, pool=1) == SHAPE            # a state a sequence without slots
    assert conv(cdims(B=65536, T=1), "step") == UNSUPPORTED


def test_conv_overlaps():
    d = cdims()
    for out, other in ((5, 0), (5, 3), (6, 0), (6, 5), (5, 1)):
        a = far(7)
        a[4] = None
        a[out] = a[other]
        assert conv(d, "fwd", a) == UNSUPPORTED, (out, other)
    for out, other in ((7, 0), (7, 5), (8, 1), (10, 3), (11, 7), (10, 6)):
        a = far(12)
        a[4] = None
        a[out] = a[other]
        assert conv(d, "bwd", a) == UNSUPPORTED, (out, other)
    a = far(6)
    a[5] = a[0]
    assert conv(d, "step", a) == UNSUPPORTED


# ---- rotary positions ----


def rdims(**kw):
    d = dict(B=2, T=50, N=0, Hq=4, Hk=2, D=64, rot=32, dtype=carve.CARVE_BF16, interleaved=0, amplitude=1.0)
    d.update({k: v for k, v in kw.items() if k in d})
    for n, h in (("q", d["Hq"]), ("k", d["Hk"]), ("qo", d["Hq"]), ("ko", d["Hk"])):
        for what, v in (("batch", d["T"] * h * d["D"]), ("token", h * d["D"]), ("head", d["D"])):
            d[f"{n}_{what}"] = kw.get(f"{n}_{what}", v)
    return carve.RotaryDims(*(d[f] for f, _ in carve.RotaryDims._fields_))


def rot(d, a=None):
    """a: q k freq positions start offsets q_out k_out"""
    if a is None:
        a = far(8)
        a[3] = None
        if d.N == 0:
            a[5] = None
        if d.Hk == 0:
            a[1] = a[7] = None
    return carve.load_library().carve_rotary(ctypes.byref(d), *a[:6], 0, *a[6:], None)


@pytest.mark.parametrize("kw,status", [
    (dict(B=0), SHAPE), (dict(T=0), SHAPE), (dict(N=2), SHAPE), (dict(Hq=0), SHAPE), (dict(Hk=-1), SHAPE), (dict(D=0), SHAPE),
    (dict(rot=0), SHAPE), (dict(rot=80), SHAPE), (dict(rot=24), UNSUPPORTED), (dict(D=68), UNSUPPORTED), (dict(D=2048), UNSUPPORTED),
    (dict(Hq=65535, Hk=1), UNSUPPORTED), (dict(dtype=3), UNSUPPORTED), (dict(amplitude=float("nan")), ARG),
    (dict(amplitude=float("inf")), ARG), (dict(q_token=-256), ARG), (dict(ko_head=68), ALIGN), (dict(k_batch=1 << 46), UNSUPPORTED),
    (dict(qo_token=0), ARG), (dict(qo_head=32), ARG), (dict(ko_batch=64), ARG)])
def test_rotary_dims(kw, status):
    assert rot(rdims(**kw)) == status


def test_rotary_arguments():
    d = rdims()
    base = far(8)
    base[3] = base[5] = None
    for i in (0, 1, 2, 6, 7):
        a = list(base)
        a[i] = None
        assert rot(d, a) == NULL
        a[i] = ctypes.c_void_p((1 << 41) + 8)
        assert rot(d, a) == ALIGN
    for extra in (4, 5):                                  # positions and a start, or offsets
        a = far(8)
        a[9 - extra] = None
        assert rot(d, a) == ARG
    a = list(base)
    a[5] = far(8)[5]
    assert rot(d, a) == ARG                               # offsets without N
    assert rot(rdims(B=1, N=2), base) == NULL             # N without offsets
    a = list(base)
    assert rot(rdims(Hk=0), a) == ARG                     # keys without heads


def test_rotary_places():
    d = rdims()
    base = far(8)
    base[3] = base[5] = None
    a = list(base)
    a[6] = a[0]
    assert rot(d, a) == ARG                               # one in place, the other not
    a = list(base)
    a[6], a[7] = a[0], a[1]
    a[2] = a[0]
    assert rot(d, a) == UNSUPPORTED                       # frequencies within the output
    a = list(base)
    a[6], a[7] = a[0], a[1]
    assert rot(rdims(q_token=512, q_batch=512 * 50), a) == ARG   # in place with other strides
    for out, other in ((6, 1), (7, 0), (6, 4), (7, 6)):
        a = list(base)
        a[out] = a[other]
        assert rot(d, a) == UNSUPPORTED, (out, other)
    # queries' and keys' outputs in one tensor's rows, but not on each other
    wide = dict(qo_token=384, qo_batch=384 * 50, ko_token=384, ko_batch=384 * 50)
    for off, status in ((128, UNSUPPORTED), (320, UNSUPPORTED)):
        a = list(base)
        a[7] = ctypes.c_void_p(a[6].value + 2 * off)
        assert rot(rdims(**wide), a) == status


# ---- the state space scan ----


def sdims(**kw):
    d = dict(B=2, T=100, N=0, G=2, H=4, P=64, S=64, dtype=carve.CARVE_BF16, softplus=1)
    d.update({k: v for k, v in kw.items() if k in d})
    for n, h, w in (("x", d["H"], d["P"]), ("b", d["G"], d["S"]), ("c", d["G"], d["S"])):
        last = "head" if n == "x" else "group"
        for what, v in (("batch", d["T"] * h * w), ("token", h * w), (last, w)):
            d[f"{n}_{what}"] = kw.get(f"{n}_{what}", v)
    d["dt_batch"], d["dt_token"] = kw.get("dt_batch", d["T"] * d["H"]), kw.get("dt_token", d["H"])
    return carve.SsmDims(*(d[f] for f, _ in carve.SsmDims._fields_))


def ssm(d, which="fwd", args=None, ws=BIG, pool=8):
    lib = carve.load_library()
    if which == "fwd":   # x dt A Bm Cm D dt_bias S0 offsets y S_T S_chunks workspace
        a = args or far(13)
        if args is None and d.N == 0:
            a[8] = None
        return lib.carve_ssm_chunk_fwd(ctypes.byref(d), *a, ws, None)
    if which == "bwd":   # x dt A Bm Cm D dt_bias S_chunks offsets dy dS_T dx ddt dA dBm dCm dD ddt_bias dS0 workspace
        a = args or far(20)
        if args is None and d.N == 0:
            a[8] = None
        return lib.carve_ssm_chunk_bwd(ctypes.byref(d), *a, ws, None)
    a = args or far(10)  # x dt A Bm Cm D dt_bias slots | state y
    return lib.carve_ssm_step(ctypes.byref(d), *a[:8], pool, *a[8:], None)


@pytest.mark.parametrize("kw,status", [
    (dict(B=0), SHAPE), (dict(T=0), SHAPE), (dict(N=-1), SHAPE), (dict(N=3), SHAPE), (dict(G=0), SHAPE), (dict(P=0), SHAPE),
    (dict(S=48), UNSUPPORTED), (dict(S=256), UNSUPPORTED), (dict(P=48), UNSUPPORTED), (dict(P=288), UNSUPPORTED),
    (dict(G=3), UNSUPPORTED), (dict(G=1, H=65536), UNSUPPORTED), (dict(dtype=5), UNSUPPORTED), (dict(x_token=-256), ARG),
    (dict(b_token=66), ALIGN), (dict(c_group=4), ALIGN), (dict(dt_token=-1), ARG), (dict(x_token=1 << 23), UNSUPPORTED),
    (dict(x_batch=1 << 46), UNSUPPORTED), (dict(dt_batch=1 << 46), UNSUPPORTED), (dict(B=1 << 15, T=1 << 16), UNSUPPORTED)])
def test_ssm_dims(kw, status):
    lib, d = carve.load_library(), sdims(**kw)
    for which in ("fwd", "bwd", "step"):
        assert ssm(d, which) == status
    assert lib.carve_ssm_chunk_count(ctypes.byref(d)) == 0
    assert lib.carve_ssm_workspace_size(ctypes.byref(d), 0) == 0 and lib.carve_ssm_workspace_size(ctypes.byref(d), 1) == 0


def test_ssm_calls_beyond_a_launch():
    """2^32 threads or more of a kernel are refused, not left to the launch."""
    for kw in (dict(B=1, N=1 << 23, T=64), dict(B=1 << 15, T=64 * 256), dict(B=1, N=1 << 20, T=64, H=8, G=1, P=256)):
        d = sdims(**kw)
        assert ssm(d) == UNSUPPORTED and ssm(d, "bwd") == UNSUPPORTED


def test_ssm_most_chunks():
    """The gradients run 768 threads a chunk: at most 5 * 2^20 of them."""
    lib, one = carve.load_library(), dict(B=1, T=64, G=1, H=1, P=32, S=32)
    for n, fits in (((5 << 20) - 2, True), (5 << 20, False), (6 << 20, False)):
        d = sdims(N=n, **one)
        assert (lib.carve_ssm_chunk_count(ctypes.byref(d)) > 0) == fits
        if not fits:
            assert ssm(d) == UNSUPPORTED and ssm(d, "bwd") == UNSUPPORTED


def test_ssm_sizes():
    lib = carve.load_library()
    count = lambda **kw: lib.carve_ssm_chunk_count(ctypes.byref(sdims(**kw)))
    assert count() == 2 * 2 and count(T=64) == 2 and count(T=1) == 2
    assert count(B=1, N=3) == 1 + 3 and count(B=1, N=1, T=64) == 2


def test_ssm_arguments():
    d, p = sdims(), sdims(B=1, N=3)
    for which, count, needed in (("fwd", 13, (0, 1, 2, 3, 4, 9)), ("bwd", 20, (0, 1, 2, 3, 4, 7, 9, 11, 12, 13, 14, 15)),
                                 ("step", 10, (0, 1, 2, 3, 4, 8, 9))):
        for i in needed:
            a = far(count)
            if which != "step":
                a[8] = None
            a[i] = None
            assert ssm(d, which, a) == NULL, (which, i)
        for i in range(count):
            a = far(count)
            if which != "step" and i != 8:
                a[8] = None
            a[i] = ctypes.c_void_p((1 << 46) + 1)   # (dt and what is one value a head: whole elements)
            assert ssm(p if i == 8 and which != "step" else d, which, a) in (ALIGN, ARG), (which, i)
    a = far(13)
    assert ssm(d, "fwd", a) == ARG                        # offsets without N
    a[8] = None
    assert ssm(p, "fwd", a) == NULL                       # N without offsets
    for i in (16, 17):                                    # D without dD, dt_bias without its gradient
        a = far(20)
        a[8] = a[i] = None
        assert ssm(d, "bwd", a) == ARG
    lib = carve.load_library()
    for which, count, back in (("fwd", 13, 0), ("bwd", 20, 1)):
        a = far(count)
        a[8] = None
        need = lib.carve_ssm_workspace_size(ctypes.byref(d), back)
        assert need > 0 and ssm(d, which, a, need - 1) == WORKSPACE
        a[-1] = None
        assert ssm(d, which, a) == WORKSPACE
    assert ssm(p, "step") == SHAPE and ssm(d, "step", pool=0) == SHAPE
    a = far(10)
    a[7] = None
    assert ssm(d, "step", a, pool=1) == SHAPE
    assert ssm(sdims(B=65536, T=1), "step") == UNSUPPORTED


def test_ssm_overlaps():
    d = sdims()
    for out, other in ((9, 0), (10, 7), (11, 10), (12, 9), (9, 1)):
        a = far(13)
        a[8] = None
        a[out] = a[other]
        assert ssm(d, "fwd", a) == UNSUPPORTED, (out, other)
    for out, other in ((11, 0), (11, 9), (12, 1), (18, 10), (14, 3), (19, 7), (13, 2), (16, 17)):
        a = far(20)
        a[8] = None
        a[out] = a[other]
        assert ssm(d, "bwd", a) == UNSUPPORTED, (out, other)
    a = far(10)
    a[9] = a[0]
    assert ssm(d, "step", a) == UNSUPPORTED


# ---- the frequencies ----


def test_frequencies():
    f = carve.rotary_frequencies(8, 10000.0, device="cpu")
    assert f.dtype == torch.float64 and torch.allclose(f, torch.tensor([1.0, 0.1, 0.01, 0.001], dtype=torch.float64), rtol=1e-14)
    assert torch.equal(carve.rotary_frequencies(8, stretch=4.0, device="cpu"), f / 4)
    # turns in a context of 1000: 159, 15.9, 1.59, 0.159; below 1 all is stretched, above 30 nothing
    g = carve.rotary_frequencies(8, stretch=4.0, low=1, high=30, length=1000, device="cpu")
    assert g[0] == f[0] and torch.isclose(g[3], f[3] / 4, rtol=1e-14)
    part = 1 - (1000 * 0.1 / (2 * torch.pi) - 1) / 29
    assert torch.isclose(g[1], f[1] * (1 - part) + f[1] / 4 * part, rtol=1e-12)
    for bad in (dict(rot=7), dict(rot=0), dict(rot=8, low=1), dict(rot=8, low=2, high=1, length=10)):
        with pytest.raises(ValueError):
            carve.rotary_frequencies(device="cpu", **bad)
