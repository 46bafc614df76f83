"""The gated delta rule (chunked forward and backward, recurrent step) against its
token-by-token definition in 64 bits.

Tolerances (relative 2-norms), from the arithmetic:
  bf16 outputs (o, dq, dk, dv, dbeta): one rounding, at most eps / 2 = 2^-8 of every
    value, and f32 intermediates as below, far smaller: 2^-8.
  f32 tokens: f32 products, sums of up to 64 + 128 terms and the triangular inverse
    of 64 steps, all errors 2^-24 of a term: 192 * 2^-24 = 1.2e-5.
  f32 outputs of bf16 tokens (S_T, dS0, dg): each f32 intermediate enters the matrix
    cores as three bf16 values, which hold its 24 bits, and a product leaves out pairs
    of pieces of 2^-24 together: the f32 bound.
dg and dbeta are sums of terms that cancel: their error is measured against the
2-norm of the result as well, with a factor 4 for the cancellation.
"""
import pytest
import torch

from paper_2606_27229_amd import carve
from tests.gdr_util import cuda, gdr_inputs, gdr_reference, rel

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


def tolerance(name, dtype):
    cancel = 4 if name in ("dg", "dbeta") else 1
    if dtype == F32 or name in ("S_T", "dS0", "dg"):
        return 1.2e-5 * cancel
    return 2.0 ** -8


def compare(got, ref, dtype, names):
    errs = {n: rel(got[n], ref[n]) for n in names}
    print("rel errors:", {n: float("%.2g" % e) for n, e in errs.items()}, flush=True)
    for n in names:
        assert torch.isfinite(got[n].float()).all(), n
        assert errs[n] <= tolerance(n, dtype), (n, errs[n])


def run(x, offsets=None, backward=True, **kw):
    o, S_T, S_c = carve.gdr_chunk_fwd(x["q"], x["k"], x["v"], x["g"], x["beta"], x["S0"], scale=x["scale"],
                                      offsets=offsets, **kw)
    got = {"o": o, "S_T": S_T}
    if backward:
        got.update(carve.gdr_chunk_bwd(x["q"], x["k"], x["v"], x["g"], x["beta"], S_c, x["dO"], x["dS_T"],
                                       scale=x["scale"], offsets=offsets))
    torch.cuda.synchronize()
    return got


FWD = ("o", "S_T")
ALL = ("o", "S_T", "dq", "dk", "dv", "dg", "dbeta", "dS0")


@pytest.mark.parametrize("B,T,Hk,Hv,Dk,Dv,dtype", [
    (1, 1, 1, 1, 32, 32, F32), (1, 64, 1, 1, 64, 64, F32), (2, 65, 2, 4, 32, 64, F32), (1, 130, 1, 2, 128, 128, F32),
    (2, 200, 4, 4, 64, 32, F32), (1, 100, 1, 3, 64, 256, F32),
    (1, 1, 1, 1, 32, 32, BF), (1, 15, 1, 1, 128, 128, BF), (1, 64, 1, 1, 128, 128, BF), (2, 63, 2, 2, 64, 64, BF),
    (2, 129, 2, 6, 128, 64, BF), (3, 190, 3, 3, 32, 128, BF), (1, 321, 1, 4, 128, 256, BF), (1, 257, 9, 9, 64, 128, BF),
])
def test_chunks(B, T, Hk, Hv, Dk, Dv, dtype):
    print(f"case chunks B={B} T={T} Hk={Hk} Hv={Hv} Dk={Dk} Dv={Dv} {dtype}", flush=True)
    x = gdr_inputs(B, T, Hk, Hv, Dk, Dv, dtype, seed=B + T + Hk + Hv + Dk + Dv)
    compare(run(cuda(x)), gdr_reference(x), dtype, ALL)


@pytest.mark.parametrize("Hk,Hv,Dk,Dv,dtype", [(80, 80, 64, 128, BF), (16, 80, 128, 128, BF), (80, 80, 64, 128, F32),
                                               (40, 40, 128, 256, F32)])
def test_many_heads(Hk, Hv, Dk, Dv, dtype):
    """More value tiles than the chains run at once (four tiles a workgroup backward)."""
    print(f"case many heads Hk={Hk} Hv={Hv} Dk={Dk} Dv={Dv} {dtype}", flush=True)
    x = gdr_inputs(1, 130, Hk, Hv, Dk, Dv, dtype, seed=Hk + Hv)
    compare(run(cuda(x)), gdr_reference(x), dtype, ALL)


@pytest.mark.parametrize("Hk,Hv,Dk,Dv,dtype", [(20, 20, 64, 256, F32), (40, 40, 64, 128, BF), (10, 20, 128, 256, BF), (33, 33, 128, 128, F32),
                                               (16, 16, 128, 256, BF), (17, 17, 64, 256, F32)])
def test_heads_between(Hk, Hv, Dk, Dv, dtype):
    """256 value tiles, a tile a workgroup, and a few more, two."""
    print(f"case heads Hk={Hk} Hv={Hv} Dk={Dk} Dv={Dv} {dtype}", flush=True)
    x = gdr_inputs(1, 200, Hk, Hv, Dk, Dv, dtype, seed=Hk + Dk)
    compare(run(cuda(x)), gdr_reference(x), dtype, ALL)


LENGTHS = [[0, 1, 64, 0, 65, 130, 1], [63], [1, 0, 0], [128, 64, 7]]


@pytest.mark.parametrize("lens", LENGTHS)
@pytest.mark.parametrize("Hk,Hv,Dk,Dv,dtype,first,behind", [(1, 2, 64, 64, F32, 0, 0), (2, 4, 128, 64, BF, 5, 3),
                                                            (3, 3, 32, 128, BF, 0, 70)])
def test_packed(lens, Hk, Hv, Dk, Dv, dtype, first, behind):
    """Packed sequences, empty and one-token ones among them; rows before the first and
    behind the last sequence are left as they were, in every output."""
    print(f"case packed {lens} Hk={Hk} Hv={Hv} Dk={Dk} Dv={Dv} {dtype} first={first} behind={behind}", flush=True)
    T = first + sum(lens) + behind
    x = gdr_inputs(1, T, Hk, Hv, Dk, Dv, dtype, seed=T + Dk, seqs=len(lens))
    for n in ("q", "k", "v", "g", "beta", "dO"):     # what lies outside is not used
        x[n][:, :first] = float("nan")
        x[n][:, T - behind:] = float("nan")
    inside = {n: (torch.nan_to_num(t) if isinstance(t, torch.Tensor) else t) for n, t in x.items()}
    inside["first"] = first
    ref = gdr_reference(inside, lens)
    d = cuda(x)
    ends = torch.tensor([first] + lens).cumsum(0)
    off = ends.to(torch.int32).cuda()
    shapes = {"dq": x["q"], "dk": x["k"], "dv": x["v"], "dg": x["g"], "dbeta": x["beta"]}
    out = {"o": torch.full_like(d["v"], 7.0)}
    bout = {n: torch.full_like(t.cuda(), 7.0) for n, t in shapes.items()}
    o, S_T, S_c = carve.gdr_chunk_fwd(d["q"], d["k"], d["v"], d["g"], d["beta"], d["S0"], scale=x["scale"], offsets=off, out=out)
    got = {"o": o, "S_T": S_T}
    got.update(carve.gdr_chunk_bwd(d["q"], d["k"], d["v"], d["g"], d["beta"], S_c, d["dO"], d["dS_T"], scale=x["scale"],
                                   offsets=off, out=bout))
    torch.cuda.synchronize()
    for n in ("o", "dq", "dk", "dv", "dg", "dbeta"):
        assert (got[n][:, :first] == 7).all() and (got[n][:, T - behind:] == 7).all(), n
        got[n][:, :first] = 0
        got[n][:, T - behind:] = 0
    compare(got, ref, dtype, ALL)
    for i, n in enumerate(lens):                     # the state of an empty sequence passes through
        if n == 0:
            assert torch.equal(got["S_T"][i], d["S0"][i]) and torch.equal(got["dS0"][i], d["dS_T"][i])


@pytest.mark.parametrize("nseq,Hk,Hv,Dk,Dv,dtype", [(64, 1, 2, 64, 64, BF), (65, 1, 2, 64, 64, BF), (70, 2, 16, 64, 64, BF),
                                                    (63, 17, 17, 64, 64, F32), (5, 32, 32, 128, 256, BF)])
def test_many_sequences(nseq, Hk, Hv, Dk, Dv, dtype):
    """Up to 64 sequences are taken longest first, more as they come; beyond 4096 value tiles
    the backward runs four a workgroup.  Lengths of every order, many of them equal."""
    print(f"case many sequences {nseq} Hk={Hk} Hv={Hv} Dk={Dk} Dv={Dv} {dtype}", flush=True)
    lens = [(0, 1, 65, 5, 130, 2)[(5 * i * i + i) % 6] if i % 9 else 70 for i in range(nseq)]
    x = gdr_inputs(1, sum(lens), Hk, Hv, Dk, Dv, dtype, seed=nseq, seqs=nseq)
    off = torch.tensor([0] + lens).cumsum(0).to(torch.int32).cuda()
    compare(run(cuda(x), off), gdr_reference(x, lens), dtype, ALL)


def test_offsets_outside_the_contract_stay_inside_the_tensors():
    """Decreasing, negative and too large offsets: the call returns, and what lies around
    the outputs keeps its values."""
    x = cuda(gdr_inputs(1, 200, 1, 2, 64, 64, BF, seed=3, seqs=4))
    for offs in ([0, 150, 50, 500, -7], [300, 10, 0, 0, 200], [-5, -4, 1 << 30, 3, 2]):
        off = torch.tensor(offs, dtype=torch.int32).cuda()
        guard = torch.full((3, 200, 2, 64), 5.0, dtype=BF, device="cuda")
        o, S_T, S_c = carve.gdr_chunk_fwd(x["q"], x["k"], x["v"], x["g"], x["beta"], x["S0"], offsets=off, out={"o": guard[1:2]})
        carve.gdr_chunk_bwd(x["q"], x["k"], x["v"], x["g"], x["beta"], S_c, x["dO"], x["dS_T"], offsets=off)
        torch.cuda.synchronize()
        assert (guard[0] == 5).all() and (guard[2] == 5).all()


@pytest.mark.parametrize("dtype", [F32, BF])
def test_strided_inputs(dtype):
    """q, k, v as slices of one projection, and queries shared by all heads (stride 0)."""
    B, T, H, Dk, Dv = 2, 100, 3, 64, 32
    x = gdr_inputs(B, T, H, H, Dk, Dv, dtype, seed=11)
    x["q"] = x["q"][:, :, :1].expand(B, T, H, Dk).clone()
    ref = gdr_reference(x)
    d = cuda(x)
    fused = torch.cat([d["k"].flatten(2), d["v"].flatten(2), d["q"][:, :, 0]], -1)
    d["k"] = fused[..., :H * Dk].unflatten(-1, (H, Dk))
    d["v"] = fused[..., H * Dk:H * (Dk + Dv)].unflatten(-1, (H, Dv))
    d["q"] = fused[..., None, H * (Dk + Dv):].expand(B, T, H, Dk)
    assert not d["k"].is_contiguous() and d["q"].stride(2) == 0
    compare(run(d), ref, dtype, ALL)


def test_rows_far_apart():
    """Rows whose offsets pass 32 bits."""
    T, H, D, width = 300, 1, 32, (1 << 23) - 64
    x = gdr_inputs(1, T, H, H, D, D, BF, seed=12)
    ref = gdr_reference(x)
    d = cuda(x)
    base = torch.zeros(T * width + 64, dtype=BF, device="cuda")
    assert T * width > 1 << 31
    far = base.as_strided((1, T, H, D), (0, width, D, 1))
    far.copy_(d["k"])
    d["k"] = far
    compare(run(d), ref, BF, ALL)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("kind", ["resets", "hard", "none", "mixed", "masked", "same_keys", "scale"])
def test_decays_and_masks(kind, dtype):
    """Decays of 0 (g = -inf), decays that leave a state only a token, none at all, hard
    ones before soft ones in one chunk, tokens taken out by beta = 0 and g = 0, equal keys
    with full write strength, and a scale of its own.  Under hard decays dg is small
    against what it is summed from in the definition, not in the kernels: same bounds."""
    print(f"case decays {kind} {dtype}", flush=True)
    x = gdr_inputs(1, 150, 2, 2, 64, 64, dtype, seed=21)
    if kind == "resets":
        x["g"][:, ::7] = float("-inf")
        x["g"][:, 64] = float("-inf")
    elif kind == "hard":
        x["g"] -= 12
    elif kind == "none":
        x["g"] *= 0
    elif kind == "mixed":
        x["g"][:, :40] -= 60
        x["g"][:, 70:100] -= 300
    elif kind == "masked":
        x["beta"][:, 20:90] = 0
        x["g"][:, 20:90] = 0
    elif kind == "same_keys":
        x["k"][:] = x["k"][:, :1]
        x["beta"][:] = 1
    elif kind == "scale":
        x["scale"] = -3.5
    ref_x = dict(x, g=x["g"].clamp(min=-1e4))   # (e^-1e4 is 0 in 64 bits too; -inf * 0 is not)
    compare(run(cuda(x)), gdr_reference(ref_x), dtype, ALL)


def test_optional_arguments():
    x = gdr_inputs(2, 70, 1, 2, 64, 64, BF, seed=31, state=False, dst=False)
    ref = gdr_reference(x)
    d = cuda(x)
    o, S_T, S_c = carve.gdr_chunk_fwd(d["q"], d["k"], d["v"], d["g"], d["beta"], want_chunks=False, want_state=False)
    assert S_T is None and S_c is None and rel(o, ref["o"]) <= 2.0 ** -8
    _, _, S_c = carve.gdr_chunk_fwd(d["q"], d["k"], d["v"], d["g"], d["beta"])
    got = carve.gdr_chunk_bwd(d["q"], d["k"], d["v"], d["g"], d["beta"], S_c, d["dO"], want_dS0=False)
    assert "dS0" not in got
    compare(dict(got, o=o), ref, BF, ("o", "dq", "dk", "dv", "dg", "dbeta"))
    ws = torch.full((1 << 26,), 255, dtype=torch.uint8, device="cuda")     # NaN everywhere
    again = carve.gdr_chunk_bwd(d["q"], d["k"], d["v"], d["g"], d["beta"], S_c, d["dO"], want_dS0=False, workspace=ws)
    for n in got:
        assert torch.equal(got[n], again[n]), n


@pytest.mark.parametrize("dtype,D", [(F32, 64), (BF, 128)])
def test_reruns_are_bitwise_identical(dtype, D):
    x = cuda(gdr_inputs(2, 333, 2, 8, D, D, dtype, seed=41))
    first = run(x)
    for _ in range(5):
        again = run(x)
        for n in first:
            assert torch.equal(first[n], again[n]), n


@pytest.mark.parametrize("name", ["q", "k", "v", "g", "beta", "S0"])
def test_gradients_against_differences(name):
    """<gradient, d> against central differences of the f32 forward along d.  With steps
    of 2^-7 of a unit direction's size the differences' own error (third derivatives) is
    below 1e-3 of the value and the forward's rounding, 1e-6 of the loss over 2^-6, below
    1e-3 of the typical slope; 5e-3 of the largest slope leaves room for small ones."""
    x = cuda(gdr_inputs(1, 97, 2, 4, 64, 64, F32, seed=51))
    got = run(x)
    gen = torch.Generator(device="cuda").manual_seed(52)
    slopes = []
    for _ in range(4):
        d = torch.randn(x[name].shape, generator=gen, device="cuda")
        d = d / d.norm() * max(1.0, float(x[name].norm()) / 8)
        loss = []
        for sign in (1, -1):
            y = dict(x)
            y[name] = x[name] + sign * 2.0 ** -7 * d
            r = run(y, backward=False)
            loss.append((r["o"].double() * x["dO"]).sum() + (r["S_T"].double() * x["dS_T"]).sum())
        slopes.append((float((loss[0] - loss[1]) / 2.0 ** -6), float((got["d" + name].double() * d).sum())))
    print(name, slopes, flush=True)
    most = max(abs(b) for _, b in slopes)
    for a, b in slopes:
        assert abs(a - b) <= 5e-3 * most, (name, slopes)


# ---- the recurrent form ------------------------------------------------------------------


@pytest.mark.parametrize("B,T,Hk,Hv,Dk,Dv,dtype,pool", [
    (1, 1, 1, 1, 32, 32, F32, 1), (3, 1, 2, 4, 64, 64, BF, 5), (2, 5, 3, 3, 128, 128, BF, 2), (4, 2, 1, 3, 128, 256, F32, 9),
    (2, 1, 1, 2, 32, 256, BF, 4), (5, 8, 2, 2, 64, 32, F32, 6),
])
def test_step(B, T, Hk, Hv, Dk, Dv, dtype, pool):
    """f32 arithmetic over at most 128 keys and T tokens: 128 T 2^-24, and the output's
    rounding; states no sequence owns and padding entries keep their values."""
    print(f"case step B={B} T={T} Hk={Hk} Hv={Hv} Dk={Dk} Dv={Dv} {dtype} pool={pool}", flush=True)
    x = gdr_inputs(B, T, Hk, Hv, Dk, Dv, dtype, seed=B + T + Dk)
    gen = torch.Generator().manual_seed(5)
    state = 0.3 * torch.randn(pool, Hv, Dv, Dk, generator=gen)
    order = torch.randperm(pool, generator=gen)[:B]
    x["S0"] = state[order]
    ref = gdr_reference(x, grads=False)
    d = cuda(x)
    st = state.cuda()
    # one padding entry each with a negative and a too large slot
    pad = lambda t: torch.cat([t, t[:1], t[:1]])
    slots = torch.cat([order, torch.tensor([-1, pool])]).to(torch.int32).cuda()
    out = torch.full((B + 2, T, Hv, Dv), 7.0, dtype=dtype, device="cuda")
    o = carve.gdr_step(*(pad(d[n]) for n in ("q", "k", "v", "g", "beta")), st, slots, scale=x["scale"], out=out)
    torch.cuda.synchronize()
    tol = 128 * T * 2.0 ** -24
    assert (o[B:] == 7).all()
    assert rel(o[:B], ref["o"]) <= (tol if dtype == F32 else 2.0 ** -8 + tol)
    assert rel(st[order.cuda()], ref["S_T"]) <= tol
    rest = [i for i in range(pool) if i not in order.tolist()]
    assert torch.equal(st[rest].cpu(), state[rest])
    # without slots
    st2 = x["S0"].cuda()
    o2 = carve.gdr_step(d["q"], d["k"], d["v"], d["g"], d["beta"], st2, scale=x["scale"])
    assert torch.equal(o2, o[:B]) and torch.equal(st2, st[order.cuda()])


def test_scale_given_as_a_tensor_is_read_at_every_call():
    x = cuda(gdr_inputs(2, 1, 2, 2, 64, 64, F32, seed=63))
    scale = torch.tensor(1.0)
    for value in (1.0, 0.5):
        scale.fill_(value)
        got, want = (carve.gdr_step(x["q"], x["k"], x["v"], x["g"], x["beta"], x["S0"].clone(), scale=s) for s in (scale, value))
        assert torch.equal(got, want)


def test_step_far_slot():
    """A slot whose state lies past 2^31 elements."""
    H, D = 32, 128
    pool = (1 << 31) // (H * D * D) + 3
    x = gdr_inputs(1, 1, H, H, D, D, BF, seed=61)
    ref = gdr_reference(x, grads=False)
    d = cuda(x)
    st = torch.zeros(pool, H, D, D, device="cuda")
    st[pool - 1] = d["S0"][0]
    o = carve.gdr_step(d["q"], d["k"], d["v"], d["g"], d["beta"], st, torch.tensor([pool - 1], dtype=torch.int32).cuda(),
                       scale=x["scale"])
    assert rel(o, ref["o"]) <= 2.0 ** -8 and rel(st[pool - 1:], ref["S_T"]) <= 1e-5
    assert not st[:pool - 1].any()


def test_prefill_then_steps():
    """A prompt in chunks, then tokens one by one on the state it left, against the whole
    sequence at once."""
    x = gdr_inputs(2, 90, 2, 4, 128, 128, BF, seed=71)
    ref = gdr_reference(x, grads=False)
    d = cuda(x)
    part = lambda a, b: [d[n][:, a:b].contiguous() for n in ("q", "k", "v", "g", "beta")]
    o, S, _ = carve.gdr_chunk_fwd(*part(0, 77), d["S0"], want_chunks=False)
    outs = [o]
    for t in range(77, 90):
        outs.append(carve.gdr_step(*part(t, t + 1), S))
    assert rel(torch.cat(outs, 1), ref["o"]) <= 2.0 ** -8
    assert rel(S, ref["S_T"]) <= 1.2e-5


# ---- streams and graphs -------------------------------------------------------------------


def test_on_another_stream():
    x = cuda(gdr_inputs(2, 300, 2, 2, 64, 64, BF, seed=81))
    ref = run(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    o, S_T, S_c = carve.gdr_chunk_fwd(x["q"], x["k"], x["v"], x["g"], x["beta"], x["S0"], scale=x["scale"], stream=side)
    got = carve.gdr_chunk_bwd(x["q"], x["k"], x["v"], x["g"], x["beta"], S_c, x["dO"], x["dS_T"], scale=x["scale"], stream=side)
    torch.cuda.current_stream().wait_stream(side)
    for n, t in dict(got, o=o, S_T=S_T).items():
        assert torch.equal(t, ref[n]), n


def test_two_calls_at_once():
    """Two streams, each with a workspace of its own (the binding's)."""
    xs = [cuda(gdr_inputs(1, 2000, 4, 4, 128, 128, BF, seed=91 + i)) for i in range(2)]
    refs = [run(x) for x in xs]
    streams = [torch.cuda.Stream() for _ in xs]
    got = []
    for x, s in zip(xs, streams):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            o, S_T, S_c = carve.gdr_chunk_fwd(x["q"], x["k"], x["v"], x["g"], x["beta"], x["S0"], scale=x["scale"])
            r = carve.gdr_chunk_bwd(x["q"], x["k"], x["v"], x["g"], x["beta"], S_c, x["dO"], x["dS_T"], scale=x["scale"])
            got.append(dict(r, o=o, S_T=S_T))
    torch.cuda.synchronize()
    for g, ref in zip(got, refs):
        for n in ref:
            assert torch.equal(g[n], ref[n]), n


def test_captured_and_replayed():
    """Forward, backward and steps in one graph, replayed on changed inputs with eager
    calls between the replays."""
    x = cuda(gdr_inputs(1, 200, 2, 4, 64, 64, BF, seed=101))
    other = cuda(gdr_inputs(1, 200, 2, 4, 64, 64, BF, seed=102))
    pool = torch.zeros(3, 4, 64, 64, device="cuda")
    slots = torch.tensor([2], dtype=torch.int32, device="cuda")

    def work():
        r = run_nosync(x)
        pool.copy_(x["S0"].expand(3, -1, -1, -1))
        r["step"] = carve.gdr_step(*(x[n][:, :3].contiguous() for n in ("q", "k", "v", "g", "beta")), pool, slots)
        r["pool"] = pool
        return r

    def run_nosync(x):
        o, S_T, S_c = carve.gdr_chunk_fwd(x["q"], x["k"], x["v"], x["g"], x["beta"], x["S0"])
        r = carve.gdr_chunk_bwd(x["q"], x["k"], x["v"], x["g"], x["beta"], S_c, x["dO"], x["dS_T"])
        return dict(r, o=o, S_T=S_T)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        work()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        res = work()
    for turn in range(4):
        src = other if turn % 2 else cuda(gdr_inputs(1, 200, 2, 4, 64, 64, BF, seed=110 + turn))
        for n in ("q", "k", "v", "g", "beta", "S0", "dO", "dS_T"):
            x[n].copy_(src[n])
        graph.replay()
        torch.cuda.synchronize()
        got = {n: t.clone() for n, t in res.items()}
        want = work()
        torch.cuda.synchronize()
        for n in want:
            assert torch.equal(got[n], want[n]), (turn, n)


def test_replayed_on_other_sequences():
    """Offsets, slots and states are read on the device: one graph serves batches that are
    packed otherwise, a sequence longer than any it was captured with among them."""
    x = cuda(gdr_inputs(1, 300, 2, 4, 128, 64, BF, seed=121, seqs=4))
    offs = [[0, 100, 100, 164, 300], [0, 0, 0, 299, 300], [10, 11, 200, 290, 290], [0, 300, 300, 300, 300]]
    off = torch.tensor(offs[0], dtype=torch.int32, device="cuda")
    pool, slots = torch.zeros(5, 4, 64, 128, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    outs = {n: torch.zeros_like(x[m]) for n, m in (("o", "v"), ("dq", "q"), ("dk", "k"), ("dv", "v"), ("dg", "g"), ("dbeta", "beta"))}

    def work():
        for t in outs.values():
            t.zero_()
        o, S_T, S_c = carve.gdr_chunk_fwd(x["q"], x["k"], x["v"], x["g"], x["beta"], x["S0"], offsets=off, out={"o": outs["o"]})
        r = carve.gdr_chunk_bwd(x["q"], x["k"], x["v"], x["g"], x["beta"], S_c, x["dO"], x["dS_T"], offsets=off,
                                out={n: t for n, t in outs.items() if n != "o"})
        pool.zero_()
        r["step"] = carve.gdr_step(*(x[n][:, :1].contiguous() for n in ("q", "k", "v", "g", "beta")), pool, slots)
        return dict(r, S_T=S_T, pool=pool, **outs)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        work()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        res = work()
    for turn, now in enumerate(offs + offs[:1]):
        off.copy_(torch.tensor(now, dtype=torch.int32))
        slots.fill_(turn % 5)
        graph.replay()
        torch.cuda.synchronize()
        got = {n: t.clone() for n, t in res.items()}
        want = {n: t.clone() for n, t in work().items()}
        torch.cuda.synchronize()
        assert got["pool"][turn % 5].any()
        for n in want:
            assert torch.equal(got[n], want[n]), (turn, n)


def test_small_step_between_large_strides():
    """A step on one token of a wide projection whose head and token strides differ from every
    other call's, with padding entries, twice on the same pool."""
    B, Hk, Hv, D = 3, 2, 4, 64
    x = gdr_inputs(B, 2, Hk, Hv, D, D, F32, seed=131)
    ref = gdr_reference(x, grads=False)
    wide = torch.zeros(B, 2, 2 * Hk * D + Hv * D + 64, device="cuda")
    q = wide[..., :Hk * D].view(B, 2, Hk, D)
    k = wide[..., Hk * D:2 * Hk * D].view(B, 2, Hk, D)
    v = wide[..., 2 * Hk * D:2 * Hk * D + Hv * D].view(B, 2, Hv, D)
    for t, n in ((q, "q"), (k, "k"), (v, "v")):
        t.copy_(x[n])
    pool = torch.zeros(7, Hv, D, D, device="cuda")
    slots = torch.tensor([6, 0, 3], dtype=torch.int32, device="cuda")
    pool[slots.long()] = x["S0"].cuda()
    for t in range(2):
        cut = slice(t, t + 1)
        o = carve.gdr_step(q[:, cut], k[:, cut], v[:, cut], x["g"][:, cut].contiguous().cuda(),
                           x["beta"][:, cut].contiguous().cuda(), pool, slots, scale=x["scale"])
        assert rel(o, ref["o"][:, cut]) <= 256 * 2.0 ** -24, t
    assert rel(pool[slots.long()], ref["S_T"]) <= 256 * 2.0 ** -24


def test_more_than_2_31_values():
    """Values, outputs and value gradients past 2^31 elements: the end of a long sequence
    against a call on that end alone, from the state that the long call had there."""
    T, Hk, Hv, Dk, Dv, n = 66 * 1024, 4, 128, 32, 256, 128
    assert T * Hv * Dv > 1 << 31
    gen = torch.Generator(device="cuda").manual_seed(7)
    rnd = lambda *s: torch.randn(*s, generator=gen, device="cuda", dtype=BF)
    q, k = rnd(1, T, Hk, Dk) / 6, rnd(1, T, Hk, Dk) / 6
    v, dO = rnd(1, T, Hv, Dv), rnd(1, T, Hv, Dv)
    g = -0.1 * torch.rand(1, T, Hv, generator=gen, device="cuda")
    beta = torch.rand(1, T, Hv, generator=gen, device="cuda").to(BF)
    o, S_T, S_c = carve.gdr_chunk_fwd(q, k, v, g, beta)
    r = carve.gdr_chunk_bwd(q, k, v, g, beta, S_c, dO)
    end = [t[:, T - n:].contiguous() for t in (q, k, v, g, beta)]
    S0 = S_c[(T - n) // 64:(T - n) // 64 + 1].contiguous()
    oe, Se, Sce = carve.gdr_chunk_fwd(*end, S0)
    re = carve.gdr_chunk_bwd(*end, Sce, dO[:, T - n:].contiguous())
    assert oe.float().abs().max() > 0.1
    assert torch.equal(o[:, T - n:], oe) and torch.equal(S_T, Se)
    for m in ("dq", "dk", "dv", "dg", "dbeta"):
        assert torch.equal(r[m][:, T - n:], re[m]), m
        assert torch.isfinite(r[m][:, :64]).all(), m
