"""The short convolution, rotary positions and the state space scan as programs call them: on
other streams, at once, captured and replayed, on many sequences, on offsets outside the
contract, at far addresses, beside broken sequences; and the launches that they make."""
import ctypes

import pytest
import torch

from gdr_util import cuda, rel
from paper_2606_27229_amd import carve
from ssm_util import TOL, conv_inputs, conv_reference, rotary_reference, ssm_inputs, ssm_reference

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32


def ends(lens, first=0):
    return torch.tensor([first] + list(lens)).cumsum(0).to(torch.int32).cuda()


def scan(x, offsets=None, stream=None, out=None, back=None, workspace=(None, None)):
    """Outputs and gradients of the scan on tensors of ssm_inputs on the card."""
    args, opt = [x[n] for n in ("x", "dt", "A", "Bm", "Cm")], {"D": x["D"], "dt_bias": x["dt_bias"], "offsets": offsets, "stream": stream}
    y, S_T, S_c = carve.ssm_chunk_fwd(*args, x["S0"], out=out, workspace=workspace[0], **opt)
    return {"y": y, "S_T": S_T, **carve.ssm_chunk_bwd(*args, S_c, x["dy"], x["dS_T"], out=back, workspace=workspace[1], **opt)}


def conv(x, offsets=None, stream=None, out=None, back=None, workspace=None):
    kw = {"bias": x["bias"], "activation": x["act"], "offsets": offsets, "stream": stream}
    y, x_T = carve.short_conv_fwd(x["x"], x["weight"], x["x0"], out=out, **kw)
    return {"y": y, "x_T": x_T, **carve.short_conv_bwd(x["x"], x["weight"], x["dy"], x["x0"], x["dx_T"], out=back, want_dx0=True,
                                                       workspace=workspace, **kw)}


def turn(x, offsets=None, stream=None, out=None, back=None):
    kw = {"offsets": offsets, "stream": stream, "start": x["start"]}
    q, k = carve.rotary_fwd(x["q"], x["k"], x["freq"], out=out, **kw)
    dq, dk = carve.rotary_bwd(x["q"], x["k"], x["freq"], out=back, **kw)
    return {"q": q, "k": k, "dq": dq, "dk": dk}


def turn_inputs(T, dtype, seed, seqs=1, Hq=4, Hk=2, D=64, rot=32):
    gen = torch.Generator().manual_seed(seed)
    return {"q": torch.randn(1, T, Hq, D, generator=gen).to(dtype), "k": torch.randn(1, T, Hk, D, generator=gen).to(dtype),
            "freq": carve.rotary_frequencies(rot, device="cpu"),
            "start": torch.randint(0, 5000, (seqs,), generator=gen).int()}


def all_inputs(T, seed, seqs=1, dtype=BF):
    """Inputs of the three, T rows of `seqs` sequences."""
    return (cuda(conv_inputs(1, T, 136, 4, dtype, seed, seqs=seqs)), cuda(turn_inputs(T, dtype, seed, seqs)),
            cuda(ssm_inputs(1, T, 2, 4, 64, 64, dtype, seed, seqs=seqs)))


CALLS = (conv, turn, scan)


def same(got, want, note=()):
    for n in want:
        assert torch.equal(got[n], want[n]), (n, *note)


# ---- streams and graphs -------------------------------------------------------------------


def test_on_another_stream():
    for call, x in zip(CALLS, all_inputs(300, 81)):
        ref = call(x)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        got = call(x, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        same(got, ref, (call.__name__,))


def test_two_calls_at_once():
    """Two streams, each with workspaces of its own (the binding's)."""
    xs = [all_inputs(3000, 91 + i) for i in range(2)]
    refs = [[call(x) for call, x in zip(CALLS, y)] for y in xs]
    streams, got = [torch.cuda.Stream() for _ in xs], []
    for y, s in zip(xs, streams):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            got.append([call(x) for call, x in zip(CALLS, y)])
    torch.cuda.synchronize()
    for g, r in zip(got, refs):
        for a, b in zip(g, r):
            same(a, b)


def captured(work):
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        work()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        res = work()
    return graph, res


def test_captured_and_replayed():
    """Forward, backward and steps of the three in one graph, replayed on changed inputs with
    eager calls between the replays."""
    xs = all_inputs(200, 101)
    pools = torch.zeros(3, 3, 136, dtype=BF, device="cuda"), torch.zeros(3, 4, 64, 64, device="cuda")
    slots = torch.tensor([2], dtype=torch.int32, device="cuda")

    def work():
        r = {f"{call.__name__} {n}": t for call, x in zip(CALLS, xs) for n, t in call(x).items()}
        c, _, s = xs
        pools[0].copy_(c["x0"].expand(3, -1, -1))
        pools[1].copy_(s["S0"].expand(3, -1, -1, -1))
        r["step"] = carve.short_conv_step(c["x"][:, :3], c["weight"], pools[0], slots, bias=c["bias"])
        r["ssm step"] = carve.ssm_step(*(s[n][:, :3] if n != "A" else s[n] for n in ("x", "dt", "A", "Bm", "Cm")), pools[1], slots,
                                       D=s["D"], dt_bias=s["dt_bias"])
        return dict(r, pool=pools[0], states=pools[1])

    graph, res = captured(work)
    for turn_ in range(4):
        for x, src in zip(xs, all_inputs(200, 110 + turn_)):
            for n, t in src.items():
                if isinstance(t, torch.Tensor):
                    x[n].copy_(t)
        graph.replay()
        torch.cuda.synchronize()
        got = {n: t.clone() for n, t in res.items()}
        want = {n: t.clone() for n, t in work().items()}
        torch.cuda.synchronize()
        same(got, want, (turn_,))


def test_replayed_on_other_sequences():
    """Offsets, starts and slots are read on the device: one graph serves batches that are
    packed otherwise, a sequence longer than any it was captured with among them."""
    xs = all_inputs(300, 121, seqs=4)
    offs = [[0, 100, 100, 164, 300], [0, 0, 0, 299, 300], [10, 11, 200, 290, 290], [0, 300, 300, 300, 300]]
    off = torch.tensor(offs[0], dtype=torch.int32, device="cuda")
    c, t, s = xs
    z = torch.zeros_like
    outs = [({"y": z(c["x"])}, {"dx": z(c["x"])}), ({"q": z(t["q"]), "k": z(t["k"])}, {"q": z(t["q"]), "k": z(t["k"])}),
            ({"y": z(s["x"])}, {"dx": z(s["x"]), "ddt": z(s["dt"]), "dBm": z(s["Bm"]), "dCm": z(s["Cm"])})]

    def work():
        r = {}
        for call, x, (fw, bw) in zip(CALLS, xs, outs):
            for o in (*fw.values(), *bw.values()):
                o.zero_()
            r.update({f"{call.__name__} {n}": o for n, o in call(x, off, out=dict(fw), back=dict(bw)).items()})
        return r

    graph, res = captured(work)
    for at, now in enumerate(offs + offs[:1]):
        off.copy_(torch.tensor(now, dtype=torch.int32))
        t["start"].copy_(torch.tensor([at, 50 * at, 7, 0], dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        got = {n: o.clone() for n, o in res.items()}
        want = {n: o.clone() for n, o in work().items()}
        torch.cuda.synchronize()
        same(got, want, (at,))


def test_two_graphs_share_a_workspace():
    """One workspace for two captured calls that are replayed one after another."""
    xs = [cuda(ssm_inputs(1, T, 1, 4, 64, 128, BF, T)) for T in (700, 130)]
    refs = [scan(x) for x in xs]
    ws = [torch.empty(1 << 26, dtype=torch.uint8, device="cuda") for _ in range(2)]
    runs = [captured(lambda x=x: scan(x, workspace=ws)) for x in xs]
    for at in (0, 1, 0, 1):
        runs[at][0].replay()
        torch.cuda.synchronize()
        same(runs[at][1], refs[at], (at,))
        ws[0].fill_(255), ws[1].fill_(255)


# ---- sequences ------------------------------------------------------------------------------


@pytest.mark.parametrize("nseq", [63, 64, 70, 300])
def test_many_sequences(nseq):
    """Up to 63 sequences the convolution finds at once, more by a search."""
    lens = [(0, 1, 65, 5, 13, 2)[(5 * i * i + i) % 6] if i % 9 else 30 for i in range(nseq)]
    T, off = sum(lens), ends(lens)
    x = conv_inputs(1, T, 40, 3, F, nseq, seqs=nseq)
    got = conv(cuda(x), off)
    for n, r in conv_reference(x, lens).items():
        assert rel(got[n], r) <= TOL[F], n
    x = ssm_inputs(1, T, 2, 4, 32, 32, F, nseq, seqs=nseq)
    got = scan(cuda(x), off)
    for n, r in ssm_reference(x, lens).items():
        assert rel(got[n], r) <= TOL[F], n
    x = turn_inputs(T, F, nseq, nseq)
    got = turn(cuda(x), off)
    pos = torch.cat([s + torch.arange(n) for s, n in zip(x["start"], lens)])[None]
    for n, sign in (("q", 1), ("dk", -1)):
        assert rel(got[n], rotary_reference(x[n[-1]], x["freq"], pos, False, 1.0, sign)) <= TOL[F], n


class Guarded:
    """Tensors that lie between values nothing may change."""

    PAD = 1 << 16     # elements on either side, more than a chunk's state of any head here

    def __init__(self):
        self.whole = []

    def __call__(self, shape, dtype, fill=5):
        n = 1
        for s in shape:
            n *= s
        flat = torch.full((n + 2 * self.PAD,), fill, dtype=dtype, device="cuda")
        self.whole.append((flat, n, fill))
        return flat[self.PAD:self.PAD + n].view(shape)

    def check(self):
        for i, (flat, n, fill) in enumerate(self.whole):
            assert (flat[:self.PAD] == fill).all() and (flat[self.PAD + n:] == fill).all(), i


OFFSETS = [[0, 150, 50, 500, -7], [300, 10, 0, 0, 200], [-5, -4, 1 << 30, 3, 2], [200, 200, 199, 63, 64], [0, 200, 200, 200, 200],
           [-(1 << 31), (1 << 31) - 1, -1, (1 << 31) - 1, 0]]


@pytest.mark.parametrize("many", [1, 20])
@pytest.mark.parametrize("G,H,P,N,dtype", [(1, 2, 64, 64, BF), (2, 4, 32, 128, BF), (1, 3, 64, 128, F), (1, 2, 96, 32, F), (1, 8, 64, 128, BF)])
def test_every_output_stays_in_its_bounds(G, H, P, N, dtype, many):
    """Offsets outside the contract (decreasing, negative, too large) among others: the calls
    return, and write within outputs and workspaces of the sizes that the library names."""
    T, C, W = 200, 136, 4
    lib, code = carve.load_library(), carve.CARVE_BF16 if dtype == BF else carve.CARVE_F32
    for offs in OFFSETS:
        off = [offs[0]] + offs[1:] * many
        n = len(off) - 1
        print(f"case bad offsets {offs} x{many} H={H} P={P} N={N} {dtype}", flush=True)
        o = torch.tensor(off, dtype=torch.int64).to(torch.int32).cuda()
        g = Guarded()
        x = cuda(ssm_inputs(1, T, G, H, P, N, dtype, 3, seqs=n))
        d = carve.SsmDims(1, T, n, G, H, P, N, code, 1, *(s for t in ("x", "Bm", "Cm") for s in x[t].stride()[:3]), *x["dt"].stride()[:2])
        chunks = lib.carve_ssm_chunk_count(ctypes.byref(d))
        ws = [g((lib.carve_ssm_workspace_size(ctypes.byref(d), b),), torch.uint8) for b in (0, 1)]
        out = {"y": g((1, T, H, P), dtype), "S_T": g((n, H, P, N), F), "S_chunks": g((chunks, H, P, N), F)}
        back = {"dx": g((1, T, H, P), dtype), "ddt": g((1, T, H), dtype), "dA": g((H,), F), "dBm": g((1, T, G, N), dtype),
                "dCm": g((1, T, G, N), dtype), "dD": g((H,), F), "ddt_bias": g((H,), F), "dS0": g((n, H, P, N), F)}
        scan(x, o, out=out, back=back, workspace=ws)
        x = cuda(conv_inputs(1, T, C, W, dtype, 3, seqs=n))
        d = carve.ShortConvDims(1, T, n, C, W, code, 1, T * C, C)
        conv(x, o, out={"y": g((1, T, C), dtype), "x_T": g((n, W - 1, C), dtype)},
             back={"dx": g((1, T, C), dtype), "dweight": g((C, W), F), "dbias": g((C,), F), "dx0": g((n, W - 1, C), dtype)},
             workspace=g((lib.carve_short_conv_workspace_size(ctypes.byref(d)),), torch.uint8))
        x = cuda(turn_inputs(T, dtype, 3, n))
        turn(x, o, out={"q": g(x["q"].shape, dtype), "k": g(x["k"].shape, dtype)}, back={"q": g(x["q"].shape, dtype), "k": g(x["k"].shape, dtype)})
        torch.cuda.synchronize()
        g.check()


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("dtype", [BF, F])
def test_a_broken_sequence_breaks_no_other(value, dtype):
    """A NaN or an infinity in one packed sequence, its start state among it."""
    lens = [70, 64, 1, 33]
    off, at = ends(lens), slice(70, 134)
    others = torch.cat([torch.arange(70), torch.arange(134, 168)])
    for call, make, names in ((conv, lambda: cuda(conv_inputs(1, 168, 40, 4, dtype, 1, seqs=4)), ("x", "dy", "x0", "dx_T")),
                              (scan, lambda: cuda(ssm_inputs(1, 168, 1, 2, 64, 64, dtype, 1, seqs=4)), ("x", "dt", "Bm", "dy", "S0", "dS_T"))):
        want, x = call(make(), off), make()
        for n in names:
            if x[n].shape[1] == 168:
                x[n][0, 70 + 20] = value
            else:
                x[n][1] = value
        got = call(x, off)
        for n, t in want.items():
            if t.shape[:2] == (1, 168):
                assert torch.equal(got[n][:, others], t[:, others]), (call.__name__, n)
            elif n in ("x_T", "S_T", "dx0", "dS0"):
                assert torch.equal(got[n][[0, 2, 3]], t[[0, 2, 3]]), (call.__name__, n)
        assert not torch.isfinite(got["y"][:, at].float()).all()


def test_a_broken_state_of_the_pool_breaks_no_other():
    x = cuda(ssm_inputs(3, 2, 1, 2, 32, 64, BF, 5))
    c = cuda(conv_inputs(3, 2, 64, 4, BF, 5))
    slots = torch.tensor([4, 1, 0], dtype=torch.int32, device="cuda")
    res = []
    for broken in (False, True):
        S, K = torch.zeros(5, 2, 32, 64, device="cuda"), torch.zeros(5, 3, 64, dtype=BF, device="cuda")
        if broken:
            S[1], K[1] = float("nan"), float("nan")
        y = carve.ssm_step(*(x[n] for n in ("x", "dt", "A", "Bm", "Cm")), S, slots, D=x["D"], dt_bias=x["dt_bias"])
        z = carve.short_conv_step(c["x"], c["weight"], K, slots, bias=c["bias"])
        res.append((y, z, S, K))
    for i, keep in enumerate(([0, 2], [0, 2], [0, 2, 3, 4], [0, 2, 3, 4])):
        assert torch.equal(res[0][i][keep], res[1][i][keep]), i


# ---- far addresses --------------------------------------------------------------------------


def test_rows_far_apart():
    """Rows whose offsets pass 32 bits."""
    T, width = 300, (1 << 23) - 64
    base = torch.zeros(T * width + 4096, dtype=BF, device="cuda")
    assert T * width > 1 << 31
    x = ssm_inputs(1, T, 1, 1, 32, 32, BF, 12)
    d = cuda(x)
    want = scan(d)
    far = base.as_strided((1, T, 1, 32), (0, width, 32, 1))
    for n in ("x", "Bm", "Cm"):
        keep = d[n]
        d[n] = far
        far.copy_(keep)
        same(scan(d), want, (n,))
        d[n] = keep
    c = cuda(conv_inputs(1, T, 64, 4, BF, 12))
    want = conv(c)
    far = base.as_strided((1, T, 64), (0, width, 1))
    far.copy_(c["x"])
    c["x"] = far
    same(conv(c), want)
    q = cuda(turn_inputs(T, BF, 12))
    want = turn(q)
    far = base.as_strided((1, T, 4, 64), (0, width, 64, 1))
    far.copy_(q["q"])
    same(turn(q | {"q": far}), want)


def test_step_far_slot():
    """Slots whose state lies past 2^31 elements."""
    H, P, N = 32, 128, 128
    pool = (1 << 31) // (H * P * N) + 3
    x = ssm_inputs(1, 1, 1, H, P, N, BF, 61, dst=False)
    ref = ssm_reference(x, grads=False)
    d = cuda(x)
    st = torch.zeros(pool, H, P, N, device="cuda")
    st[pool - 1] = d["S0"][0]
    slot = torch.tensor([pool - 1], dtype=torch.int32).cuda()
    y = carve.ssm_step(*(d[n] for n in ("x", "dt", "A", "Bm", "Cm")), st, slot, D=d["D"], dt_bias=d["dt_bias"])
    assert rel(y, ref["y"]) <= TOL[BF] and rel(st[pool - 1:], ref["S_T"]) <= TOL[F]
    assert not st[:pool - 1].any()
    C, W = 16384, 4
    pool = (1 << 31) // ((W - 1) * C) + 3
    c = conv_inputs(1, 1, C, W, BF, 61)
    ref, d = conv_reference(c), cuda(c)
    st = torch.zeros(pool, W - 1, C, dtype=BF, device="cuda")
    st[pool - 1] = d["x0"][0]
    y = carve.short_conv_step(d["x"], d["weight"], st, torch.tensor([pool - 1], dtype=torch.int32).cuda(), bias=d["bias"])
    assert rel(y, ref["y"]) <= TOL[BF] and torch.equal(st[pool - 1].cpu().double(), ref["x_T"][0])
    assert not st[:pool - 1].any()


def rnd(seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return lambda *s: torch.randn(*s, generator=gen, device="cuda", dtype=BF)


def test_scan_of_more_than_2_31_values():
    """The end of a long sequence against a call on that end alone, from the state that the
    long call had there."""
    T, H, P, N, n = 66 * 1024, 128, 256, 32, 128
    assert T * H * P > 1 << 31
    r = rnd(7)
    x, dy, dt, Bm, Cm = r(1, T, H, P), r(1, T, H, P), r(1, T, H) - 3, r(1, T, 1, N), r(1, T, 1, N)
    A = -torch.rand(H, device="cuda") - 1
    y, S_T, S_c = carve.ssm_chunk_fwd(x, dt, A, Bm, Cm)
    g = carve.ssm_chunk_bwd(x, dt, A, Bm, Cm, S_c, dy)
    cut = lambda t: t[:, T - n:].contiguous()
    end = cut(x), cut(dt), A, cut(Bm), cut(Cm)
    ye, Se, Sce = carve.ssm_chunk_fwd(*end, S_c[(T - n) // 64:(T - n) // 64 + 1].contiguous())
    ge = carve.ssm_chunk_bwd(*end, Sce, cut(dy))
    assert ye.float().abs().max() > 0.1
    assert rel(y[:, T - n:], ye.cpu()) <= TOL[BF] and rel(S_T, Se.cpu()) <= TOL[F]
    for m in ("dx", "ddt", "dBm", "dCm"):
        assert rel(g[m][:, T - n:], ge[m].cpu()) <= TOL[BF], m
        assert torch.isfinite(g[m][:, :64]).all(), m


def test_convolution_and_positions_of_more_than_2_31_values():
    T, C, n = 132 * 1024, 16384, 96
    assert T * C > 1 << 31
    r = rnd(8)
    x, dy, w = r(1, T, C), r(1, T, C), r(C, 4).float()
    y, x_T = carve.short_conv_fwd(x, w)
    g = carve.short_conv_bwd(x, w, dy)
    end, x0 = x[:, T - n:].contiguous(), x[:, T - n - 3:T - n].contiguous()
    ye, xe = carve.short_conv_fwd(end, w, x0)
    ge = carve.short_conv_bwd(end, w, dy[:, T - n:].contiguous(), x0)
    # (runs of rows begin elsewhere: a run's own order of sums is the same)
    assert rel(y[:, T - n:], ye.cpu()) <= TOL[BF] and torch.equal(x_T, xe)
    assert rel(g["dx"][:, T - n:], ge["dx"].cpu()) <= TOL[BF]
    freq = carve.rotary_frequencies(128)
    q = x.view(1, T, 128, 128)
    out, _ = carve.rotary_fwd(q, None, freq)
    tail, _ = carve.rotary_fwd(q[:, T - n:].contiguous(), None, freq, start=torch.tensor([T - n], dtype=torch.int32, device="cuda"))
    assert torch.equal(out[:, T - n:], tail) and torch.equal(out[:, 0], q[:, 0])


# ---- the measurement hook and what is no tensor ------------------------------------------------


def recorded(call):
    """Events the hook records during one call: those after a marker recorded first."""
    ev = [torch.cuda.Event(enable_timing=True) for _ in range(16)]
    mark = torch.cuda.Event(enable_timing=True)
    for e in ev:
        e.record()
    mark.record()
    torch.cuda.synchronize()
    carve.profile_events(ev)
    call()
    torch.cuda.synchronize()
    return sum(mark.elapsed_time(e) > 0 for e in ev)


def test_launches():
    """As the header states them: two more where a sequence may have several spans, one for
    the shares of dB and dC."""
    c, t, _ = all_inputs(200, 5)
    kw = {"bias": c["bias"]}
    assert recorded(lambda: carve.short_conv_fwd(c["x"], c["weight"], **kw)) == 1 + 1
    assert recorded(lambda: carve.short_conv_bwd(c["x"], c["weight"], c["dy"], **kw)) == 2 + 1
    assert recorded(lambda: carve.short_conv_step(c["x"], c["weight"], c["x0"], **kw)) == 1 + 1
    assert recorded(lambda: carve.rotary_fwd(t["q"], t["k"], t["freq"])) == 1 + 1
    for T, H, fwd, bwd in ((128, 1, 2, 4), (2000, 1, 4, 6), (128, 4, 2, 5), (2000, 4, 4, 7)):
        x = cuda(ssm_inputs(1, T, 1, H, 64, 64, BF, 5))
        args = [x[n] for n in ("x", "dt", "A", "Bm", "Cm")]
        assert recorded(lambda: carve.ssm_chunk_fwd(*args)) == fwd + 1, T
        S_c = carve.ssm_chunk_fwd(*args)[2]
        assert recorded(lambda: carve.ssm_chunk_bwd(*args, S_c, x["dy"])) == bwd + 1, (T, H)
    assert recorded(lambda: carve.ssm_step(*args, x["S0"])) == 1 + 1


def test_every_tensor_of_the_entry_points():
    z = lambda *s, dt=F: torch.zeros(s, dtype=dt, device="cuda")
    x, w, st, f = z(1, 4, 64), z(64, 4), z(1, 3, 64), torch.zeros(8, dtype=torch.float64, device="cuda")
    q, a = z(1, 4, 1, 32), (z(1, 4, 1, 32), z(1, 4, 1), z(1), z(1, 4, 1, 32), z(1, 4, 1, 32))
    S, no = z(1, 1, 32, 32), [0.0]
    calls = {
        "x": lambda: carve.short_conv_fwd(no, w), "weight": lambda: carve.short_conv_fwd(x, no),
        "bias": lambda: carve.short_conv_fwd(x, w, bias=no), "x0": lambda: carve.short_conv_fwd(x, w, no),
        "offsets": lambda: carve.short_conv_fwd(x, w, offsets=[0, 4]), "y": lambda: carve.short_conv_fwd(x, w, out={"y": no}),
        "dy": lambda: carve.short_conv_bwd(x, w, no), "dx_T": lambda: carve.short_conv_bwd(x, w, x, None, no),
        "dx": lambda: carve.short_conv_bwd(x, w, x, out={"dx": no}), "workspace": lambda: carve.short_conv_bwd(x, w, x, workspace=4),
        "slots": lambda: carve.short_conv_step(x, w, st, [0]), "out": lambda: carve.short_conv_step(x, w, st, out=no),
        "q": lambda: carve.rotary_fwd(no, None, f), "k": lambda: carve.rotary_fwd(q, no, f), "freq": lambda: carve.rotary_fwd(q, None, no),
        "positions": lambda: carve.rotary_fwd(q, None, f, positions=no), "start": lambda: carve.rotary_fwd(q, None, f, start=no),
        "out q": lambda: carve.rotary_fwd(q, None, f, out={"q": no}),
        "dt": lambda: carve.ssm_chunk_fwd(a[0], no, *a[2:]), "A": lambda: carve.ssm_chunk_fwd(*a[:2], no, *a[3:]),
        "Bm": lambda: carve.ssm_chunk_fwd(*a[:3], no, a[4]), "Cm": lambda: carve.ssm_chunk_fwd(*a[:4], no),
        "D": lambda: carve.ssm_chunk_fwd(*a, D=no), "dt_bias": lambda: carve.ssm_chunk_fwd(*a, dt_bias=no),
        "S0": lambda: carve.ssm_chunk_fwd(*a, no), "S_T": lambda: carve.ssm_chunk_fwd(*a, out={"S_T": no}),
        "S_chunks": lambda: carve.ssm_chunk_bwd(*a, no, q), "dS_T": lambda: carve.ssm_chunk_bwd(*a, z(2, 1, 32, 32), q, no),
        "dBm": lambda: carve.ssm_chunk_bwd(*a, z(2, 1, 32, 32), q, out={"dBm": no}),
    }
    for name, call in calls.items():
        with pytest.raises(TypeError, match=f"^{name} must be a GPU tensor"):
            call()
    for call in (lambda: carve.short_conv_fwd(x.cpu(), w), lambda: carve.rotary_fwd(q, None, f.cpu()), lambda: carve.ssm_chunk_fwd(*a, S.cpu()),
                 lambda: carve.short_conv_fwd(x, w[:, :3].contiguous().half()), lambda: carve.short_conv_fwd(x, z(32, 4)),
                 lambda: carve.short_conv_fwd(x, w, z(1, 2, 64)), lambda: carve.rotary_fwd(q, None, f.float()),
                 lambda: carve.rotary_fwd(q, z(1, 4, 1, 64), f), lambda: carve.ssm_chunk_fwd(a[0], a[1].bfloat16(), *a[2:]),
                 lambda: carve.ssm_chunk_fwd(*a, z(1, 1, 32, 64)), lambda: carve.ssm_step(*a, z(1, 2, 32, 32)),
                 lambda: carve.short_conv_fwd(x, w, activation="gelu"), lambda: carve.short_conv_fwd(x[..., ::2], w[:32].contiguous())):
        with pytest.raises((TypeError, ValueError)):
            call()
