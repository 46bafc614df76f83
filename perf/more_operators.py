"""Performance cases of the short causal convolution, the rotary positions and the
selective state space scan: the calls a program that trains or serves such layers makes.

A case is a dict of plain values.  "kind" says which call:
  conv_step   T tokens for each of B sequences on the last inputs kept in a pool
  conv        the convolution of prompts: outputs and the last inputs
  conv_train  the convolution and its backward
  rot         queries and keys turned by their positions
  rot_train   the same and its backward
  ssm_step    T tokens for each of B sequences on their states in a pool
  ssm         the chunked scan: outputs and final states (prefill)
  ssm_train   the chunked scan and its backward
Every case has B, T, dtype, nseq and cut (nseq = 0: B sequences of T tokens; n: n
sequences of unequal lengths, some of them empty or of one token, packed into T rows,
their lengths made from `cut`), and state (a carried start state; far: the position that
the first row of a rotary case may have).
"""
from __future__ import annotations

import itertools
import math
import random

import torch

own = False

CHUNK = 64          # chunk of the plain form of the scan
BASE = 10000.0      # of the rotary frequencies
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _conv(name, kind, B, T, C, W=4, dtype="bf16", act="silu", bias=True, state=False, nseq=0, cut=0, pool=0):
    return {"name": name, "kind": kind, "B": B, "T": T, "C": C, "W": W, "dtype": dtype, "act": act, "bias": bias,
            "state": state, "nseq": nseq, "cut": cut, "pool": pool}


def _rot(name, kind, B, T, Hq, Hk, Dh, rot, dtype="bf16", interleaved=False, far=0, factor=1.0, nseq=0, cut=0):
    return {"name": name, "kind": kind, "B": B, "T": T, "Hq": Hq, "Hk": Hk, "Dh": Dh, "rot": rot, "dtype": dtype,
            "interleaved": interleaved, "far": far, "factor": factor, "nseq": nseq, "cut": cut}


def _ssm(name, kind, B, T, G, H, N, P, dtype="bf16", skip=True, state=False, nseq=0, cut=0, pool=0):
    return {"name": name, "kind": kind, "B": B, "T": T, "G": G, "H": H, "N": N, "P": P, "dtype": dtype, "skip": skip,
            "state": state, "nseq": nseq, "cut": cut, "pool": pool}


def listed():
    return [
        # a decoding batch's convolution of 32 heads of 64 with keys and queries of 128: latency
        _conv("conv_step", "conv_step", 64, 1, 2304, pool=96),
        # prompts of unequal lengths arriving together, some continuing
        _conv("conv_ragged", "conv", 1, 1777, 2304, state=True, nseq=9, cut=3),
        # a training step's
        _conv("conv_train", "conv_train", 4, 4096, 2304),
        # queries and keys of a decoding batch far into a long context: latency
        _rot("rot_decode", "rot", 64, 1, 16, 8, 128, 128, far=200000, factor=8.0),
        # packed prompts, half of each head turned, neighbouring pairs
        _rot("rot_packed", "rot", 1, 8191, 16, 4, 128, 64, dtype="f32", interleaved=True, far=1000, nseq=7, cut=2),
        # a training step at the 1.3B-scale layer's shape
        _rot("rot_train", "rot_train", 4, 4096, 16, 16, 128, 128),
        # a full decoding batch, states scattered over the pool
        _ssm("ssm_step_batch", "ssm_step", 64, 1, 1, 32, 128, 64, pool=96),
        # prompts of unequal lengths arriving together, some continuing from a state
        _ssm("ssm_ragged", "ssm", 1, 1777, 1, 32, 128, 64, state=True, nseq=9, cut=3),
        # prefill of 4 x 4096 tokens of 32 heads of 64
        _ssm("ssm_layer", "ssm", 4, 4096, 1, 32, 128, 64),
        # one long document, its length no multiple of anything
        _ssm("ssm_long", "ssm", 1, 16381, 2, 32, 128, 64, state=True),
        # a small f32 layer trained from a carried state (as in tests)
        _ssm("ssm_train_f32_small", "ssm_train", 2, 200, 1, 4, 64, 64, dtype="f32", state=True),
        # a training step of 4 x 4096 tokens
        _ssm("ssm_train_layer", "ssm_train", 4, 4096, 1, 32, 128, 64),
    ]


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    kind = rng.choice(("conv_step", "conv", "conv_train", "rot", "rot", "rot_train", "ssm_step", "ssm", "ssm", "ssm_train", "ssm_train"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    state = rng.random() < 0.5

    def rows(most):
        """Tokens of all sequences, and how they are cut into sequences."""
        total = _log(rng, 1, max(2, most))
        nseq = rng.choice((0, 0, rng.randrange(1, 12)))
        B = 1 if nseq else rng.choice([b for b in (1, 1, 2, 3, 4, 8) if b <= total])
        return {"B": B, "T": max(1, total // B), "nseq": nseq, "cut": rng.randrange(1000)}

    if kind.startswith("conv"):
        C, W, act, bias = 8 * _log(rng, 4, 1024), rng.choice((2, 3, 4, 4)), rng.choice(("silu", "silu", "")), rng.random() < 0.7
        if kind == "conv_step":
            B = _log(rng, 1, 256)
            return _conv("", kind, B, rng.choice((1, 1, 1, 2, 5)), C, W, dtype, act, bias, True, pool=B + rng.randrange(0, 17))
        return _conv("", kind, 1, 1, C, W, dtype, act, bias, state) | rows(min(16384, (16384 if dtype == "bf16" else 8192) * 2304 // C))
    if kind.startswith("rot"):
        Dh = rng.choice((64, 128, 192, 256))
        Hk = rng.choice((1, 2, 4, 8, 16))
        Hq = min(32, Hk * rng.choice((1, 1, 2, 4)))
        rot = rng.choice((Dh, Dh, Dh // 2, 32))
        most = 16384 * 4096 // ((Hq + Hk) * Dh) // (1 if dtype == "bf16" else 2)
        return _rot("", kind, 1, 1, Hq, Hk, Dh, rot, dtype, rng.random() < 0.4, rng.choice((0, 0, 4000, 1000000)),
                    rng.choice((1.0, 4.0))) | rows(min(16384, most))
    G = rng.choice((1, 1, 2, 4))
    H = min(32, G * rng.choice((1, 2, 4, 8, 16)))
    N, P = rng.choice((32, 64, 128)), rng.choice((32, 64, 64, 96, 128))
    if kind == "ssm_step":
        B = _log(rng, 1, 64)
        return _ssm("", kind, B, rng.choice((1, 1, 1, 2, 3, 5)), G, H, N, P, dtype, rng.random() < 0.7, True, pool=B + rng.randrange(0, 17))
    # tokens of all sequences, so that a case costs no more than the largest listed one
    most = int((16384 if dtype == "bf16" else 4096) * (32 * 64 * 128) / (H * N * P))
    return _ssm("", kind, 1, 1, G, H, N, P, dtype, rng.random() < 0.7, state) | rows(min(max(64, most), 16384))


def _lengths(case):
    """Lengths of the packed sequences: random cuts, an empty one and one of one
    token among them where there are enough."""
    n, T = case["nseq"], case["T"]
    rng = random.Random(case["cut"])
    cuts = sorted(rng.randrange(0, T + 1) for _ in range(n - 1))
    if n >= 4 and T >= 8:
        at = rng.randrange(0, n - 3)
        cuts[at + 1] = cuts[at]                        # an empty sequence
        cuts[-1] = T - 1                               # and one of one token, the last
        cuts.sort()
    ends = [0] + cuts + [T]
    return [b - a for a, b in zip(ends, ends[1:])]


def _frequencies(case):
    """Angles a position, in 64 bits: base^(-2 i / rot), all divided by the factor that
    stretches a context."""
    i = torch.arange(case["rot"] // 2, dtype=torch.float64)
    return (BASE ** (-2.0 * i / case["rot"]) / case["factor"]).cuda()


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    dt = TYPES[case["dtype"]]
    kind, B, T = case["kind"], case["B"], case["T"]

    def randn(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    s = {"case": case}
    seqs = case["nseq"] or B
    if case["nseq"]:
        lens = _lengths(case)
        offsets = list(itertools.accumulate(lens, initial=0))
        s["offsets"] = torch.tensor(offsets, dtype=torch.int32, device="cuda")
        # each sequence's rows in a padded batch, and back (the plain form's layout)
        row = torch.arange(max(lens), device="cuda")
        start = s["offsets"][:-1].long()
        s["lens"] = s["offsets"][1:].long() - start
        s["there"] = row[None] < s["lens"][:, None]
        s["rows"] = torch.where(s["there"], start[:, None] + row[None], 0)
        s["back"] = s["there"].reshape(-1).nonzero()[:, 0]
    if kind.endswith("step"):
        order = list(range(case["pool"]))
        random.Random(int(seed)).shuffle(order)
        s["slots"] = torch.tensor(order[:B], dtype=torch.int32, device="cuda")
    if kind.startswith("conv"):
        C, W = case["C"], case["W"]
        s["x"] = randn(B, T, C).to(dt)
        s["weight"] = randn(C, W) * W ** -0.5
        s["bias"] = 0.1 * randn(C) if case["bias"] else None
        if kind == "conv_step":
            s["pool"] = randn(case["pool"], W - 1, C).to(dt)
            return s
        s["x0"] = randn(seqs, W - 1, C).to(dt) if case["state"] else None
        if kind == "conv_train":
            s["dy"] = randn(B, T, C).to(dt)
            s["dx_T"] = randn(seqs, W - 1, C).to(dt) if case["state"] else None
        return s
    if kind.startswith("rot"):
        s["q"], s["k"] = randn(B, T, case["Hq"], case["Dh"]).to(dt), randn(B, T, case["Hk"], case["Dh"]).to(dt)
        s["freq"] = _frequencies(case)
        s["amplitude"] = 1.0 + 0.1 * math.log(case["factor"])
        s["start"] = torch.randint(0, case["far"] + 1, (seqs,), generator=gen, device="cuda", dtype=torch.int32)
        if kind == "rot_train":
            s["dq"], s["dk"] = randn(*s["q"].shape).to(dt), randn(*s["k"].shape).to(dt)
        return s
    G, H, N, P = (case[n] for n in ("G", "H", "N", "P"))
    # x, B and C are slices of what the convolution left, as a layer has them; steps of
    # 0.001 to 0.1 at dt = 0, decays of one to a few thousand tokens
    xbc = randn(B, T, H * P + 2 * G * N)
    xbc = (xbc * torch.sigmoid(xbc)).to(dt)
    s["x"] = xbc[..., :H * P].unflatten(-1, (H, P))
    s["Bm"] = xbc[..., H * P:H * P + G * N].unflatten(-1, (G, N))
    s["Cm"] = xbc[..., H * P + G * N:].unflatten(-1, (G, N))
    s["dt"] = randn(B, T, H).to(dt)
    step = torch.exp(torch.rand(H, generator=gen, device="cuda") * math.log(100.0) + math.log(0.001))
    s["dt_bias"] = step + torch.log(-torch.expm1(-step))
    s["A"] = -(1 + 15 * torch.rand(H, generator=gen, device="cuda"))
    s["D"] = 1 + 0.1 * randn(H) if case["skip"] else None
    if kind == "ssm_step":
        s["pool"] = 0.3 * randn(case["pool"], H, P, N)
        return s
    s["S0"] = 0.3 * randn(seqs, H, P, N) if case["state"] else None
    if kind == "ssm_train":
        s["dy"] = randn(B, T, H, P).to(dt)
        s["dS_T"] = 0.3 * randn(seqs, H, P, N) if case["state"] else None
    return s


# ---- the plain form -----------------------------------------------------------------------


def _padded(s, x):
    """[1, T, ...] -> [nseq, longest, ...], zeros behind each sequence."""
    if "rows" not in s:
        return x
    x = x[0][s["rows"]]
    return x * s["there"].reshape(s["there"].shape + (1,) * (x.dim() - 2))


def _packed(s, x):
    return x if "rows" not in s else x.reshape((-1,) + x.shape[2:])[s["back"]][None]


def _grads(outs, leaves):
    """Gradients of sum <d, out>, each rounded to its input's type; leaves: {name: (input, f32 leaf)}."""
    have = {n: x for n, x in leaves.items() if x[0] is not None}
    pairs = [(o, d.float()) for o, d in outs if d is not None]
    got = torch.autograd.grad([o for o, _ in pairs], [leaf for _, leaf in have.values()], [d for _, d in pairs])
    return {"d" + n: g.to(x.dtype) for (n, (x, _)), g in zip(have.items(), got)}


def _leaves(s, names):
    return {n: (s[n], None if s[n] is None else s[n].float().requires_grad_()) for n in names}


def _plain_taps(past, weight, bias, act, T):
    y = (past.unfold(1, weight.shape[1], 1) * weight).sum(-1)[:, :T]
    y = y if bias is None else y + bias
    return y * torch.sigmoid(y) if act else y


def _plain_conv(s, x, weight, bias, x0):
    """Outputs and the last inputs."""
    case = s["case"]
    W = case["W"]
    x = _padded(s, x)
    x0 = torch.zeros(x.shape[0], W - 1, x.shape[2], device=x.device) if x0 is None else x0
    past = torch.cat([x0, x], 1)
    y = _packed(s, _plain_taps(past, weight, bias, case["act"], x.shape[1]))
    at = torch.arange(W - 1, device=x.device)[None] + (s["lens"][:, None] if "lens" in s else x.shape[1])
    x_T = torch.gather(past, 1, at.expand(x.shape[0], -1)[..., None].expand(-1, -1, past.shape[2]))
    return y, x_T


def _run_plain_conv(s):
    case = s["case"]
    dt = s["x"].dtype
    if case["kind"] == "conv_step":
        at = s["slots"].long()
        past = torch.cat([s["pool"][at], s["x"]], 1)
        s["pool"][at] = past[:, case["T"]:]
        bias = None if s["bias"] is None else s["bias"]
        return {"y": _plain_taps(past.float(), s["weight"], bias, case["act"], case["T"]).to(dt), "pool": s["pool"]}
    names = ("x", "weight", "bias", "x0")
    if case["kind"] == "conv":
        y, x_T = _plain_conv(s, *(None if s[n] is None else s[n].float() for n in names))
        return {"y": y.to(dt), "x_T": x_T.to(dt)}
    leaves = _leaves(s, names)
    y, x_T = _plain_conv(s, *(leaf for _, leaf in leaves.values()))
    return {"y": y.detach().to(dt), "x_T": x_T.detach().to(dt), **_grads([(y, s["dy"]), (x_T, s["dx_T"])], leaves)}


def _turned(s, x, sign):
    """x turned by its rows' angles (sign -1: back), in 32 bits with angles in 64."""
    case = s["case"]
    half = case["rot"] // 2
    T = x.shape[1]
    row = torch.arange(T, device=x.device)
    if "offsets" in s:
        seq = torch.searchsorted(s["offsets"][1:], row.int(), right=True)
        pos = (row - s["offsets"][seq] + s["start"][seq])[None]
    else:
        pos = s["start"][:, None] + row[None]
    angle = pos.double()[..., None] * s["freq"]
    m = s["amplitude"]
    cos, sin = (m * torch.cos(angle)).float()[:, :, None], (sign * m * torch.sin(angle)).float()[:, :, None]
    turn, rest = x[..., :2 * half].float(), x[..., 2 * half:].float()
    if case["interleaved"]:
        a, b = turn[..., 0::2], turn[..., 1::2]
        turn = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = turn[..., :half], turn[..., half:]
        turn = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turn, rest], -1).to(x.dtype)


def _run_plain_rot(s):
    out = {"q": _turned(s, s["q"], 1), "k": _turned(s, s["k"], 1)}
    if s["case"]["kind"] == "rot_train":
        out.update(dq=_turned(s, s["dq"], -1), dk=_turned(s, s["dk"], -1))
    return out


def _softplus(x):
    return torch.clamp(x, min=0) + torch.log1p(torch.exp(-torch.abs(x)))


def _plain_ssm(s, x, dt, A, Bm, Cm, D, dt_bias, S0):
    """The chunk form in f32: outputs and final states.  Sums of decays and their
    differences are taken in 64 bits; the states of chunks come from one another by a
    triangle of decays, as the tokens of a chunk do."""
    x, dt, Bm, Cm = (_padded(s, t) for t in (x, dt, Bm, Cm))
    B, T, H, P = x.shape
    G, N = Bm.shape[2:]
    C = min(CHUNK, T)
    n = -(-T // C)
    step = _softplus(dt + dt_bias)
    if "there" in s:
        step = step * s["there"][..., None]

    def chunks(t):   # [B, T, h, ...] -> [B, h, n, C, ...]
        t = torch.nn.functional.pad(t, [0, 0] * (t.dim() - 2) + [0, n * C - T])
        return t.reshape(B, n, C, *t.shape[2:]).movedim(3, 1)

    def triangle(total, strict):   # decays between the entries of the last dimension
        size = total.shape[-1]
        low = torch.ones(size, size, dtype=torch.bool, device=x.device).tril(-1 if strict else 0)
        diff = total[..., :, None] - total[..., None, :]
        return low, diff

    a = chunks(step * A)
    xd = chunks(step[..., None] * x)
    Bc, Cc = (chunks(t).repeat_interleave(H // G, 1) for t in (Bm, Cm))
    inner = a.double().cumsum(-1)
    low, diff = triangle(inner, False)
    L = torch.exp(diff.masked_fill(~low, -1e4)).float()
    y = (L * (Cc @ Bc.transpose(-1, -2))) @ xd
    end = torch.exp(inner[..., -1:] - inner).float()[..., None]
    Z = (end * xd).transpose(-1, -2) @ Bc                     # [B, H, n, P, N]: what each chunk adds
    if S0 is not None:
        Z = torch.cat([S0[:, :, None], Z], 2)
    # the state before chunk c: what every part before it added, decayed by the chunks between
    total = inner[..., -1].cumsum(-1)                         # [B, H, n]
    zero = torch.zeros_like(total[..., :1])
    upto = torch.cat([zero, total], -1)                       # decay up to the start of chunk 0 .. n
    made = upto if S0 is not None else total                  # and up to where each part was added
    diff = upto[..., :, None] - made[..., None, :]
    at, by = torch.arange(n + 1, device=x.device)[:, None], torch.arange(made.shape[-1], device=x.device)[None]
    seen = by <= at if S0 is not None else by < at
    W = torch.exp(diff.masked_fill(~seen, -1e4)).float()
    S = (W @ Z.flatten(-2)).unflatten(-1, (P, N))             # [B, H, n + 1, P, N]
    y = y + torch.exp(inner).float()[..., None] * (Cc @ S[:, :, :n].transpose(-1, -2))
    y = y.movedim(1, 3).reshape(B, n * C, H, P)[:, :T]
    if D is not None:
        y = y + D[:, None] * x
    return _packed(s, y), S[:, :, n]


SSM_IN = ("x", "dt", "A", "Bm", "Cm", "D", "dt_bias", "S0")


def _run_plain_ssm(s):
    case = s["case"]
    dt = s["x"].dtype
    if case["kind"] == "ssm_step":
        rep = case["H"] // case["G"]
        x, d, Bm, Cm = (s[n].float() for n in ("x", "dt", "Bm", "Cm"))
        Bm, Cm = Bm.repeat_interleave(rep, 2), Cm.repeat_interleave(rep, 2)
        step = _softplus(d + s["dt_bias"])
        at = s["slots"].long()
        S = s["pool"][at]
        y = torch.empty_like(x)
        for t in range(case["T"]):
            S = torch.exp(step[:, t] * s["A"])[..., None, None] * S + (step[:, t, :, None] * x[:, t])[..., None] * Bm[:, t, :, None]
            y[:, t] = (S * Cm[:, t, :, None]).sum(-1)
        s["pool"][at] = S
        y = y if s["D"] is None else y + s["D"][:, None] * x
        return {"y": y.to(dt), "pool": s["pool"]}
    if case["kind"] == "ssm":
        y, S_T = _plain_ssm(s, *(None if s[n] is None else s[n].float() for n in SSM_IN))
        return {"y": y.to(dt), "S_T": S_T}
    leaves = _leaves(s, SSM_IN)
    y, S_T = _plain_ssm(s, *(leaf for _, leaf in leaves.values()))
    return {"y": y.detach().to(dt), "S_T": S_T.detach(), **_grads([(y, s["dy"]), (S_T, s["dS_T"])], leaves)}


# ---- the framework's calls ------------------------------------------------------------------


def _run_own(s):
    from paper_2606_27229_amd import carve

    case = s["case"]
    kind = case["kind"]
    if kind == "conv_step":
        y = carve.short_conv_step(s["x"], s["weight"], s["pool"], s["slots"], bias=s["bias"], activation=case["act"] or None)
        return {"y": y, "pool": s["pool"]}
    if kind.startswith("conv"):
        kw = {"bias": s["bias"], "activation": case["act"] or None, "offsets": s.get("offsets")}
        y, x_T = carve.short_conv_fwd(s["x"], s["weight"], s["x0"], **kw)
        out = {"y": y, "x_T": x_T}
        if kind == "conv_train":
            out.update(carve.short_conv_bwd(s["x"], s["weight"], s["dy"], s["x0"], s["dx_T"], **kw))
        return out
    if kind.startswith("rot"):
        kw = {"start": s["start"], "offsets": s.get("offsets"), "interleaved": case["interleaved"], "amplitude": s["amplitude"]}
        q, k = carve.rotary_fwd(s["q"], s["k"], s["freq"], **kw)
        out = {"q": q, "k": k}
        if kind == "rot_train":
            out["dq"], out["dk"] = carve.rotary_bwd(s["dq"], s["dk"], s["freq"], **kw)
        return out
    args = (s["x"], s["dt"], s["A"], s["Bm"], s["Cm"])
    kw = {"D": s["D"], "dt_bias": s["dt_bias"]}
    if kind == "ssm_step":
        y = carve.ssm_step(*args, s["pool"], s["slots"], **kw)
        return {"y": y, "pool": s["pool"]}
    kw["offsets"] = s.get("offsets")
    y, S_T, S_chunks = carve.ssm_chunk_fwd(*args, s["S0"], want_chunks=kind == "ssm_train", **kw)
    out = {"y": y, "S_T": S_T}
    if kind == "ssm_train":
        out.update(carve.ssm_chunk_bwd(*args, S_chunks, s["dy"], s["dS_T"], want_dS0=s["S0"] is not None, **kw))
    return out


def run(state):
    if own:
        return _run_own(state)
    kind = state["case"]["kind"]
    return _run_plain_conv(state) if kind.startswith("conv") else _run_plain_rot(state) if kind.startswith("rot") else _run_plain_ssm(state)


def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    kind, B, T = case["kind"], case["B"], case["T"]
    seqs = case["nseq"] or B
    if kind.startswith("conv"):
        C, W = case["C"], case["W"]
        keeps = 2 if kind == "conv_step" else 1 + case["state"]
        nbytes, flops = (2 * B * T + keeps * seqs * (W - 1)) * C * e, B * T * C * (2 * W + 4)
        if kind == "conv_train":   # dy, dx and the gradients of the kept inputs
            nbytes, flops = nbytes + (2 * B * T + 2 * case["state"] * seqs * (W - 1)) * C * e, 4 * flops
        return {"bytes": nbytes, "flops": flops}
    if kind.startswith("rot"):
        nbytes = 2 * B * T * (case["Hq"] + case["Hk"]) * case["Dh"] * e
        return {"bytes": nbytes * (2 if kind == "rot_train" else 1), "flops": nbytes // e * 2}
    G, H, N, P = (case[n] for n in ("G", "H", "N", "P"))
    tok = B * T * (2 * G * N + 2 * H * P + H) * e             # B, C, x, y, dt
    states = B * 2 if kind == "ssm_step" else seqs * (1 + case["state"])
    nbytes = tok + states * H * N * P * 4
    if kind == "ssm_step":
        return {"bytes": nbytes, "flops": B * T * H * N * P * 5}
    fwd = B * T * (G * 2 * CHUNK * N + H * (2 * CHUNK * P + 4 * N * P))
    if kind == "ssm_train":
        nbytes *= 2          # dy and the gradients of every input: as many bytes again
        fwd *= 3             # the forward's products and two for each of them
    return {"bytes": nbytes, "flops": fwd}


# ---- the definitions in 64 bits ----------------------------------------------------------------


def _sequences(s):
    """(batch index, first row, rows) of every sequence."""
    case = s["case"]
    if not case["nseq"]:
        return [(b, 0, case["T"]) for b in range(case["B"])]
    ends = list(itertools.accumulate(_lengths(case), initial=0))
    return [(0, a, b - a) for a, b in zip(ends, ends[1:])]


def _exact_conv(case, s):
    """Tap by tap and sequence by sequence."""
    W, T = case["W"], case["T"]
    w = s["weight"].double()
    bias = 0.0 if s["bias"] is None else s["bias"].double()
    step = case["kind"] == "conv_step"
    train = case["kind"] == "conv_train"
    y, dx = torch.zeros_like(s["x"], dtype=torch.float64), torch.zeros_like(s["x"], dtype=torch.float64)
    pool = s["pool"].double() if step else None
    slots = s["slots"].tolist() if step else None
    last, dw, db, d0 = [], torch.zeros_like(w), torch.zeros_like(w[:, 0]), []
    for i, (b, first, n) in enumerate(_sequences(s)):
        x = s["x"][b, first:first + n].double()
        old = pool[slots[i]] if step else torch.zeros_like(s["x"][0, :1]).double().expand(W - 1, -1) if s["x0"] is None else s["x0"][i].double()
        z = torch.cat([old, x])
        pre = bias + torch.zeros_like(x)
        for j in range(W):
            pre = pre + z[j:j + n] * w[:, j]
        sig = 1 / (1 + torch.exp(-pre))
        y[b, first:first + n] = pre * sig if case["act"] else pre
        if step:
            pool[slots[i]] = z[T:]
            continue
        last.append(z[n:])
        if train:
            dp = s["dy"][b, first:first + n].double()
            if case["act"]:
                dp = dp * sig * (1 + pre * (1 - sig))
            dz = torch.zeros_like(z)
            if s["dx_T"] is not None:
                dz[n:] += s["dx_T"][i].double()
            for j in range(W):
                dz[j:j + n] += dp * w[:, j]
                dw[:, j] += (dp * z[j:j + n]).sum(0)
            db += dp.sum(0)
            dx[b, first:first + n] = dz[W - 1:]
            d0.append(dz[:W - 1])
    if step:
        return {"y": y, "pool": pool}
    out = {"y": y, "x_T": torch.stack(last)}
    if train:
        out.update(dx=dx, dweight=dw)
        if s["bias"] is not None:
            out["dbias"] = db
        if s["x0"] is not None:
            out["dx0"] = torch.stack(d0)
    return out


def _exact_rot(case, s):
    """Complex numbers, multiplied by e^(i angle)."""
    half = case["rot"] // 2
    pos = torch.zeros(case["B"], case["T"], dtype=torch.float64, device="cuda")
    for i, (b, first, n) in enumerate(_sequences(s)):
        pos[b, first:first + n] = torch.arange(n, dtype=torch.float64, device="cuda") + s["start"][i].double()
    phase = torch.polar(torch.full_like(pos[..., None] * s["freq"], s["amplitude"]), pos[..., None] * s["freq"])[:, :, None]

    def turn(x, p):
        x = x.double()
        t = x[..., :2 * half]
        t = t.unflatten(-1, (half, 2)) if case["interleaved"] else t.unflatten(-1, (2, half)).transpose(-1, -2)
        t = torch.view_as_real(torch.view_as_complex(t.contiguous()) * p)
        t = t.flatten(-2) if case["interleaved"] else t.transpose(-1, -2).flatten(-2)
        return torch.cat([t, x[..., 2 * half:]], -1)

    out = {"q": turn(s["q"], phase), "k": turn(s["k"], phase)}
    if case["kind"] == "rot_train":
        out.update(dq=turn(s["dq"], phase.conj()), dk=turn(s["dk"], phase.conj()))
    return out


def _exact_ssm(case, s):
    """Token by token; the gradients backwards over the states kept."""
    G, H, N, P = (case[n] for n in ("G", "H", "N", "P"))
    rep = H // G
    train = case["kind"] == "ssm_train"

    def rows(x):
        x = x.double()
        if "rows" not in s:
            return x
        x = x[0, s["rows"].reshape(-1)].reshape(s["rows"].shape + x.shape[2:])
        return torch.where(s["there"].reshape(s["there"].shape + (1,) * (x.dim() - 2)), x, torch.zeros_like(x))

    x, raw = rows(s["x"]), rows(s["dt"]) + s["dt_bias"].double()
    Bm, Cm = rows(s["Bm"]).repeat_interleave(rep, 2), rows(s["Cm"]).repeat_interleave(rep, 2)
    n, T = x.shape[:2]
    A = s["A"].double()
    step = torch.logaddexp(raw, torch.zeros_like(raw))
    if "there" in s:
        step = torch.where(s["there"][..., None], step, torch.zeros_like(step))
    decay = torch.exp(step * A)
    if case["kind"] == "ssm_step":
        at = s["slots"].long()
        S = s["pool"][at].double()
    else:
        S = torch.zeros(n, H, P, N, device="cuda", dtype=torch.float64) if s["S0"] is None else s["S0"].double()
    keep = torch.empty(T, n, H, P, N, device="cuda", dtype=torch.float64) if train else None
    y = torch.zeros_like(x)
    for t in range(T):
        if train:
            keep[t] = S
        S = decay[:, t, :, None, None] * S + (step[:, t, :, None] * x[:, t])[..., None] * Bm[:, t, :, None, :]
        y[:, t] = (S @ Cm[:, t, ..., None])[..., 0]
    if s["D"] is not None:
        y = y + s["D"].double()[:, None] * x

    def flat(t):
        return t if "rows" not in s else t.reshape((-1,) + t.shape[2:])[s["back"]][None]

    if case["kind"] == "ssm_step":
        pool = s["pool"].double()
        pool[at] = S
        return {"y": y, "pool": pool}
    out = {"y": flat(y), "S_T": S}
    if not train:
        return out
    dy = rows(s["dy"])
    dS = torch.zeros_like(S) if s["dS_T"] is None else s["dS_T"].double()
    dx, dB, dC, dstep, da = (torch.zeros_like(t) for t in (x, Bm, Cm, step, step))
    after = S
    for t in range(T - 1, -1, -1):
        dS = dS + dy[:, t, ..., None] * Cm[:, t, :, None, :]
        dC[:, t] = (after.transpose(-1, -2) @ dy[:, t, ..., None])[..., 0]
        write = (dS @ Bm[:, t, ..., None])[..., 0]
        dx[:, t] = step[:, t, :, None] * write
        dstep[:, t] = (x[:, t] * write).sum(-1)
        dB[:, t] = step[:, t, :, None] * (dS.transpose(-1, -2) @ x[:, t, ..., None])[..., 0]
        after = keep[t]
        dS = decay[:, t, :, None, None] * dS
        da[:, t] = (dS * after).sum((-1, -2))
    dstep = dstep + A * da
    ddt = dstep / (1 + torch.exp(-raw))
    if "there" in s:
        ddt = torch.where(s["there"][..., None], ddt, torch.zeros_like(ddt))
    if s["D"] is not None:
        out["dD"] = (dy * x).sum((0, 1, 3))
        dx = dx + s["D"].double()[:, None] * dy
    out.update(dx=flat(dx), ddt=flat(ddt), dA=(step * da).sum((0, 1)), ddt_bias=ddt.sum((0, 1)))
    out.update(dBm=flat(dB.unflatten(2, (G, rep)).sum(3)), dCm=flat(dC.unflatten(2, (G, rep)).sum(3)))
    if s["S0"] is not None:
        out["dS0"] = dS
    return out


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "ssm_train" and (max(_lengths(case)) if case["nseq"] else case["T"]) * (case["nseq"] or case["B"]) * case["H"] * case["N"] * case["P"] * 8 > 90e9:
        return None
    return _exact_conv(case, s) if kind.startswith("conv") else _exact_rot(case, s) if kind.startswith("rot") else _exact_ssm(case, s)
