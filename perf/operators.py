"""Performance cases of the gated delta rule and of the block norm: the calls a
program that trains or serves such layers makes.

A case is a dict of plain values.  "kind" says which call:
  step   T tokens for each of B sequences on their states in a pool of `pool`
         states, updated in place (decoding; T > 1: drafted tokens)
  fwd    the chunked forward: outputs and final states (prefill)
  train  the chunked forward and its backward
  norm   the block norm's forward (serving)
  norm_train  its forward and backward
Token cases: B, T, Hk, Hv, Dk, Dv, dtype, state (a carried start state), nseq
(0: B sequences of T tokens; n: n sequences of unequal lengths, some of them
empty or of one token, packed into T rows, their lengths made from `cut`).
Norm cases: rows, N, groups, dtype, gate ("", "silu", "sigmoid"), residual,
scale, next (whether the next block's norm follows).
"""
from __future__ import annotations

import itertools
import random

import torch

own = False

EPS = 1e-6
ALPHA = 0.75        # residual multiplier of the norm cases that have a residual
CHUNK = 64          # chunk of the plain form


def _tok(name, kind, B, T, Hk, Hv, Dk, Dv, dtype="bf16", state=False, nseq=0, cut=0, pool=0):
    return {"name": name, "kind": kind, "B": B, "T": T, "Hk": Hk, "Hv": Hv, "Dk": Dk, "Dv": Dv, "dtype": dtype,
            "state": state, "nseq": nseq, "cut": cut, "pool": pool}


def _norm(name, kind, rows, N, groups=1, dtype="bf16", gate="", residual=True, scale=True, next=True):
    return {"name": name, "kind": kind, "rows": rows, "N": N, "groups": groups, "dtype": dtype, "gate": gate,
            "residual": residual, "scale": scale, "next": next}


def listed():
    return [
        # one sequence of a small server answers token by token: latency
        _tok("step_one", "step", 1, 1, 16, 16, 128, 128, pool=1),
        # a full decoding batch, value heads sharing key heads, states scattered over the pool
        _tok("step_batch", "step", 64, 1, 16, 32, 128, 128, pool=96),
        # four drafted tokens a sequence, a small f32 model
        _tok("step_draft_f32", "step", 24, 4, 8, 8, 64, 64, dtype="f32", pool=24),
        # prompts of unequal lengths arriving together, some continuing from a state
        _tok("fwd_ragged", "fwd", 1, 1777, 8, 16, 128, 128, state=True, nseq=9, cut=3),
        # prefill at the 1.3B-scale layer's shape
        _tok("fwd_layer", "fwd", 4, 4096, 16, 16, 128, 128),
        # one long document, its length no multiple of anything
        _tok("fwd_long", "fwd", 1, 16381, 16, 16, 128, 128, state=True),
        # a small f32 layer trained from a carried state (as in tests)
        _tok("train_f32_small", "train", 2, 200, 4, 4, 64, 64, dtype="f32", state=True),
        # a training step at the 1.3B-scale layer's shape
        _tok("train_layer", "train", 4, 4096, 16, 16, 128, 128),
        # documents packed into one row, four value heads a key head, narrow keys
        _tok("train_packed", "train", 1, 8191, 4, 16, 64, 128, nseq=5, cut=1),
        # the norm / gate / residual between two blocks, one decoding batch
        _norm("norm_decode", "norm", 64, 2048, gate="sigmoid"),
        # the same in a training step of 16384 tokens
        _norm("norm_layer", "norm_train", 16384, 2048, gate="sigmoid"),
        # the gated norm of every head's output, before the output projection
        _norm("norm_heads", "norm_train", 16381, 2048, groups=16, gate="silu", residual=False, scale=False, next=False),
    ]


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    kind = rng.choice(("step", "step", "fwd", "fwd", "train", "train", "norm", "norm_train"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    if kind.startswith("norm"):
        groups = rng.choice((1, 1, 8, 32))
        N = groups * rng.choice((64, 128)) if groups > 1 else 8 * _log(rng, 16, 512)
        rows = min(_log(rng, 1, 16384), 16384 * 2048 // N)
        return _norm("", kind, rows, N, groups, dtype, rng.choice(("", "silu", "sigmoid")), rng.random() < 0.7,
                     rng.random() < 0.5, rng.random() < 0.5)
    Hk = rng.choice((1, 2, 4, 8, 16))
    Hv = min(32, Hk * rng.choice((1, 1, 2, 4)))
    Dk, Dv = rng.choice((32, 64, 128)), rng.choice((32, 64, 128))
    if kind == "step":
        B, T = _log(rng, 1, 64), rng.choice((1, 1, 1, 2, 3, 5, 8))
        return _tok("", kind, B, T, Hk, Hv, Dk, Dv, dtype, True, pool=B + rng.randrange(0, 17))
    # tokens of all sequences, so that a case costs no more than the largest listed one
    most = max(64, int((16384 if dtype == "bf16" else 4096) * (16 * 128 * 128) / (Hv * Dk * Dv)))
    total = _log(rng, 1, min(most, 16384))
    nseq = rng.choice((0, 0, rng.randrange(1, 12)))
    B = 1 if nseq else rng.choice([b for b in (1, 1, 2, 3, 4, 8) if b <= total])
    return _tok("", kind, B, max(1, total // B), Hk, Hv, Dk, Dv, dtype, rng.random() < 0.5, nseq, rng.randrange(1000))


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


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32

    def randn(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    s = {"case": case}
    if case["kind"].startswith("norm"):
        rows, N = case["rows"], case["N"]
        s["y"] = (randn(rows, N) * torch.exp(randn(rows, 1))).to(dt)
        s["weight"] = 1 + 0.1 * randn(N)
        s["gate"] = randn(rows, N).to(dt) if case["gate"] else None
        s["residual"] = (2 * randn(rows, N)).to(dt) if case["residual"] else None
        s["scale"] = 0.5 + 0.2 * randn(N) if case["scale"] else None
        s["next_weight"] = 1 + 0.1 * randn(N) if case["next"] else None
        if case["kind"] == "norm_train":
            s["dx"] = randn(rows, N).to(dt)
            s["dh"] = randn(rows, N).to(dt) if case["next"] else None
        return s
    B, T, Hk, Hv, Dk, Dv = (case[x] for x in ("B", "T", "Hk", "Hv", "Dk", "Dv"))
    # unit queries and keys, decays of a few to a few hundred tokens, write strengths in (0, 1)
    s["q"], s["k"] = (torch.nn.functional.normalize(randn(B, T, Hk, Dk), dim=-1).to(dt) for _ in range(2))
    s["v"] = randn(B, T, Hv, Dv).to(dt)
    s["g"] = -torch.nn.functional.softplus(1.5 * randn(B, T, Hv) - 3)
    s["beta"] = torch.sigmoid(randn(B, T, Hv)).to(dt)
    seqs = case["nseq"] or B
    if case["kind"] == "step":
        s["pool"] = 0.3 * randn(case["pool"], Hv, Dv, Dk)
        order = list(range(case["pool"]))
        random.Random(int(seed)).shuffle(order)
        s["slots"] = torch.tensor(order[:B], dtype=torch.int32, device="cuda")
        return s
    s["S0"] = 0.3 * randn(seqs, Hv, Dv, Dk) if case["state"] else None
    if case["nseq"]:
        lens = _lengths(case)
        offsets = list(itertools.accumulate(lens, initial=0))
        s["offsets"] = torch.tensor(offsets, dtype=torch.int32, device="cuda")
        # each sequence's rows in a padded batch, and back (the plain form's layout)
        most = max(lens)
        row = torch.arange(most, device="cuda")
        start = s["offsets"][:-1].long()
        s["there"] = row[None] < (s["offsets"][1:].long() - start)[:, None]
        s["rows"] = torch.where(s["there"], start[:, None] + row[None], 0)
        s["back"] = s["there"].reshape(-1).nonzero()[:, 0]
    if case["kind"] == "train":
        s["dO"] = randn(B, T, Hv, Dv).to(dt)
        s["dS_T"] = 0.3 * randn(seqs, Hv, Dv, Dk) if case["state"] else None
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


def _unit_lower_inverse(A):
    """(I + A)^-1 of strictly lower A: diagonal blocks of 1, 2, 4, ... at a time, the
    lower one of each pair's corner being -T22 A21 T11."""
    C = A.shape[-1]
    at = torch.arange(C, device=A.device)
    inv, size = torch.eye(C, device=A.device).expand(A.shape), 1
    while size < C:
        pair = (at[:, None] // (2 * size) == at // (2 * size)) & (at[:, None] // size > at // size)
        inv = inv - inv @ (A * pair) @ inv
        size *= 2
    return inv


def _plain_chunks(s, q, k, v, g, beta, S0):
    """The chunk form in f32: outputs and final states.  Sums of decays and their
    differences are taken in 64 bits."""
    q, k, v, g, beta = (_padded(s, x.float()) for x in (q, k, v, g, beta))
    B, T, Hk, Dk = q.shape
    Hv, Dv = v.shape[2:]
    C = min(CHUNK, T)
    n = -(-T // C)

    def chunks(x):   # [B, T, H, ...] -> [B, Hv, n, C, ...]
        x = torch.nn.functional.pad(x, [0, 0] * (x.dim() - 2) + [0, n * C - T])
        x = x.reshape(B, n, C, *x.shape[2:]).movedim(3, 1)
        return x if x.shape[1] == Hv else x.repeat_interleave(Hv // x.shape[1], 1)

    q, k, v, g, beta = (chunks(x) for x in (q, k, v, g, beta))
    q = q * Dk ** -0.5
    G = g.double().cumsum(-1)
    low = torch.ones(C, C, dtype=torch.bool, device=q.device).tril()
    D = torch.exp((G[..., :, None] - G[..., None, :]).masked_fill(~low, -1e4)).float()
    gam, end = torch.exp(G).float()[..., None], torch.exp(G[..., -1:] - G).float()[..., None]
    beta = beta[..., None]
    A = (beta * D * (k @ k.transpose(-1, -2))).tril(-1)
    inv = _unit_lower_inverse(A)
    U0, W = inv @ (beta * v), inv @ (beta * gam * k)
    P = D * (q @ k.transpose(-1, -2))
    qg, ke = gam * q, end * k
    S = S0 if S0 is not None else torch.zeros(B, Hv, Dv, Dk, device=q.device)
    o = []
    for c in range(n):
        St = S.transpose(-1, -2)
        u = U0[:, :, c] - W[:, :, c] @ St
        o.append(qg[:, :, c] @ St + P[:, :, c] @ u)
        S = gam[:, :, c, -1:] * S + u.transpose(-1, -2) @ ke[:, :, c]
    o = torch.stack(o, 2).movedim(1, 3).reshape(B, n * C, Hv, Dv)[:, :T]
    return _packed(s, o), S


def _plain_step(s):
    case = s["case"]
    q, k, v, beta = (s[x].float() for x in ("q", "k", "v", "beta"))
    rep = case["Hv"] // case["Hk"]
    q, k = q.repeat_interleave(rep, 2) * case["Dk"] ** -0.5, k.repeat_interleave(rep, 2)
    slots = s["slots"].long()
    S = s["pool"][slots]
    o = []
    for t in range(case["T"]):
        S = S * torch.exp(s["g"][:, t, :, None, None])
        u = beta[:, t, :, None] * (v[:, t] - (S * k[:, t, :, None]).sum(-1))
        S = S + u[..., None] * k[:, t, :, None]
        o.append((S * q[:, t, :, None]).sum(-1))
    s["pool"][slots] = S
    return {"o": torch.stack(o, 1).to(s["q"].dtype), "pool": s["pool"]}


def _plain_norm(s, y, weight, gate, residual, scale, next_weight):
    case = s["case"]
    rows, N = y.shape
    yg = y.reshape(rows, case["groups"], -1)
    t = (yg * torch.rsqrt(yg.square().mean(-1, keepdim=True) + EPS)).reshape(rows, N) * weight
    if gate is not None:
        t = t * (torch.sigmoid(gate) * gate if case["gate"] == "silu" else torch.sigmoid(gate))
    if scale is not None:
        t = t * scale
    x = t if residual is None else ALPHA * residual + t
    h = None
    if next_weight is not None:
        h = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * next_weight
    return x, h


NORM_IN = ("y", "weight", "gate", "residual", "scale", "next_weight")


def _leaves(s, names):
    return [None if s[n] is None else s[n].float().requires_grad_() for n in names]


def _gradients(s, names, leaves, outs, grads):
    """d<grads, outs>/d leaves, each rounded to its input's type."""
    have = [(n, x) for n, x in zip(names, leaves) if x is not None]
    pairs = [(o, d.float()) for o, d in zip(outs, grads) if d is not None]
    got = torch.autograd.grad([o for o, _ in pairs], [x for _, x in have], [d for _, d in pairs])
    return {"d" + n: d.to(s[n].dtype) for (n, _), d in zip(have, got)}


def _run_plain(s):
    case = s["case"]
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    kind = case["kind"]
    if kind == "step":
        return _plain_step(s)
    if kind == "fwd":
        o, S_T = _plain_chunks(s, s["q"], s["k"], s["v"], s["g"], s["beta"], s["S0"])
        return {"o": o.to(dt), "S_T": S_T}
    if kind == "norm":
        x, h = _plain_norm(s, *(None if s[n] is None else s[n].float() for n in NORM_IN))
        return {"x": x.to(dt), "h": None if h is None else h.to(dt)}
    if kind == "norm_train":
        leaves = _leaves(s, NORM_IN)
        x, h = _plain_norm(s, *leaves)
        grads = _gradients(s, NORM_IN, leaves, (x, h), (s["dx"], s["dh"]))
        return {"x": x.detach().to(dt), "h": None if h is None else h.detach().to(dt), **grads}
    names = ("q", "k", "v", "g", "beta", "S0")
    leaves = _leaves(s, names)
    o, S_T = _plain_chunks(s, *leaves)
    grads = _gradients(s, names, leaves, (o, S_T), (s["dO"], s["dS_T"]))
    return {"o": o.detach().to(dt), "S_T": S_T.detach(), **grads}


# ---- the framework's calls ------------------------------------------------------------------


def _run_own(s):
    from paper_2606_27229_amd import carve

    case = s["case"]
    kind = case["kind"]
    if kind == "step":
        o = carve.gdr_step(s["q"], s["k"], s["v"], s["g"], s["beta"], s["pool"], s["slots"])
        return {"o": o, "pool": s["pool"]}
    if kind.startswith("norm"):
        kw = {"groups": case["groups"], "gate": s["gate"], "gate_act": case["gate"] or "silu", "residual": s["residual"],
              "alpha": ALPHA, "scale": s["scale"], "next_weight": s["next_weight"], "eps": EPS}
        x, h = carve.block_norm_fwd(s["y"], s["weight"], **kw)
        out = {"x": x, "h": h}
        if kind == "norm_train":
            out.update(carve.block_norm_bwd(s["y"], s["weight"], s["dx"], s["dh"], **kw))
        return out
    args = (s["q"], s["k"], s["v"], s["g"], s["beta"])
    kw = {"offsets": s.get("offsets")}
    o, S_T, S_chunks = carve.gdr_chunk_fwd(*args, s["S0"], want_chunks=kind == "train", **kw)
    out = {"o": o, "S_T": S_T}
    if kind == "train":
        out.update(carve.gdr_chunk_bwd(*args, S_chunks, s["dO"], s["dS_T"], want_dS0=s["S0"] is not None, **kw))
    return out


def run(state):
    if own:
        return _run_own(state)
    return _run_plain(state)


def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    if case["kind"].startswith("norm"):
        rows, N = case["rows"], case["N"]
        extra = bool(case["gate"]) + case["residual"]
        nbytes = rows * N * e * (2 + extra + case["next"])               # y, gate, residual; x, h
        if case["kind"] == "norm_train":
            nbytes += rows * N * e * (3 + 2 * extra + case["next"] - 1)  # dx, dh; dy, dgate, dresidual
        return {"bytes": nbytes, "flops": rows * N * (30 if case["kind"] == "norm_train" else 10)}
    B, T, Hk, Hv, Dk, Dv = (case[x] for x in ("B", "T", "Hk", "Hv", "Dk", "Dv"))
    tok = B * T * (2 * Hk * Dk * e + 2 * Hv * Dv * e + Hv * (4 + e))     # q, k, v, o, g, beta
    states = B * 2 if case["kind"] == "step" else (case["nseq"] or B) * (1 + case["state"])
    nbytes = tok + states * Hv * Dk * Dv * 4
    if case["kind"] == "step":
        return {"bytes": nbytes, "flops": B * T * Hv * Dk * Dv * 7}
    C = CHUNK
    fwd = B * T * (Hk * 2 * C * Dk + Hv * (2 * C * Dv + 6 * Dk * Dv))
    if case["kind"] == "train":
        nbytes *= 2          # dO and the gradients of every input: as many bytes again
        fwd *= 3.5           # the forward's products and two for each of them, some formed again
    return {"bytes": nbytes, "flops": fwd}


# ---- the definition in 64 bits ----------------------------------------------------------------


def _exact_tokens(s, tokens, S, keep):
    """Token by token: outputs, the final state and, with `keep`, the decayed state
    before every token's write."""
    q, k, v, g, beta = tokens
    o, before, errors = torch.zeros_like(v), [], []
    for t in range(q.shape[1]):
        S = torch.exp(g[:, t])[..., None, None] * S
        e = v[:, t] - (S @ k[:, t, ..., None])[..., 0]
        if keep is not None:
            keep[t] = S
            errors.append(e)
        S = S + (beta[:, t, :, None] * e)[..., None] * k[:, t, :, None]
        o[:, t] = (S @ q[:, t, ..., None])[..., 0]
    return o, S, errors


def _exact_norm(case, s):
    d = {n: None if s[n] is None else s[n].double() for n in NORM_IN}
    rows, N = s["y"].shape
    shape = (rows, case["groups"], N // case["groups"])
    r1 = (1 / (d["y"].reshape(shape).pow(2).mean(-1, keepdim=True) + EPS).sqrt()).expand(shape).reshape(rows, N)
    yh = d["y"] * r1
    nrm = yh * d["weight"]
    act, slope = torch.ones((), device="cuda", dtype=torch.float64), 0.0
    if d["gate"] is not None:
        sig = 1 / (1 + torch.exp(-d["gate"]))
        act = sig if case["gate"] == "sigmoid" else d["gate"] * sig
        slope = sig * (1 - sig) if case["gate"] == "sigmoid" else sig * (1 + d["gate"] * (1 - sig))
    sc = d["scale"] if d["scale"] is not None else torch.ones((), device="cuda", dtype=torch.float64)
    x = sc * nrm * act + (ALPHA * d["residual"] if d["residual"] is not None else 0)
    out = {"x": x, "h": None}
    if d["next_weight"] is not None:
        r2 = 1 / (x.pow(2).mean(-1, keepdim=True) + EPS).sqrt()
        out["h"] = x * r2 * d["next_weight"]
    if case["kind"] == "norm":
        return out
    dX = s["dx"].double()
    if d["next_weight"] is not None:
        dh = s["dh"].double()
        dn2 = dh * d["next_weight"]
        dX = dX + r2 * (dn2 - x * r2 * (dn2 * x * r2).mean(-1, keepdim=True))
        out["dnext_weight"] = (dh * x * r2).sum(0)
    if d["residual"] is not None:
        out["dresidual"] = ALPHA * dX
    if d["scale"] is not None:
        out["dscale"] = (dX * nrm * act).sum(0)
    dt = dX * sc
    if d["gate"] is not None:
        out["dgate"] = dt * nrm * slope
    dn = dt * act
    out["dweight"] = (dn * yh).sum(0)
    dnw = dn * d["weight"]
    dot = (dnw * yh).reshape(shape).mean(-1, keepdim=True).expand(shape).reshape(rows, N)
    out["dy"] = r1 * (dnw - yh * dot)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"].startswith("norm"):
        return _exact_norm(case, s)
    Hk, Hv, Dk, Dv = (case[x] for x in ("Hk", "Hv", "Dk", "Dv"))
    rep = Hv // Hk
    scale = float(Dk) ** -0.5

    def rows(x):
        x = x.double()
        if "rows" not in s:
            return x
        x = x[0, s["rows"].reshape(-1)].reshape(s["rows"].shape + x.shape[2:])
        return torch.where(s["there"].reshape(s["there"].shape + (1,) * (x.dim() - 2)), x, torch.zeros_like(x))

    q = scale * rows(s["q"]).repeat_interleave(rep, 2)
    k = rows(s["k"]).repeat_interleave(rep, 2)
    v, g, beta = rows(s["v"]), rows(s["g"]), rows(s["beta"])
    n, T = q.shape[:2]
    if case["kind"] == "step":
        at = s["slots"].long()
        o, S, _ = _exact_tokens(s, (q, k, v, g, beta), s["pool"][at].double(), None)
        pool = s["pool"].double()
        pool[at] = S
        return {"o": o, "pool": pool}
    train = case["kind"] == "train"
    if train and n * T * Hv * Dk * Dv * 8 > 90e9:
        return None
    S = torch.zeros(n, Hv, Dv, Dk, device="cuda", dtype=torch.float64) if s["S0"] is None else s["S0"].double()
    keep = torch.empty(T, n, Hv, Dv, Dk, device="cuda", dtype=torch.float64) if train else None
    o, S_T, errors = _exact_tokens(s, (q, k, v, g, beta), S, keep)

    def flat(x):
        return x if "rows" not in s else x.reshape((-1,) + x.shape[2:])[s["back"]][None]

    out = {"o": flat(o), "S_T": S_T}
    if not train:
        return out
    dO = rows(s["dO"])
    dS = torch.zeros_like(S_T) if s["dS_T"] is None else s["dS_T"].double()
    dq, dk, dv, dg, db = (torch.zeros_like(x) for x in (q, k, v, g, beta))
    for t in range(T - 1, -1, -1):
        before, e, kt, bt = keep[t], errors[t], k[:, t], beta[:, t, :, None]
        u = bt * e
        after = before + u[..., None] * kt[:, :, None]
        dS = dS + dO[:, t, ..., None] * q[:, t, :, None]
        dq[:, t] = (after.transpose(-1, -2) @ dO[:, t, ..., None])[..., 0] * scale
        du = (dS @ kt[..., None])[..., 0]
        de = bt * du
        db[:, t] = (du * e).sum(-1)
        dv[:, t] = de
        dk[:, t] = (dS.transpose(-1, -2) @ u[..., None] - before.transpose(-1, -2) @ de[..., None])[..., 0]
        dS = dS - de[..., None] * kt[:, :, None]
        dg[:, t] = (dS * before).sum((-1, -2))
        dS = torch.exp(g[:, t])[..., None, None] * dS

    def shared(x):
        return x.reshape(n, T, Hk, rep, Dk).sum(3)

    out.update(dq=flat(shared(dq)), dk=flat(shared(dk)), dv=flat(dv), dg=flat(dg), dbeta=flat(db))
    if s["S0"] is not None:
        out["dS0"] = dS
    return out
