"""Timed cases of the sequence operators: group norm with an activation, the short causal convolution and the selective
state space scan, all on tensors whose last extent is the channels.

A case is one operator in one form.  "train" is Forward and Backward, as one training step makes them; "fwd" is Forward
alone (inference, a prompt); "step" is the single-token form that decodes with a pool of states, updated in place.

  norm   x (N, S, C): N samples of S positions, C channels in G groups; statistics over a sample's positions and a
         group's channels; y = act(gamma * (x - mean) / sqrt(var + eps) + beta).  S = 1 is a norm of single tokens.
  conv   x (B, L, D), w (D, K): y_t = act(bias + sum_k w_k x_{t-K+1+k}), every channel by itself, zeros before the
         first token; the state is a sequence's last K - 1 tokens.
  scan   u, dt, z (B, L, D), A (D, N), Bm, Cm (B, L, G, N): d = softplus(dt + dt_bias),
         h_t = exp(d_t A) h_{t-1} + d_t u_t Bm_t, y_t = (Cm_t . h_t + skip u_t) * silu(z_t).

Sequences of one call have lengths of their own where "lengths" is true, zero and one among them: tokens behind a
length are padding, whose inputs hold anything and whose outputs and gradients are 0.
"""
import math
import random

import torch

own = False

EPS = 1e-5


def _norm(name, form, dtype, n, s, c, g, act):
    return {"name": name, "op": "norm", "form": form, "dtype": dtype, "N": n, "S": s, "C": c, "G": g, "act": act}


def _conv(name, form, dtype, b, l, d, k, lengths=False, half=False):
    return {"name": name, "op": "conv", "form": form, "dtype": dtype, "B": b, "L": l, "D": d, "K": k, "lengths": lengths,
            "half": half}


def _scan(name, form, dtype, b, l, d, n, g=1, gate=True, lengths=False):
    return {"name": name, "op": "scan", "form": form, "dtype": dtype, "B": b, "L": l, "D": d, "N": n, "G": g,
            "gate": gate, "lengths": lengths}


def listed():
    return [
        # one token of one sequence behind a scan's heads: the latency of a decoding step
        _norm("norm one token", "fwd", "bf16", 1, 1, 1024, 16, False),
        # the same norm in training, over the tokens of a batch
        _norm("norm tokens train", "train", "bf16", 8192, 1, 2048, 16, False),
        # feature maps of 32 x 32 behind a convolution, 32 groups, the activation fused
        _norm("norm images train", "train", "bf16", 64, 1024, 512, 32, True),
        # odd and ragged in every extent: 45 x 29 positions, three channels to a group, 32-bit tensors
        _norm("norm ragged train", "train", "f32", 37, 1305, 231, 77, True),
        # one token of each of 64 sequences
        _conv("conv step", "step", "bf16", 64, 1, 2048, 4),
        # a training batch; its input is one half of a projection's output
        _conv("conv train", "train", "bf16", 8, 2048, 2048, 4, half=True),
        # an odd number of channels, sequences of all lengths, 32-bit tensors
        _conv("conv ragged train", "train", "f32", 13, 1021, 509, 3, lengths=True),
        # one token of one sequence: latency
        _scan("scan one token", "step", "bf16", 1, 1, 2048, 16),
        # one token of each of 256 sequences: the states are what is read and written
        _scan("scan step", "step", "bf16", 256, 1, 4096, 16),
        # a training batch
        _scan("scan train", "train", "bf16", 8, 2048, 2048, 16),
        # one long prompt
        _scan("scan prompt", "fwd", "bf16", 1, 16384, 4096, 16),
        # two groups of an odd number of channels, 13 states, sequences of all lengths, 32-bit tensors
        _scan("scan ragged train", "train", "f32", 5, 677, 770, 13, g=2, gate=False, lengths=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


# elements of a tensor, and of all states of all tokens: those of the largest listed cases
_MOST, _MOST_STATES = 64 * 1024 * 512, {"train": 8 * 2048 * 2048 * 16, "fwd": 16384 * 4096 * 16}


def draw(rng):
    """Any operator in any form: single tokens to 16384 of them, 1 to 256 sequences, 32 to 8192 channels, bf16 twice as
    often as 32-bit tensors."""
    while True:
        op = rng.choice(["norm", "conv", "scan"])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        if op == "norm":
            g = rng.choice([1, 2, 8, 16, 32, 32, _log(rng, 3, 100)])
            c = g * max(1, _log(rng, 32, 8192) // g)
            s = 1 if rng.random() < 0.4 else _log(rng, 2, 16384)
            n = _log(rng, 1, 8192) if s == 1 else _log(rng, 1, 256)
            case = _norm("", rng.choice(["train", "train", "fwd"]), dtype, n, s, c, g, rng.random() < 0.6)
            size = n * s * c
        elif op == "conv":
            form = rng.choice(["train", "train", "fwd", "step"])
            b, d, k = _log(rng, 1, 256), _log(rng, 32, 8192), rng.choice([2, 3, 4, 4, 4, _log(rng, 5, 8)])
            l = 1 if form == "step" else _log(rng, 1, 16384)
            case = _conv("", form, dtype, b, l, d, k, form != "step" and rng.random() < 0.4, rng.random() < 0.3)
            size = b * l * d
        else:
            form = rng.choice(["train", "train", "fwd", "step"])
            n = rng.choice([16, 16, 16, 8, 32, 64, _log(rng, 3, 64)])
            g = rng.choice([1, 1, 1, 2, 4])
            d = g * max(1, _log(rng, 32, 8192) // g)
            l = 1 if form == "step" else _log(rng, 1, 16384)
            b = _log(rng, 1, 256)
            case = _scan("", form, dtype, b, l, d, n, g, rng.random() < 0.7, form != "step" and rng.random() < 0.4)
            size = b * l * d
            if size * n > _MOST_STATES.get(form, 256 * 4096 * 16):
                continue
        if size <= 2 * _MOST:
            del case["name"]
            return case


# ---- inputs --------------------------------------------------------------------------------------------------------


class _Random:
    def __init__(self, seed, dtype):
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(seed)
        self.dtype = torch.bfloat16 if dtype == "bf16" else torch.float32

    def normal(self, *shape, std=1.0):
        return torch.randn(shape, device="cuda", generator=self.gen).mul_(std)

    def uniform(self, *shape, lo=0.0, hi=1.0):
        return torch.rand(shape, device="cuda", generator=self.gen).mul_(hi - lo).add_(lo)

    def tokens(self, *shape, std=1.0):
        return self.normal(*shape, std=std).to(self.dtype)


def _lengths(case, seed):
    """Lengths of all sizes: a full sequence, one of a single token, an empty one, the others in between."""
    if not case["lengths"]:
        return None
    rng = random.Random(seed)
    got = [case["L"], 1, 0][:case["B"]]
    got += [rng.randint(0, case["L"]) for _ in range(case["B"] - len(got))]
    rng.shuffle(got)
    return torch.tensor(got, dtype=torch.int32, device="cuda")


def _slots(case, seed):
    """A place in the pool for each sequence, in any order; the pool has a few more."""
    order = list(range(case["B"] + 3))
    random.Random(seed).shuffle(order)
    return torch.tensor(order[:case["B"]], dtype=torch.int32, device="cuda")


def prepare(case, seed):
    r = _Random(seed, case["dtype"])
    state = {"case": dict(case)}
    if case["op"] == "norm":
        shape = (case["N"], case["S"], case["C"])
        # features with a mean and a scale of their own per channel
        state["x"] = (r.normal(*shape) * r.uniform(case["C"], lo=0.5, hi=2.0) + r.normal(case["C"], std=0.5)).to(r.dtype)
        state["gamma"], state["beta"] = 1.0 + r.normal(case["C"], std=0.2), r.normal(case["C"], std=0.2)
        if case["form"] == "train":
            state["dy"] = r.tokens(*shape, std=0.1)
        return state
    b, l, d = case["B"], case["L"], case["D"]
    state["lengths"] = None if case["form"] == "step" else _lengths(case, seed)
    if case["form"] == "step":
        state["slots"] = _slots(case, seed)
    if case["op"] == "conv":
        k = case["K"]
        state["x"] = r.tokens(b, l, 2 * d)[:, :, :d] if case["half"] else r.tokens(b, l, d)
        state["w"], state["bias"] = r.tokens(d, k, std=1.0 / math.sqrt(k)), r.normal(d, std=0.2)
        if case["form"] == "step":
            state["state"] = r.tokens(b + 3, k - 1, d)
    else:
        n, g = case["N"], case["G"]
        u = r.normal(b, l, d)
        state["u"] = (u / (1 + torch.exp(-u))).to(r.dtype)           # what the convolution's activation gives
        state["dt"] = r.tokens(b, l, d, std=0.5)
        step = torch.exp(r.uniform(d, lo=math.log(1e-3), hi=math.log(1e-1)))
        state["dt_bias"] = step + torch.log(-torch.expm1(-step))     # softplus(dt_bias) spans 0.001 to 0.1
        state["A"] = -torch.arange(1, n + 1, device="cuda") * r.uniform(d, n, lo=0.7, hi=1.3)
        state["Bm"], state["Cm"] = r.tokens(b, l, g, n), r.tokens(b, l, g, n)
        state["skip"] = 1.0 + r.normal(d, std=0.1)
        state["z"] = r.tokens(b, l, d) if case["gate"] else None
        if case["form"] == "step":
            state["state"] = r.normal(b + 3, d, n, std=0.3)
    if case["form"] == "train":
        state["dy"] = r.tokens(b, l, d, std=0.1)
    if state["lengths"] is not None:  # what stands behind a sequence's end is anything
        behind = torch.arange(l, device="cuda")[None, :] >= state["lengths"][:, None]
        for name in ("x", "u", "dt", "Bm", "Cm", "z", "dy"):
            if state.get(name) is not None:
                state[name][behind] = float("nan")
    return state


def run(state):
    form = globals()["_%s_%s" % ("own" if own else "plain", state["case"]["op"])]
    return form(state)


# ---- plain forms ---------------------------------------------------------------------------------------------------


def _sigmoid(v):
    return 1 / (1 + torch.exp(-v))


def _plain_norm(state):
    case, x = state["case"], state["x"].float()
    n, s, c, g = (case[k] for k in ("N", "S", "C", "G"))
    gamma, beta = (state[k].view(1, 1, g, c // g) for k in ("gamma", "beta"))
    xg = x.view(n, s, g, c // g)
    centred = xg - xg.mean((1, 3), keepdim=True)
    rstd = 1 / torch.sqrt((centred * centred).mean((1, 3), keepdim=True) + EPS)
    xhat = centred * rstd
    u = xhat * gamma + beta
    kind = state["x"].dtype
    sig = _sigmoid(u) if case["act"] else None
    out = {"y": (u * sig if case["act"] else u).view(n, s, c).to(kind)}
    if case["form"] == "train":
        du = state["dy"].float().view_as(u)
        if case["act"]:
            du = du * (sig * (1 + u * (1 - sig)))
        dxhat = du * gamma
        mean1, mean2 = dxhat.mean((1, 3), keepdim=True), (dxhat * xhat).mean((1, 3), keepdim=True)
        out["dx"] = (rstd * (dxhat - mean1 - xhat * mean2)).view(n, s, c).to(kind)
        out["dgamma"], out["dbeta"] = (du * xhat).sum((0, 1)).view(c), du.sum((0, 1)).view(c)
    return out


def _valid(state, like):
    """Truth values (B, L, 1, ...) of the tokens that are not padding."""
    at = torch.arange(like.shape[1], device="cuda")[None, :] < state["lengths"][:, None]
    return at.view(at.shape + (1,) * (like.dim() - 2))


def _tokens(state, name):
    """A (B, L, ...) input in 32 bits, padding as 0."""
    v = state[name].float()
    return v if state["lengths"] is None else torch.where(_valid(state, v), v, torch.zeros((), device="cuda"))


def _plain_conv(state):
    case, kind = state["case"], state["x"].dtype
    k, l = case["K"], case["L"]
    x, w = _tokens(state, "x"), state["w"].float()
    if case["form"] == "step":
        slots = state["slots"].long()
        before = state["state"][slots].float()
    else:
        before = torch.zeros_like(x[:, :1]).expand(-1, k - 1, -1)
    xs = torch.cat([before, x], 1)
    windows = xs.unfold(1, k, 1)                           # (B, L, D, K)
    u = (windows * w).sum(-1) + state["bias"]
    sig = _sigmoid(u)
    y = u * sig
    if case["form"] == "step":
        state["state"][slots] = xs[:, 1:].to(kind)
        return {"y": y.to(kind), "state": state["state"]}
    if state["lengths"] is not None:
        y = torch.where(_valid(state, y), y, torch.zeros((), device="cuda"))
        last = state["lengths"].long()[:, None] + torch.arange(k - 1, device="cuda")
        tail = torch.gather(xs, 1, last[:, :, None].expand(-1, -1, xs.shape[2]))
    else:
        tail = xs[:, l:]
    out = {"y": y.to(kind), "state": tail.to(kind)}
    if case["form"] == "train":
        du = _tokens(state, "dy") * (sig * (1 + u * (1 - sig)))
        out["dw"], out["dbias"] = (windows * du[..., None]).sum((0, 1)), du.sum((0, 1))
        after = torch.cat([du, torch.zeros_like(du[:, :1]).expand(-1, k - 1, -1)], 1)
        dx = (after.unfold(1, k, 1) * w.flip(1)).sum(-1)
        if state["lengths"] is not None:
            dx = torch.where(_valid(state, dx), dx, torch.zeros((), device="cuda"))
        out["dx"] = dx.to(kind)
    return out


def _recurrence(a, b):
    """h_t = a_t h_{t-1} + b_t along dim 1, h_{-1} = 0: pairs of steps are joined, then pairs of pairs."""
    step = 1
    while step < a.shape[1]:
        b = torch.cat([b[:, :step], b[:, step:] + a[:, step:] * b[:, :-step]], 1)
        if 2 * step < a.shape[1]:
            a = torch.cat([a[:, :step], a[:, step:] * a[:, :-step]], 1)
        step *= 2
    return b


def _plain_scan(state):
    case, kind = state["case"], state["u"].dtype
    d, n, g = case["D"], case["N"], case["G"]
    u = _tokens(state, "u")
    raw = _tokens(state, "dt") + state["dt_bias"]
    delta = torch.where(raw > 20, raw, torch.log1p(torch.exp(raw)))
    if state["lengths"] is not None:
        delta = torch.where(_valid(state, delta), delta, torch.zeros((), device="cuda"))
    shape = u.shape[:2] + (g, d // g, n)
    a = torch.exp(delta[..., None] * state["A"]).view(shape)
    bm, cm = _tokens(state, "Bm")[:, :, :, None], _tokens(state, "Cm")[:, :, :, None]   # (B, L, G, 1, N)
    du = (delta * u).view(shape[:-1] + (1,))
    b = du * bm
    if case["form"] == "step":
        slots = state["slots"].long()
        h = a * state["state"][slots].view((-1, 1) + shape[2:]) + b
    else:
        h = _recurrence(a, b)
    y = (h * cm).sum(-1).view(u.shape) + state["skip"] * u
    pre = y
    if case["gate"]:
        z = _tokens(state, "z")
        sig = _sigmoid(z)
        y = y * (z * sig)
    last = h[:, -1].reshape(-1, d, n)
    if case["form"] == "step":
        state["state"][slots] = last
        return {"y": y.to(kind), "state": state["state"]}
    out = {"y": y.to(kind), "state": last}
    if case["form"] == "train":
        dy = _tokens(state, "dy")
        if case["gate"]:
            out["dz"] = (dy * pre * (sig * (1 + z * (1 - sig)))).to(kind)
            dy = dy * (z * sig)
        dyg = dy.view(shape[:-1] + (1,))
        # dh_t = Cm_t dy_t + a_{t+1} dh_{t+1}
        after = torch.cat([a[:, 1:], torch.zeros_like(a[:, :1])], 1).flip(1)
        dh = _recurrence(after, (dyg * cm).flip(1)).flip(1)
        out["dBm"], out["dCm"] = (dh * du).sum(3).to(kind), (dyg * h).sum(3).to(kind)
        grown = (dh * bm).sum(-1).view(u.shape)
        decay = dh[:, 1:] * a[:, 1:] * h[:, :-1]                            # with respect to d_t A
        decay = torch.cat([torch.zeros_like(dh[:, :1]), decay], 1).view(u.shape + (n,))
        out["dA"] = (decay * delta[..., None]).sum((0, 1))
        out["dskip"] = (dy * u).sum((0, 1))
        out["du"] = (grown * delta + dy * state["skip"]).to(kind)
        ddelta = ((decay * state["A"]).sum(-1) + grown * u) * _sigmoid(raw)
        out["ddt_bias"] = ddelta.sum((0, 1))
        out["ddt"] = ddelta.to(kind)
    return out


# ---- the framework's operators -------------------------------------------------------------------------------------


def _workspace(nbytes):
    return torch.empty(nbytes, dtype=torch.uint8, device="cuda") if nbytes else None


def _dtype(state):
    return 1 if state["case"]["dtype"] == "bf16" else 0


def _own_norm(state):
    from paper_1804_04806_amd import seq
    case, x = state["case"], state["x"]
    train = case["form"] == "train"
    if "desc" not in state:
        desc = seq.group_norm(N=case["N"], S=case["S"], C=case["C"], G=case["G"], eps=EPS,
                              act=seq.ACT_SILU if case["act"] else seq.ACT_NONE, dtype=_dtype(state))
        state["ws"] = _workspace(max(seq.ucd_group_norm_workspace_size(desc, op)
                                     for op in ((seq.FWD, seq.BWD) if train else (seq.FWD,))))
        state["y"] = torch.empty_like(x)
        if train:
            state["stats"] = torch.empty(2, case["N"], case["G"], device="cuda")
            state["dx"], state["dgamma"], state["dbeta"] = (torch.empty_like(state[k]) for k in ("x", "gamma", "beta"))
        state["desc"] = desc
    desc = state["desc"]
    seq.ucd_group_norm_fwd(desc, x, state["gamma"], state["beta"], state["y"], state.get("stats"), ws=state["ws"])
    out = {"y": state["y"]}
    if train:
        seq.ucd_group_norm_bwd(desc, x, state["gamma"], state["beta"], state["stats"], state["dy"], state["dx"],
                               state["dgamma"], state["dbeta"], ws=state["ws"])
        out.update({k: state[k] for k in ("dx", "dgamma", "dbeta")})
    return out


def _own_conv(state):
    from paper_1804_04806_amd import seq
    case, x, w, bias = state["case"], state["x"], state["w"], state["bias"]
    if "desc" not in state:
        step = case["form"] == "step"
        desc = seq.causal_conv(B=case["B"], L=case["L"], D=case["D"], K=case["K"], act=seq.ACT_SILU, dtype=_dtype(state),
                               n_slots=case["B"] + 3 if step else 0, x_stride=x.stride()[:2])
        state["y"] = torch.empty(x.shape, dtype=x.dtype, device="cuda")
        if not step:
            state["tail"] = torch.empty(case["B"], case["K"] - 1, case["D"], dtype=x.dtype, device="cuda")
        if case["form"] == "train":
            state["ws"] = _workspace(seq.ucd_causal_conv_workspace_size(desc))
            state["dx"] = torch.empty_strided(x.shape, x.stride(), dtype=x.dtype, device="cuda")
            state["dw"], state["dbias"] = torch.empty(w.shape, device="cuda"), torch.empty_like(bias)
        state["desc"] = desc
    desc = state["desc"]
    if case["form"] == "step":
        seq.ucd_causal_conv_step(desc, x, w, bias, state["state"], state["y"], slots=state["slots"])
        return {"y": state["y"], "state": state["state"]}
    seq.ucd_causal_conv_fwd(desc, x, w, bias, state["y"], lengths=state["lengths"], state_out=state["tail"])
    out = {"y": state["y"], "state": state["tail"]}
    if case["form"] == "train":
        seq.ucd_causal_conv_bwd(desc, x, w, bias, state["dy"], state["dx"], state["dw"], state["dbias"],
                                lengths=state["lengths"], ws=state["ws"])
        out.update({k: state[k] for k in ("dx", "dw", "dbias")})
    return out


def _own_scan(state):
    from paper_1804_04806_amd import seq
    case = state["case"]
    step, train = case["form"] == "step", case["form"] == "train"
    if "desc" not in state:
        desc = seq.scan(B=case["B"], L=case["L"], D=case["D"], N=case["N"], G=case["G"], dtype=_dtype(state), softplus=True,
                        n_slots=case["B"] + 3 if step else 0)
        state["y"] = torch.empty_like(state["u"])
        if not step:
            state["last"] = torch.empty(case["B"], case["D"], case["N"], device="cuda")
            state["ws"] = _workspace(max(seq.ucd_scan_workspace_size(desc, op)
                                         for op in ((seq.FWD, seq.BWD) if train else (seq.FWD,))))
        if train:
            state["saved"] = _workspace(seq.ucd_scan_saved_size(desc))
            for name in ("u", "dt", "A", "Bm", "Cm", "skip", "z", "dt_bias"):
                state["d" + name] = None if state[name] is None else torch.empty_like(state[name])
        state["desc"] = desc
    desc = state["desc"]
    inputs = [state[k] for k in ("u", "dt", "A", "Bm", "Cm")]
    more = {k: state[k] for k in ("skip", "z", "dt_bias")}
    if step:
        seq.ucd_scan_step(desc, *inputs, state["state"], state["y"], slots=state["slots"], **more)
        return {"y": state["y"], "state": state["state"]}
    more["lengths"] = state["lengths"]
    seq.ucd_scan_fwd(desc, *inputs, state["y"], state_out=state["last"], saved=state.get("saved"), ws=state["ws"], **more)
    out = {"y": state["y"], "state": state["last"]}
    if train:
        seq.ucd_scan_bwd(desc, *inputs, state["dy"], state["saved"], *(state["d" + k] for k in ("u", "dt", "A", "Bm", "Cm")),
                         dskip=state["dskip"], dz=state["dz"], ddt_bias=state["ddt_bias"], ws=state["ws"], **more)
        out.update({"d" + k: state["d" + k] for k in ("u", "dt", "A", "Bm", "Cm", "skip", "z", "dt_bias")
                    if state["d" + k] is not None})
    return out


# ---- what a pass cannot do without ---------------------------------------------------------------------------------


def work(case):
    """Bytes: each input once, each output once.  Flops: multiplications, additions and exponentials of the formulas, one
    each.  Lengths are not counted: a case with them has at most this work."""
    e = 2 if case["dtype"] == "bf16" else 4
    train = case["form"] == "train"
    if case["op"] == "norm":
        m, c = case["N"] * case["S"] * case["C"], case["C"]
        act = 4 if case["act"] else 0
        return {"bytes": (4 if train else 2) * m * e + (16 if train else 8) * c,
                "flops": m * (7 + act + (12 + 2 * act if train else 0))}
    b, l, d = case["B"], case["L"], case["D"]
    m = b * l * d
    if case["op"] == "conv":
        k = case["K"]
        state = b * (k - 1) * d * e * (2 if case["form"] == "step" else 1)
        return {"bytes": (4 if train else 2) * m * e + state + d * (k * e + 4) + (d * (k + 1) * 4 if train else 0),
                "flops": m * (2 * k + 4 + (4 * k + 8 if train else 0))}
    n, g = case["N"], case["G"]
    tokens = (3 + case["gate"]) * m * e + 2 * b * l * g * n * e            # u, dt, y, z, Bm, Cm
    state = b * d * n * 4 * (2 if case["form"] == "step" else 1)
    weights = d * (n + 2) * 4
    if train:  # dy too; du, ddt, dz, dBm, dCm and the gradients of the weights
        tokens += (3 + case["gate"]) * m * e + 2 * b * l * g * n * e
        weights *= 2
    return {"bytes": tokens + state + weights, "flops": m * (n * (7 + (17 if train else 0)) + 14 + (30 if train else 0))}


# ---- in 64 bits ----------------------------------------------------------------------------------------------------


def exact(case, seed):
    """The definitions in 64 bits, gradients by automatic differentiation, the recurrence token by token."""
    state = prepare(case, seed)
    train = case["form"] == "train"
    v = {k: t.double() for k, t in state.items() if isinstance(t, torch.Tensor) and t.is_floating_point()}
    if case["form"] != "step" and state.get("lengths") is not None:
        keep = torch.arange(case["L"], device="cuda")[None, :] < state["lengths"][:, None]
        for name in ("x", "u", "dt", "Bm", "Cm", "z", "dy"):
            if name in v:
                v[name][~keep] = 0
    else:
        keep = None
    wanted = {"norm": ("x", "gamma", "beta"), "conv": ("x", "w", "bias"),
              "scan": ("u", "dt", "A", "Bm", "Cm", "skip", "z", "dt_bias")}[case["op"]]
    wanted = [name for name in wanted if name in v]
    with torch.set_grad_enabled(train):
        for name in wanted:
            v[name].requires_grad_(train)
        out = {"norm": _exact_norm, "conv": _exact_conv, "scan": _exact_scan}[case["op"]](case, state, v, keep)
    if train:
        grads = torch.autograd.grad(out["y"], [v[name] for name in wanted], v["dy"])
        out.update({"d" + name: grad for name, grad in zip(wanted, grads)})
    return {name: t.detach() for name, t in out.items()}


def _exact_norm(case, state, v, keep):
    n, s, c, g = (case[k] for k in ("N", "S", "C", "G"))
    x = v["x"].reshape(n, s, g, c // g).transpose(1, 2).reshape(n, g, -1)
    var, mean = torch.var_mean(x, 2, correction=0, keepdim=True)
    x = ((x - mean) * (var + EPS).rsqrt()).reshape(n, g, s, c // g).transpose(1, 2).reshape(n, s, c)
    y = v["gamma"] * x + v["beta"]
    return {"y": torch.nn.functional.silu(y) if case["act"] else y}


def _exact_conv(case, state, v, keep):
    k, l = case["K"], case["L"]
    y = v["bias"].expand(case["B"], l, case["D"])
    if case["form"] == "step":
        slots = state["slots"].long()
        before = torch.cat([v["state"][slots], v["x"]], 1)
    else:
        before = torch.nn.functional.pad(v["x"], (0, 0, k - 1, 0))
    for tap in range(k):
        y = y + before[:, tap:tap + l] * v["w"][:, tap]
    y = torch.nn.functional.silu(y)
    if case["form"] == "step":
        pool = v["state"].clone()
        pool[slots] = before[:, 1:]
        return {"y": y, "state": pool}
    if keep is None:
        return {"y": y, "state": before[:, l:]}
    tails = [row[n:n + k - 1] for row, n in zip(before, state["lengths"].tolist())]
    return {"y": y * keep[:, :, None], "state": torch.stack(tails)}


def _exact_scan(case, state, v, keep):
    b, d, n, g = (case[k] for k in ("B", "D", "N", "G"))
    delta = torch.nn.functional.softplus(v["dt"] + v["dt_bias"], threshold=40)
    if keep is not None:
        delta = delta * keep[:, :, None]
    if case["form"] == "step":
        slots = state["slots"].long()
        h = v["state"][slots]
    else:
        h = torch.zeros(b, d, n, dtype=torch.float64, device="cuda")
    shape = (b, g, d // g, n)
    steps = zip(delta.unbind(1), (delta * v["u"]).unbind(1), v["Bm"].unbind(1), v["Cm"].unbind(1))
    y = []
    for delta_t, gain, bm, cm in steps:
        h = torch.exp(delta_t[:, :, None] * v["A"]) * h + (gain.reshape(shape[:3] + (1,)) * bm[:, :, None]).reshape(b, d, n)
        y.append((h.reshape(shape) * cm[:, :, None]).sum(-1).reshape(b, d))
    y = torch.stack(y, 1) + v["skip"] * v["u"]
    if case["gate"]:
        y = y * torch.nn.functional.silu(v["z"])
    if case["form"] == "step":
        pool = v["state"].clone()
        pool[slots] = h
        return {"y": y, "state": pool}
    return {"y": y, "state": h}
