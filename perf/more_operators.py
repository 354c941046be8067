"""Timed cases of two more operators of a sequence model's layer: linear attention with a decay for each head, and the gated
projection of a feed-forward block.

A case is one operator in one form.  "train" is Forward and Backward, as one training step makes them; "fwd" is Forward
alone (inference, a prompt); "step" is the single-token form that decodes with a pool of states, updated in place.

  attention  q, k (B, L, Hk, Dk), v (B, L, H, Dv): each of the Hk heads of q and k serves H / Hk neighbouring heads of v.
             S_t = exp(l_t) S_{t-1} + k_t^T v_t,  y_t = scale q_t S_t,  a state S of Dk by Dv for every head;
             l_t is decay (H), constants of the heads ("head"), or g (B, L, H), one for each token and head ("token"), or
             their sum ("both").  Where "resets" is true some g are -inf: a document ends within its row.
  gated      x (M, D), w_gate, w_up (F, D): y = act(x w_gate^T) * (x w_up^T), on tokens one by one.

Sequences of one call have lengths of their own where "lengths" is true, zero and one among them: tokens behind a
length are padding, whose inputs hold anything and whose outputs and gradients are 0.
"""
import math
import random

import torch

own = False


def _attention(name, form, dtype, b, l, h, hk, dk, dv, decay="token", lengths=False, resets=False):
    return {"name": name, "op": "attention", "form": form, "dtype": dtype, "B": b, "L": l, "H": h, "Hk": hk, "Dk": dk, "Dv": dv,
            "decay": decay, "lengths": lengths, "resets": resets}


def _gated(name, form, dtype, m, d, f, act="silu"):
    return {"name": name, "op": "gated", "form": form, "dtype": dtype, "M": m, "D": d, "F": f, "act": act}


def listed():
    return [
        # one token of one sequence: the latency of a decoding step
        _attention("attention one token", "step", "bf16", 1, 1, 16, 16, 128, 128),
        # one token of each of 128 sequences: the states are what is read and written
        _attention("attention step", "step", "bf16", 128, 1, 16, 4, 128, 128),
        # a training batch of a layer of 2048 channels
        _attention("attention train", "train", "bf16", 8, 2048, 16, 16, 128, 128),
        # small heads with constant decays, rows that are no whole chunks
        _attention("attention small heads train", "train", "bf16", 3, 1537, 12, 12, 64, 64, decay="head"),
        # one long prompt, four heads of v to each head of q and k
        _attention("attention prompt", "fwd", "bf16", 1, 16384, 16, 4, 128, 128),
        # odd heads, sequences of all lengths, documents that end within a row, 32-bit tensors
        _attention("attention ragged train", "train", "f32", 5, 677, 6, 3, 72, 41, decay="both", lengths=True, resets=True),
        # one token: latency, the weights are what is read
        _gated("gated one token", "fwd", "bf16", 1, 2048, 8192),
        # one token of each of 64 sequences
        _gated("gated step", "fwd", "bf16", 64, 2048, 8192),
        # a training batch
        _gated("gated train", "train", "bf16", 8192, 2048, 8192),
        # a prompt of a narrower layer
        _gated("gated prompt", "fwd", "bf16", 4096, 1024, 2816, act="gelu"),
        # rows of odd lengths
        _gated("gated odd train", "train", "bf16", 1021, 1030, 2731),
        # 32-bit tensors
        _gated("gated f32 train", "train", "f32", 2048, 768, 2048, act="gelu"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


# tokens times heads times the state's elements, and tokens times both sides of the weights: those of the largest listed cases
_MOST_STATES, _MOST_PRODUCTS = 8 * 2048 * 16 * 128 * 128, 8192 * 2048 * 8192


def draw(rng):
    """Either operator in any form: single tokens to 16384 of them, 1 to 256 sequences, heads of 16 to 128 channels, rows of
    32 to 8192; bf16 twice as often as 32-bit tensors."""
    while True:
        dtype = rng.choice(["bf16", "bf16", "f32"])
        if rng.random() < 0.5:
            form = rng.choice(["train", "train", "fwd", "step"])
            hk, shared = _log(rng, 1, 24), rng.choice([1, 1, 2, 4, _log(rng, 1, 8)])
            dk, dv = (rng.choice([64, 128, 128, 32, _log(rng, 16, 128)]) for _ in range(2))
            b, l = _log(rng, 1, 256), 1 if form == "step" else _log(rng, 1, 16384)
            decay = rng.choice(["token", "token", "head", "both"])
            case = _attention("", form, dtype, b, l, hk * shared, hk, dk, dv, decay, form != "step" and rng.random() < 0.4,
                              decay != "head" and rng.random() < 0.3)
            if b * l * hk * shared * dk * dv > _MOST_STATES // (4 if dtype == "f32" else 1):
                continue
            if b * l * l * hk * shared > 8 * 16 * 4096 * 4096:      # what it takes in 64 bits
                continue
        else:
            form = rng.choice(["train", "train", "fwd"])
            m = rng.choice([_log(rng, 1, 16384), _log(rng, 1, 128)])
            d, f = _log(rng, 32, 4096), _log(rng, 32, 8192)
            if rng.random() < 0.6:
                d, f = -(-d // 32) * 32, -(-f // 32) * 32
            case = _gated("", form, dtype, m, d, f, rng.choice(["silu", "silu", "gelu", "none"]))
            if m * d * f > _MOST_PRODUCTS // (8 if dtype == "f32" else 1):
                continue
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
    if case["op"] == "gated":
        m, d, f = (case[k] for k in ("M", "D", "F"))
        state["x"] = r.tokens(m, d)                       # behind a norm
        state["w_gate"], state["w_up"] = (r.tokens(f, d, std=1.0 / math.sqrt(d)) for _ in range(2))
        if case["form"] == "train":
            state["dy"] = r.tokens(m, f, std=0.1)
        return state
    b, l, h, hk, dk, dv = (case[k] for k in ("B", "L", "H", "Hk", "Dk", "Dv"))
    state["scale"] = 1.0 / math.sqrt(dk)
    state["q"], state["k"], state["v"] = r.tokens(b, l, hk, dk), r.tokens(b, l, hk, dk, std=dk ** -0.25), r.tokens(b, l, h, dv)
    state["g"] = state["decay"] = state["lengths"] = None
    if case["decay"] != "head":
        # decays from 0.999 to 0.4 of a token, as a projection of the token gives them
        state["g"] = (-torch.exp(r.uniform(b, l, h, lo=math.log(1e-3), hi=0.0))).to(r.dtype)
        if case["resets"]:
            state["g"][r.uniform(b, l, h) < 0.005] = -math.inf
    if case["decay"] != "token":
        # memories of 2 to 500 tokens, spread over the heads
        state["decay"] = -torch.exp(r.uniform(h, lo=math.log(2e-3), hi=math.log(0.5)))
    if case["form"] == "step":
        state["slots"], state["state"] = _slots(case, seed), r.normal(b + 3, h, dk, dv)
        return state
    state["lengths"] = _lengths(case, seed)
    if case["form"] == "train":
        state["dy"] = r.tokens(b, l, h, dv, std=0.1)
    if state["lengths"] is not None:  # what stands behind a sequence's end is anything
        behind = torch.arange(l, device="cuda")[None, :] >= state["lengths"][:, None]
        for name in ("q", "k", "v", "g", "dy"):
            if state.get(name) is not None:
                state[name][behind] = float("nan")
    return state


def run(state):
    form = globals()["_%s_%s" % ("own" if own else "plain", state["case"]["op"])]
    return form(state)


# ---- plain forms ---------------------------------------------------------------------------------------------------


_GELU, _CUBE = 2 * math.sqrt(2 / math.pi), 0.044715


def _activation(kind, v, slope=False):
    """act(v), and its derivative where it is asked for; GELU by its tanh form, v sigmoid(2 sqrt(2/pi) (v + 0.044715 v^3))."""
    if kind == "none":
        return v, torch.ones_like(v) if slope else None
    sig = 1 / (1 + torch.exp(-(v if kind == "silu" else _GELU * (v + _CUBE * v * v * v))))
    if not slope:
        return v * sig, None
    inner = 1 if kind == "silu" else _GELU * (1 + 3 * _CUBE * v * v)
    return v * sig, sig * (1 + v * (1 - sig) * inner)


def _plain_gated(state):
    case, kind = state["case"], state["x"].dtype
    train = case["form"] == "train"
    x, wg, wu = (state[k].float() for k in ("x", "w_gate", "w_up"))
    gate, up = x @ wg.T, x @ wu.T
    act, slope = _activation(case["act"], gate, train)
    out = {"y": (act * up).to(kind)}
    if train:
        dy = state["dy"].float()
        dgate, dup = dy * up * slope, dy * act
        out["dx"] = (dgate @ wg + dup @ wu).to(kind)
        out["dw_gate"], out["dw_up"] = (dgate.T @ x).to(kind), (dup.T @ x).to(kind)
    return out


_CHUNK = 64


def _chunks(state, name, padded):
    """A (B, L, heads, D) input in 32 bits, padding as 0, as (B, heads, chunks, tokens, D)."""
    v = state[name].float()
    if state["lengths"] is not None:
        keep = torch.arange(v.shape[1], device="cuda")[None, :] < state["lengths"][:, None]
        v = torch.where(keep[:, :, None, None], v, torch.zeros((), device="cuda"))
    b, l, heads, d = v.shape
    v = torch.cat([v, v.new_zeros(b, padded - l, heads, d)], 1)
    return v.view(b, padded // _CHUNK, _CHUNK, heads, d).permute(0, 3, 1, 2, 4).contiguous()


def _log_decays(state, b, l, h):
    """l_t in 64 bits, 0 behind a sequence's end; exp(-100) is as good as 0."""
    ld = torch.zeros(b, l, h, dtype=torch.float64, device="cuda")
    if state["g"] is not None:
        ld = ld + state["g"].double()
    if state["decay"] is not None:
        ld = ld + state["decay"].double()
    ld = torch.clamp(ld, min=-100.0)
    if state["lengths"] is not None:
        keep = torch.arange(l, device="cuda")[None, :] < state["lengths"][:, None]
        ld = torch.where(keep[:, :, None], ld, torch.zeros((), dtype=torch.float64, device="cuda"))
    return ld


def _states(a, b):
    """s_i = a_i s_{i-1} + b_i along dim 2, s_{-1} = 0: pairs of chunks are joined, then pairs of pairs."""
    step = 1
    while step < a.shape[2]:
        b = torch.cat([b[:, :, :step], b[:, :, step:] + a[:, :, step:] * b[:, :, :-step]], 2)
        if 2 * step < a.shape[2]:
            a = torch.cat([a[:, :, :step], a[:, :, step:] * a[:, :, :-step]], 2)
        step *= 2
    return b


def _shift(s, back):
    """The neighbour's along dim 2: the chunk's before (back) or after it, 0 at the end."""
    zero = torch.zeros_like(s[:, :, :1])
    return torch.cat([zero, s[:, :, :-1]], 2) if back else torch.cat([s[:, :, 1:], zero], 2)


def _tokens(v, l):
    """(B, heads, chunks, tokens, D) as (B, L, heads, D)."""
    b, heads, n, c, d = v.shape
    return v.permute(0, 2, 3, 1, 4).reshape(b, n * c, heads, d)[:, :l]


def _plain_step(state):
    case, kind = state["case"], state["q"].dtype
    shared = case["H"] // case["Hk"]
    q, k = (state[n][:, 0].float().repeat_interleave(shared, 1) for n in ("q", "k"))
    v, slots = state["v"][:, 0].float(), state["slots"].long()
    a = torch.exp(_log_decays(state, case["B"], 1, case["H"])[:, 0]).float()
    s = a[:, :, None, None] * state["state"][slots] + k[:, :, :, None] * v[:, :, None, :]
    y = state["scale"] * (q[:, :, :, None] * s).sum(2)
    state["state"][slots] = s
    return {"y": y[:, None].to(kind), "state": state["state"]}


def _plain_attention(state):
    case, kind = state["case"], state["q"].dtype
    state.setdefault("lengths", None)
    if case["form"] == "step":
        return _plain_step(state)
    b, l, h, hk = (case[n] for n in ("B", "L", "H", "Hk"))
    scale, padded = state["scale"], -(-l // _CHUNK) * _CHUNK
    q, k = (_chunks(state, n, padded).repeat_interleave(h // hk, 1) for n in ("q", "k"))
    v = _chunks(state, "v", padded)
    ld = _log_decays(state, b, l, h)
    ld = torch.cat([ld, ld.new_zeros(b, padded - l, h)], 1).view(b, -1, _CHUNK, h).permute(0, 3, 1, 2)
    total = ld.cumsum(3)                                                        # (B, H, chunks, tokens)
    before = torch.arange(_CHUNK, device="cuda")
    seen = before[:, None] >= before[None, :]
    pair = torch.where(seen, total[..., :, None] - total[..., None, :], torch.full((), -math.inf, device="cuda"))
    pair = torch.exp(pair).float()                                              # from token s to token t
    first, last = torch.exp(total).float()[..., None], torch.exp(total[..., -1:] - total).float()[..., None]
    whole = first[..., -1:, :]                                                  # a chunk's decay
    weights = q @ k.transpose(-1, -2) * (scale * pair)
    states = _states(whole, (last * k).transpose(-1, -2) @ v)
    entry = _shift(states, True)
    y = weights @ v + scale * first * (q @ entry)
    out = {"y": _tokens(y, l).to(kind), "state": states[:, :, -1]}
    if case["form"] == "train":
        dy = _chunks(state, "dy", padded)
        # gradients of the states behind each chunk, from the last to the first
        grown = (scale * first * q).transpose(-1, -2) @ dy
        leaving = _shift(_states(whole.flip(2), grown.flip(2)).flip(2), False)
        moved = dy @ v.transpose(-1, -2) * (scale * pair)
        dq_before, dk_after = scale * first * (dy @ entry.transpose(-1, -2)), last * (v @ leaving.transpose(-1, -2))
        dq, dk = moved @ k + dq_before, moved.transpose(-1, -2) @ q + dk_after
        out["dv"] = _tokens(weights.transpose(-1, -2) @ dy + last * (k @ leaving), l).to(kind)
        for name, grad in (("dq", dq), ("dk", dk)):
            out[name] = _tokens(grad.view(b, hk, h // hk, *grad.shape[2:]).sum(2), l).to(kind)
        if state["g"] is not None:
            # pairs that a token's decay lies between, tokens from it on with the state before the chunk, tokens before it
            # with what is behind the chunk, and the state that passes through all of it
            crossed = (moved * (q @ k.transpose(-1, -2)) * ~torch.eye(_CHUNK, dtype=torch.bool, device="cuda")).double()
            ahead = crossed.sum(-1) - crossed.sum(-2) + (q * dq_before).sum(-1).double()
            behind = (k * dk_after).sum(-1).double()
            dl = ahead.flip(3).cumsum(3).flip(3) + behind.cumsum(3) - behind
            dl = dl + (whole * entry * leaving).sum((-1, -2))[..., None]
            out["dg"] = dl.permute(0, 2, 3, 1).reshape(b, padded, h)[:, :l]
            if state["lengths"] is not None:
                keep = torch.arange(l, device="cuda")[None, :, None] < state["lengths"][:, None, None]
                out["dg"] = torch.where(keep, out["dg"], torch.zeros((), dtype=torch.float64, device="cuda"))
            out["dg"] = out["dg"].to(kind)
    return out


# ---- the framework's operators -------------------------------------------------------------------------------------


def _workspace(nbytes):
    return torch.empty(nbytes, dtype=torch.uint8, device="cuda") if nbytes else None


def _dtype(state):
    return 1 if state["case"]["dtype"] == "bf16" else 0


def _own_gated(state):
    from paper_1804_04806_amd import seq
    case, x, wg, wu = state["case"], state["x"], state["w_gate"], state["w_up"]
    train = case["form"] == "train"
    if "desc" not in state:
        act = {"none": seq.ACT_NONE, "silu": seq.ACT_SILU, "gelu": seq.ACT_GELU}[case["act"]]
        desc = seq.gated_projection(M=case["M"], D=case["D"], F=case["F"], act=act, dtype=_dtype(state))
        state["ws"] = _workspace(max(seq.ucd_gated_projection_workspace_size(desc, op)
                                     for op in ((seq.FWD, seq.BWD) if train else (seq.FWD,))))
        state["y"] = torch.empty(case["M"], case["F"], dtype=x.dtype, device="cuda")
        if train:
            state["saved"] = _workspace(seq.ucd_gated_projection_saved_size(desc))
            state["dx"], state["dw_gate"], state["dw_up"] = torch.empty_like(x), torch.empty_like(wg), torch.empty_like(wu)
        state["desc"] = desc
    desc = state["desc"]
    seq.ucd_gated_projection_fwd(desc, x, wg, wu, state["y"], saved=state.get("saved"), ws=state["ws"])
    out = {"y": state["y"]}
    if train:
        seq.ucd_gated_projection_bwd(desc, x, wg, wu, state["dy"], state["saved"], state["dx"], state["dw_gate"], state["dw_up"],
                                     ws=state["ws"])
        out.update({k: state[k] for k in ("dx", "dw_gate", "dw_up")})
    return out


def _own_attention(state):
    from paper_1804_04806_amd import seq
    case = state["case"]
    step, train = case["form"] == "step", case["form"] == "train"
    if "desc" not in state:
        desc = seq.linear_attention(B=case["B"], L=case["L"], H=case["H"], Hk=case["Hk"], Dk=case["Dk"], Dv=case["Dv"],
                                    scale=state["scale"], dtype=_dtype(state), n_slots=case["B"] + 3 if step else 0)
        state["y"] = torch.empty_like(state["v"])
        if not step:
            state["last"] = torch.empty(case["B"], case["H"], case["Dk"], case["Dv"], device="cuda")
            state["ws"] = _workspace(max(seq.ucd_linear_attention_workspace_size(desc, op)
                                         for op in ((seq.FWD, seq.BWD) if train else (seq.FWD,))))
        if train:
            state["saved"] = _workspace(seq.ucd_linear_attention_saved_size(desc))
            for name in ("q", "k", "v", "g"):
                state["d" + name] = None if state[name] is None else torch.empty_like(state[name])
        state["desc"] = desc
    desc = state["desc"]
    inputs, more = [state[k] for k in ("q", "k", "v")], {k: state[k] for k in ("g", "decay")}
    if step:
        seq.ucd_linear_attention_step(desc, *inputs, state["state"], state["y"], slots=state["slots"], **more)
        return {"y": state["y"], "state": state["state"]}
    more["lengths"] = state["lengths"]
    seq.ucd_linear_attention_fwd(desc, *inputs, state["y"], state_out=state["last"], saved=state.get("saved"), ws=state["ws"],
                                 **more)
    out = {"y": state["y"], "state": state["last"]}
    if train:
        seq.ucd_linear_attention_bwd(desc, *inputs, state["dy"], state["saved"], state["dq"], state["dk"], state["dv"],
                                     dg=state["dg"], ws=state["ws"], **more)
        out.update({"d" + k: state["d" + k] for k in ("q", "k", "v", "g") if state["d" + k] is not None})
    return out


# ---- what a pass cannot do without ---------------------------------------------------------------------------------


def work(case):
    """Bytes: each input once, each output once.  Flops: those of the products; of the attention the recurrence's, two
    products of a token with a state forward and four backward.  Lengths are not counted: a case with them has at most
    this work."""
    e = 2 if case["dtype"] == "bf16" else 4
    train = case["form"] == "train"
    if case["op"] == "gated":
        m, d, f = (case[k] for k in ("M", "D", "F"))
        return {"bytes": e * ((m * d + m * f) * (2 if train else 1) + 2 * f * d * (2 if train else 1)),
                "flops": m * d * f * (12 if train else 4)}
    b, l, h, hk, dk, dv = (case[k] for k in ("B", "L", "H", "Hk", "Dk", "Dv"))
    per_token = 2 * hk * dk + 2 * h * dv + (h if case["decay"] != "head" else 0)
    if train:   # dy, and the gradients of q, k, v and g
        per_token += 2 * hk * dk + 2 * h * dv + (h if case["decay"] != "head" else 0)
    state = 4 * b * h * dk * dv * (2 if case["form"] == "step" else 1)
    return {"bytes": e * b * l * per_token + state + (4 * h if case["decay"] != "token" else 0),
            "flops": b * l * h * dk * dv * (12 if train else 4)}


# ---- in 64 bits ----------------------------------------------------------------------------------------------------


def exact(case, seed):
    """The definitions in 64 bits, gradients by automatic differentiation; the attention as sums over all pairs of tokens."""
    state = prepare(case, seed)
    return (_exact_gated if case["op"] == "gated" else _exact_attention)(case, state)


def _exact_gated(case, state):
    train = case["form"] == "train"
    x, wg, wu = (state[k].double().requires_grad_(train) for k in ("x", "w_gate", "w_up"))
    gate = torch.nn.functional.linear(x, wg)
    if case["act"] == "silu":
        gate = torch.nn.functional.silu(gate)
    elif case["act"] == "gelu":
        gate = torch.nn.functional.gelu(gate, approximate="tanh")
    y = gate * torch.nn.functional.linear(x, wu)
    out = {"y": y.detach()}
    if train:
        grads = torch.autograd.grad(y, (x, wg, wu), state["dy"].double())
        out.update(zip(("dx", "dw_gate", "dw_up"), grads))
    return out


def _exact_attention(case, state):
    b, l, h, hk = (case[n] for n in ("B", "L", "H", "Hk"))
    train = case["form"] == "train"
    v = {n: state[n].double() for n in ("q", "k", "v", "g", "dy") if state.get(n) is not None}
    lengths = state["lengths"].tolist() if state.get("lengths") is not None else [l] * b
    for n in v.values():
        for row, length in zip(n, lengths):
            row[length:] = 0
    ld = torch.zeros(b, l, h, dtype=torch.float64, device="cuda")
    if "g" in v:
        ld = ld + v["g"]
    if state["decay"] is not None:
        ld = ld + state["decay"].double()
    ld = torch.where(ld == -math.inf, torch.full_like(ld, -1e4), ld)     # exp(-1e4) is 0, differences of sums of it are not NaN
    for row, length in zip(ld, lengths):
        row[length:] = 0
    if case["form"] == "step":
        slots = state["slots"].long()
        pool = state["state"].double()
        q, k = (v[n][:, 0].repeat_interleave(h // hk, 1) for n in ("q", "k"))
        s = torch.exp(ld[:, 0])[..., None, None] * pool[slots] + torch.einsum("bhi,bhj->bhij", k, v["v"][:, 0])
        pool[slots] = s
        return {"y": state["scale"] * torch.einsum("bhi,bhij->bhj", q, s)[:, None], "state": pool}
    names = ["q", "k", "v"] + (["g"] if "g" in v else [])
    out = {"y": torch.empty_like(v["v"]), "state": v["v"].new_empty(b, h, case["Dk"], case["Dv"])}
    if train:
        out.update({"d" + n: torch.zeros_like(v[n]) for n in names})
    at = torch.arange(l, device="cuda")
    unseen = at[:, None] < at[None, :]
    some = max(1, min(b, (1 << 27) // (l * l)))      # sequences at a time, head by head
    for i in range(0, b, some):
        for j in range(h):
            with torch.set_grad_enabled(train):
                q, k, vv, lj = (t[i:i + some, :, n].detach().requires_grad_(train) for t, n in
                                ((v["q"], j // (h // hk)), (v["k"], j // (h // hk)), (v["v"], j), (ld, j)))
                total = lj.cumsum(1)
                seen = (total[:, :, None] - total[:, None, :]).masked_fill(unseen, -math.inf).exp()
                y = state["scale"] * ((q @ k.transpose(1, 2)) * seen) @ vv
                out["y"][i:i + some, :, j] = y.detach()
                out["state"][i:i + some, j] = ((torch.exp(total[:, -1:] - total)[..., None] * k).transpose(1, 2) @ vv).detach()
                if train:
                    grads = torch.autograd.grad(y, (q, k, vv, lj), v["dy"][i:i + some, :, j])
                    for n, grad in zip(("q", "k", "v", "g"), grads):
                        if n in names:
                            out["d" + n][i:i + some, :, j // (h // hk) if n in "qk" else j] += grad
            del seen, y
    if train and "g" in names:
        for row, length in zip(out["dg"], lengths):
            row[length:] = 0
    return out
