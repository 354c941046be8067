"""What linear attention's elements are sums of: chunk by chunk in 64 bits on the device, the values and the sums of the squares of the terms that a 16-bit
call rounds an operand of.  The values have to be the oracle's (which goes token by token), so that the terms are those of what is compared."""
import numpy as np

CHUNK = 64


def _crossing(m):
    """sum of m[t, s] over s < u <= t, for every u."""
    both = m.flip(-2).cumsum(-2).flip(-2).cumsum(-1)      # [u, s]: rows from u on, columns up to s
    import torch
    return torch.cat([both.new_zeros(both.shape[:-2] + (1,)), torch.diagonal(both, offset=-1, dim1=-2, dim2=-1)], -1)


def forms(v, scale, lengths=None):
    """({name: values}, {name: sums of squares}) of y and of the gradients of q, k, v and g as numpy arrays; v: arrays by name, as the oracle takes
    them.

    y and the gradients of q, k and v mix rows (x, z, w) by pairs' weights P = scale (x z^T) D within the chunk and by the state before or behind it:
    the operands that are rounded are P and the state, so that the terms are P w and x S.  The decays' gradient has the pairs that cross it, the
    state before the chunk (in the tokens from it on, and in what passes through) and the state's gradient behind it (in the tokens before it)."""
    import torch
    B, L, H, Dv = v["v"].shape
    Hk, Dk = v["q"].shape[2:]
    padded = -(-max(L, 1) // CHUNK) * CHUNK
    here = torch.arange(padded, device="cuda:0")[None, :] < torch.as_tensor(np.full(B, L) if lengths is None else lengths, device="cuda:0")[:, None]

    def rows(a):
        """(B, H, padded, ...), 0 behind a sequence's end"""
        t = torch.zeros((B, padded) + a.shape[2:], dtype=torch.float64, device="cuda:0")
        t[:, :L] = torch.as_tensor(np.asarray(a, np.float64), device="cuda:0")
        t = torch.where(here.view(B, padded, *[1] * (t.dim() - 2)), t, torch.zeros((), dtype=torch.float64, device="cuda:0"))
        return (t.repeat_interleave(H // t.shape[2], 2)).transpose(1, 2)
    q, k, val, dy = (rows(v[n]) for n in ("q", "k", "v", "dy"))
    ld = torch.zeros(B, padded, H, dtype=torch.float64, device="cuda:0")
    if v["g"] is not None:
        ld[:, :L] += torch.as_tensor(v["g"].astype(np.float64), device="cuda:0")
    if v["decay"] is not None:
        ld += torch.as_tensor(v["decay"].astype(np.float64), device="cuda:0")
    ld = torch.where(here[:, :, None], ld.clamp(min=-1e4), torch.zeros((), dtype=torch.float64, device="cuda:0")).transpose(1, 2)
    none = torch.zeros(B, H, Dk, Dv, dtype=torch.float64, device="cuda:0")
    first, last = (none if v[n] is None else torch.as_tensor(v[n].astype(np.float64), device="cuda:0") for n in ("state", "dstate"))
    seen = torch.ones(CHUNK, CHUNK, dtype=torch.bool, device="cuda:0").tril()
    parts, squares, begin = {n: [] for n in "yqkvg"}, {n: [] for n in "yqkvg"}, []

    def of(c):
        part = slice(c, c + CHUNK)
        total = ld[:, :, part].cumsum(-1)
        pair = torch.where(seen, total[..., :, None] - total[..., None, :], torch.full((), -1e300, dtype=torch.float64, device="cuda:0")).exp()
        return q[:, :, part], k[:, :, part], val[:, :, part], dy[:, :, part], pair, scale * total.exp()[..., None], \
            (total[..., -1:] - total).exp()[..., None], total[..., -1].exp()[..., None, None]

    def put(name, weights, w, x, factor, state):
        parts[name].append(weights @ w + factor * (x @ state))
        squares[name].append(weights ** 2 @ w ** 2 + factor ** 2 * (x ** 2 @ state ** 2))
    state = first
    for c in range(0, padded, CHUNK):
        qc, kc, vc, _, pair, before, behind, whole = of(c)
        begin.append(state)
        put("y", scale * (qc @ kc.transpose(-1, -2)) * pair, vc, qc, before, state)
        state = whole * state + (behind * kc).transpose(-1, -2) @ vc
    grad = last
    for c in reversed(range(0, padded, CHUNK)):
        qc, kc, vc, dyc, pair, before, behind, whole = of(c)
        state, dots, keys = begin[c // CHUNK], scale * (dyc @ vc.transpose(-1, -2)) * pair, qc @ kc.transpose(-1, -2)
        put("q", dots, kc, dyc, before, state.transpose(-1, -2))
        put("k", dots.transpose(-1, -2), qc, vc, behind, grad.transpose(-1, -2))
        put("v", (scale * keys * pair).transpose(-1, -2), dyc, kc, behind, grad)
        w = dots * keys
        a = (qc * before * (dyc @ state.transpose(-1, -2))).sum(-1)
        b = (kc * behind * (vc @ grad.transpose(-1, -2))).sum(-1)
        parts["g"].append(_crossing(w) + a.flip(-1).cumsum(-1).flip(-1) + b.cumsum(-1) - b + (whole * state * grad).sum((-1, -2))[..., None])
        of_state = ((before * qc)[..., :, None] * dyc[..., None, :]).flip(2).cumsum(2).flip(2) + (whole * grad)[:, :, None]
        share = _crossing(w ** 2) + (of_state ** 2 * state[:, :, None] ** 2).sum((-1, -2))
        of_state = (behind * kc)[..., :, None] * vc[..., None, :]
        of_state = of_state.cumsum(2) - of_state
        squares["g"].append(share + (of_state ** 2 * grad[:, :, None] ** 2).sum((-1, -2)))
        grad = whole * grad + (before * qc).transpose(-1, -2) @ dyc

    def whole_tensor(name, chunks):
        t = torch.cat(chunks if name == "y" else chunks[::-1], 2)[:, :, :L].transpose(1, 2)
        if name in "qk":
            t = t.reshape(B, L, Hk, H // Hk, Dk).sum(3)
        if name == "g":      # a decay behind a sequence's end is none of it
            t = t * here[:, :L, None]
        return t.cpu().numpy()
    return tuple({n: whole_tensor(n, c) for n, c in d.items()} for d in (parts, squares))
