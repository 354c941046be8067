"""Linear attention's gradient of the decays where it is far smaller than the tokens' own products: a token that forgets nearly everything, between others
whose pairs do not cross it and have to cancel."""
import numpy as np
import pytest

from oracle import seq as os_
from paper_1804_04806_amd import seq
from seq_helpers import device, kind_of, values, workspace

pytestmark = pytest.mark.gpu

FIRST, LAST = 24, 40      # tokens of a chunk between resets; the first one of them is the strong one


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("B, L, H, Hk, Dk, Dv", [(4, 64, 16, 16, 16, 16), (2, 128, 16, 8, 64, 32), (3, 128, 8, 8, 40, 72), (1, 64, 16, 16, 128, 128)])
def test_what_does_not_cross_cancels(B, L, H, Hk, Dk, Dv, dtype):
    """Chunks of resets, a token of e^-30, weak decays, resets.  What crosses the strong token is e^-30 of the rest, so that its gradient is what is left of
    pairs of tokens behind it, each of which is in a row's sum A_t and in a column's B_s:  with the same products in both nothing is left but
    rounding of 32 bits.  A row's sum takes its up to 64 tokens and Dk channels and then some 16 joins, one rounding each: (64 + Dk + 16) 2^-24 of
    the sum of its terms' absolute values at most, a column's as well.  Rows' and columns' are independent, so that their squares add up; over all
    strong tokens the 2-norms are compared.  Products that are rounded to 8 bits on one side as they are not on the other would leave 2^-8 of them."""
    rng = np.random.default_rng(B + L + Dk)
    q, k = values(rng, B, L, Hk, Dk, dtype=dtype), values(rng, B, L, Hk, Dk, std=Dk ** -0.25, dtype=dtype)
    v, dy = values(rng, B, L, H, Dv, dtype=dtype), values(rng, B, L, H, Dv, dtype=dtype)
    scale = Dk ** -0.5
    g = np.full((B, L, H), -np.inf, np.float32)
    at = np.arange(L) % 64
    weak = (at > FIRST) & (at < LAST)
    g[:, weak] = -np.exp(rng.uniform(np.log(1e-3), np.log(0.5), (B, int(weak.sum()), H)))
    g[:, at == FIRST] = -30
    t = {n: device(a).to(kind_of(dtype)) for n, a in (("q", q), ("k", k), ("v", v), ("dy", dy), ("g", g))}
    g = t["g"].float().cpu().numpy()
    import torch
    desc = seq.linear_attention(B, L, H, Dk, Dv, Hk, scale, dtype)
    ws, ws_bytes, ws_check = workspace(max(seq.ucd_linear_attention_workspace_size(desc, d) for d in (seq.FWD, seq.BWD)))
    saved, saved_bytes, saved_check = workspace(seq.ucd_linear_attention_saved_size(desc))
    y, dq, dk, dv, dg = (torch.empty_like(t[n]) for n in ("v", "q", "k", "v", "g"))
    seq.ucd_linear_attention_fwd(desc, t["q"], t["k"], t["v"], y, g=t["g"], saved=saved, saved_bytes=saved_bytes, ws=ws, ws_bytes=ws_bytes)
    seq.ucd_linear_attention_bwd(desc, t["q"], t["k"], t["v"], t["dy"], saved, dq, dk, dv, g=t["g"], dg=dg, saved_bytes=saved_bytes, ws=ws,
                                 ws_bytes=ws_bytes)
    ws_check(), saved_check()
    got = dg.float().cpu().numpy().astype(np.float64)
    want = os_.attention_bwd(q, k, v, scale, dy, g, None)["g"]
    got, want = got[:, at == FIRST], want[:, at == FIRST]      # (B, chunks, H)
    room = np.zeros(want.shape)
    share = H // Hk
    for c in range(L // 64):
        part = slice(64 * c + FIRST, 64 * c + LAST)
        qc, kc = (np.abs(np.repeat(m[:, part].astype(np.float64), share, 2)) for m in (q, k))
        total = np.cumsum(np.where(np.arange(LAST - FIRST)[None, :, None] > 0, g[:, part], 0).astype(np.float64), 1)
        decay = np.exp(total[:, :, None] - total[:, None, :])      # (B, t, s, H)
        seen = np.arange(LAST - FIRST)[:, None] > np.arange(LAST - FIRST)[None, :]
        weights = np.abs(np.einsum("bthd,bshd->btsh", dy[:, part].astype(np.float64), v[:, part].astype(np.float64))) * scale
        terms = np.where(seen[None, :, :, None], weights * np.minimum(decay, 1) * np.einsum("bthd,bshd->btsh", qc, kc), 0)
        each = (64 + Dk + 16) * 2.0 ** -24
        room[:, c] = each * np.sqrt((terms.sum(2) ** 2).sum(1) + (terms.sum(1) ** 2).sum(1))
    off, allowed = np.linalg.norm(got - want), np.linalg.norm(room)
    assert off <= allowed, (off, allowed, np.linalg.norm(want))
