"""Linear attention against the 64-bit oracle: heads of 1 to 128 channels, shared heads, single tokens to many chunks, segments,
constant decays, decays of tokens and resets, lengths with empty sequences, strides, states in pools, gradients of everything, and
what single tokens make of a prompt's state."""
import numpy as np
import pytest

from oracle import seq as os_
from paper_1804_04806_amd import seq
from seq_helpers import BF16, F32_ELEMENT, F32_L2, Placed, check, device, lengths_for, values, workspace

pytestmark = pytest.mark.gpu

# B, L, H, Hk, Dk, Dv
SHAPES = [(1, 1, 1, 1, 1, 1), (2, 5, 2, 2, 64, 64), (1, 64, 2, 1, 128, 128), (2, 65, 4, 2, 32, 128), (1, 200, 3, 3, 128, 33), (3, 63, 2, 2, 17, 72),
          (1, 130, 6, 2, 65, 64), (2, 128, 1, 1, 128, 65), (1, 700, 1, 1, 48, 20), (1, 1100, 2, 1, 64, 128), (5, 9, 3, 1, 127, 3)]

# A bf16 output is rounded once (2^-8 of it at most).  Before it two operands of its products were: the weights of the chunk's tokens, and the
# state (for gradients the same of other rows); errors of their elements are independent, each 2^-8 of its term at most (half of that in the mean), so
# that in the 2-norm they add up to 2^-8 of the result for each.  A single element of the result may be six of
# its standard deviations off, 6 * 2^-8 / sqrt(3) * sqrt(2) < 5 * 2^-8 of the tensor's rms, beside its own rounding.  dg is the sum of four parts of which
# three have a rounded operand, and may be smaller than those: 6 * 2^-8 of the 2-norm, twice the elements' share.
L2, ELEMENT = {0: F32_L2, 1: 2 * BF16}, {0: F32_ELEMENT, 1: 5 * BF16}


def off(got, ref, dtype, what, n=None):
    if n is not None:      # the rms is that of tokens: padding is 0, exactly, and no part of it
        got, ref, live = np.asarray(got), np.asarray(ref), np.arange(ref.shape[1])[None, :] < n[:, None]
        assert (got[~live] == 0).all(), what
        got, ref = got[live], ref[live]
    wide = 2 if what == "g" and dtype == 1 else 1
    check(got, ref, dtype, what, l2=wide * L2[dtype], element=wide * ELEMENT[dtype])


def inputs(shape, dtype, seed, decays="both", resets=False):
    B, L, H, Hk, Dk, Dv = shape
    rng = np.random.default_rng(seed)
    v = {"q": values(rng, B, L, Hk, Dk, dtype=dtype), "k": values(rng, B, L, Hk, Dk, std=Dk ** -0.25, dtype=dtype),
         "v": values(rng, B, L, H, Dv, dtype=dtype), "dy": values(rng, B, L, H, Dv, std=0.3, dtype=dtype),
         "state": values(rng, B, H, Dk, Dv), "dstate": values(rng, B, H, Dk, Dv, std=0.3), "g": None, "decay": None}
    if decays in ("token", "both", "strong"):
        g = -np.exp(rng.uniform(np.log(1e-3), 0, (B, L, H))) if decays != "strong" else -rng.uniform(6, 9, (B, L, H))
        if resets:
            g[rng.uniform(size=g.shape) < 0.02] = -np.inf
        v["g"] = np.asarray(values(rng, 1), np.float32) * 0 + g.astype(np.float32)
        if dtype == 1:
            from paper_1804_04806_amd import synth
            v["g"] = synth.from_bf16_bits(synth.to_bf16_bits(v["g"]))
    if decays in ("head", "both"):
        v["decay"] = -np.exp(rng.uniform(np.log(2e-3), np.log(0.5), H)).astype(np.float32)
    return v, rng


def run(shape, dtype, seed=0, decays="both", resets=False, lengths=False, state=True, strides=False, shift=0, scale=0.3):
    B, L, H, Hk, Dk, Dv = shape
    v, rng = inputs(shape, dtype, seed, decays, resets)
    n = lengths_for(rng, B, L) if lengths else None
    if lengths:
        for b in range(B):
            for name in ("q", "k", "v", "g", "dy"):
                if v[name] is not None:
                    v[name][b, n[b]:] = np.nan
    if not state:
        v["state"] = v["dstate"] = None
    width = {"q": Hk * Dk, "k": Hk * Dk, "v": H * Dv, "g": H, "y": H * Dv}
    st = {k: None for k in width}
    if strides is True:
        st = {k: (L * (w + 4 * i + 4) + 8, w + 4 * i + 4) for i, (k, w) in enumerate(width.items())}
    elif strides == "tokens first":
        st = {k: (w, B * w) for k, w in width.items()}
    desc = seq.linear_attention(B, L, H, Dk, Dv, Hk, scale, dtype, **{k + "_stride": s or (0, 0) for k, s in st.items()})
    p, grads = {}, {}
    for name in ("q", "k", "v", "g"):
        if v[name] is not None:
            p[name] = Placed(v[name].shape, dtype, st[name], v[name], shift)
            grads[name] = Placed(v[name].shape, dtype, st[name], shift=shift)
    py, pdy = Placed(v["v"].shape, dtype, st["y"], shift=shift), Placed(v["dy"].shape, dtype, st["y"], v["dy"], shift)
    d = {k: device(v[k]) for k in ("decay", "state", "dstate")}
    dlen = device(n)
    import torch
    last = torch.full((B, H, Dk, Dv), float("nan"), device="cuda:0")
    dfirst = torch.full_like(last, float("nan"))
    ws, ws_bytes, ws_check = workspace(seq.ucd_linear_attention_workspace_size(desc, seq.FWD))
    saved, saved_bytes, saved_check = workspace(seq.ucd_linear_attention_saved_size(desc))
    g = p["g"].ptr() if "g" in p else None
    for with_saved in (False, True):
        py.t.fill_(Placed.POISON)
        seq.ucd_linear_attention_fwd(desc, p["q"].ptr(), p["k"].ptr(), p["v"].ptr(), py.ptr(), g=g, decay=d["decay"], lengths=dlen,
                                     state_in=d["state"], state_out=last, saved=saved if with_saved else None,
                                     saved_bytes=saved_bytes if with_saved else None, ws=ws, ws_bytes=ws_bytes)
    with np.errstate(all="ignore"):
        ref, ref_state = os_.attention_fwd(v["q"], v["k"], v["v"], scale, v["g"], v["decay"], n, v["state"])
        want = os_.attention_bwd(v["q"], v["k"], v["v"], scale, v["dy"], v["g"], v["decay"], n, v["state"], v["dstate"])
    off(py.get(), ref, dtype, "y", n)
    check(last.cpu().numpy(), ref_state, 0, "state")
    ws_check(), saved_check()
    ws, ws_bytes, ws_check = workspace(seq.ucd_linear_attention_workspace_size(desc, seq.BWD))
    seq.ucd_linear_attention_bwd(desc, p["q"].ptr(), p["k"].ptr(), p["v"].ptr(), pdy.ptr(), saved, grads["q"].ptr(), grads["k"].ptr(),
                                 grads["v"].ptr(), g=g, dg=grads["g"].ptr() if "g" in grads else None, decay=d["decay"], lengths=dlen,
                                 dstate_out=d["dstate"], dstate_in=dfirst, saved_bytes=saved_bytes, ws=ws, ws_bytes=ws_bytes)
    ws_check()
    for name in grads:
        off(grads[name].get(), want[name], dtype, name, n)
    if resets:      # what forgets everything has no gradient, exactly
        forgotten = np.isneginf(v["g"])
        assert forgotten.any() and not grads["g"].get()[forgotten].any()
    check(dfirst.cpu().numpy(), want["state"], 0, "dstate")


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_against_oracle(shape, dtype):
    run(shape, dtype, seed=sum(shape))


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("decays", ["none", "head", "token"])
def test_decays(decays, dtype):
    run((2, 140, 3, 3, 40, 64), dtype, 1, decays)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("shape", [(2, 140, 3, 3, 40, 64), (1, 70, 2, 1, 128, 128)], ids=str)
def test_strong_decays(shape, dtype):
    """Each token forgets all but a thousandth of those before it: what the decays' gradient is of is that much smaller than a token's own part."""
    run(shape, dtype, 5, "strong")


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("shape", [(4, 150, 4, 2, 64, 64), (3, 600, 1, 1, 72, 41)], ids=str)
def test_resets_and_lengths(shape, dtype):
    run(shape, dtype, 2, "both", resets=True, lengths=True)
    run(shape, dtype, 3, "token", resets=True, lengths=True, state=False)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("strides", [True, "tokens first"])
@pytest.mark.parametrize("shift", [0, 1])
def test_strides(strides, shift, dtype):
    run((2, 70, 4, 2, 24, 40), dtype, 4, strides=strides, shift=shift)


@pytest.mark.parametrize("dtype", [0, 1])
def test_pools(dtype):
    """A prompt into a pool, then single tokens: the same as the whole sequence; idle sequences and other places stay."""
    import torch
    B, L, H, Hk, Dk, Dv, more = 4, 77, 4, 2, 48, 72, 3
    v, rng = inputs((B, L + more, H, Hk, Dk, Dv), dtype, 5)
    n = np.array([77, 1, 0, 40], np.int32)
    pool = values(rng, 7, H, Dk, Dv)
    slots = np.array([5, 2, 6, -1], np.int32)
    kind = torch.bfloat16 if dtype == 1 else torch.float32
    t = {k: device(v[k]).to(kind) for k in ("q", "k", "v", "g")}
    state, decay = device(pool), device(v["decay"])
    head = {k: a[:, :L].contiguous() for k, a in t.items()}
    y = torch.full((B, L, H, Dv), float("nan"), dtype=kind, device="cuda:0")
    desc = seq.linear_attention(B, L, H, Dk, Dv, Hk, 0.5, dtype, n_slots=7)
    ws, ws_bytes, ws_check = workspace(seq.ucd_linear_attention_workspace_size(desc, seq.FWD))
    seq.ucd_linear_attention_fwd(desc, head["q"], head["k"], head["v"], y, g=head["g"], decay=decay, lengths=device(n), slots=device(slots),
                                 state_in=state, state_out=state, ws=ws, ws_bytes=ws_bytes)
    ws_check()
    real = slots.copy()
    real[3] = 0
    ref, ref_state = os_.attention_fwd(v["q"][:, :L], v["k"][:, :L], v["v"][:, :L], 0.5, v["g"][:, :L], v["decay"], n, pool[real])
    got = y.float().cpu().numpy()
    off(got[:3], ref[:3], dtype, "y", n[:3])
    assert (got[3] == 0).all()
    want = pool.copy()
    want[slots[:3]] = ref_state[:3]
    check(state.cpu().numpy(), want, 0, "pool")
    assert np.array_equal(state.cpu().numpy()[[0, 1, 3, 4]], pool[[0, 1, 3, 4]])
    step = seq.linear_attention(B, 1, H, Dk, Dv, Hk, 0.5, dtype, n_slots=7)
    for i in range(more):
        one = {k: a[:, L + i:L + i + 1].contiguous() for k, a in t.items()}
        out = torch.full((B, 1, H, Dv), float("nan"), dtype=kind, device="cuda:0")
        seq.ucd_linear_attention_step(step, one["q"], one["k"], one["v"], state, out, g=one["g"], decay=decay, slots=device(slots))
        before = want[real]
        ref, ref_state = os_.attention_fwd(*(v[k][:, L + i:L + i + 1] for k in ("q", "k", "v")), 0.5, v["g"][:, L + i:L + i + 1], v["decay"],
                                           None, before)
        check(out.float().cpu().numpy()[:3], ref[:3], dtype, "step")
        assert (out[3] == 0).all()
        want[slots[:3]] = ref_state[:3]
        check(state.cpu().numpy(), want, 0, "pool behind a step")


@pytest.mark.parametrize("dtype", [0, 1])
def test_no_tokens(dtype):
    """The state passes through a call without tokens, and its gradient."""
    import torch
    B, H, Dk, Dv = 2, 3, 16, 24
    rng = np.random.default_rng(6)
    desc = seq.linear_attention(B, 0, H, Dk, Dv, dtype=dtype)
    state, out = device(values(rng, B, H, Dk, Dv)), torch.zeros(B, H, Dk, Dv, device="cuda:0")
    saved, saved_bytes, saved_check = workspace(seq.ucd_linear_attention_saved_size(desc))
    seq.ucd_linear_attention_fwd(desc, None, None, None, None, state_in=state, state_out=out, saved=saved, saved_bytes=saved_bytes)
    assert torch.equal(state, out)
    back = torch.zeros_like(out)
    seq.ucd_linear_attention_bwd(desc, None, None, None, None, saved, None, None, None, dstate_out=state, dstate_in=back, saved_bytes=saved_bytes)
    assert torch.equal(state, back)
    saved_check()


def test_same_bits():
    """Two calls give the same bits, whatever the workspace held."""
    import torch
    B, L, H, Hk, Dk, Dv = 2, 1000, 4, 2, 64, 96
    v, _ = inputs((B, L, H, Hk, Dk, Dv), 1, 7)
    t = {k: device(v[k]).to(torch.bfloat16) for k in ("q", "k", "v", "g", "dy")}
    desc = seq.linear_attention(B, L, H, Dk, Dv, Hk, 0.1, 1)
    sizes = [seq.ucd_linear_attention_workspace_size(desc, d) for d in (seq.FWD, seq.BWD)]
    got = []
    for fill in (0, 255):
        ws = torch.full((max(sizes),), fill, dtype=torch.uint8, device="cuda:0")
        saved = torch.full((seq.ucd_linear_attention_saved_size(desc),), fill, dtype=torch.uint8, device="cuda:0")
        y, (dq, dk, dv, dg) = torch.empty_like(t["v"]), (torch.empty_like(t[k]) for k in ("q", "k", "v", "g"))
        seq.ucd_linear_attention_fwd(desc, t["q"], t["k"], t["v"], y, g=t["g"], saved=saved, ws=ws)
        seq.ucd_linear_attention_bwd(desc, t["q"], t["k"], t["v"], t["dy"], saved, dq, dk, dv, g=t["g"], dg=dg, ws=ws)
        got.append([a.clone() for a in (y, dq, dk, dv, dg)])
    assert all(torch.equal(a, b) for a, b in zip(*got))
