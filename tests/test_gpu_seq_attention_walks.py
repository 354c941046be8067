"""Linear attention whose workgroups walk over several chunks each, against the 64-bit oracle: whole sequences, and segments of several chunks, the last of
them shorter.  What passes from chunk to chunk is the state, the decays of the chunk that comes, and what is read ahead."""
import numpy as np
import pytest

from oracle import seq as os_
from paper_1804_04806_amd import seq
from seq_attention_terms import forms
from seq_helpers import BF16, F32_ELEMENT, F32_L2, Placed, check, device, lengths_for, workspace
from test_gpu_seq_attention import L2, inputs

pytestmark = pytest.mark.gpu

# B, L, H, Hk, Dk, Dv; heads of either side of 64, rows of whole pieces and others, shared heads
SEQUENCES = [(6, 200, 44, 22, 24, 16), (5, 130, 53, 53, 41, 72), (4, 190, 66, 33, 72, 40), (1, 70, 260, 130, 128, 128), (3, 129, 88, 88, 128, 33)]
SEGMENTS = [(4, 700, 24, 12, 24, 16), (4, 650, 25, 25, 64, 64), (3, 700, 32, 32, 72, 41), (5, 450, 20, 4, 128, 72), (2, 577, 50, 50, 33, 128)]


def off(got, ref, squares, dtype, what, n):
    """bf16: as in the 2-norm in the tests of single chunks, but an element is held to its own terms instead of the tensor's rms, which says nothing of one
    whose row remembers four times as much.  The operands that are rounded are off by 2^-8 of themselves at most, each by itself: an element's
    variance is 2^-16 / 3 of its terms' squares at most, and among some ten million elements none is six standard deviations off (1 in 5 * 10^8 of
    a normal error; sums of fewer terms are bounded closer).  Beside them its own rounding, 2^-8 of it, and sums in fp32."""
    if n is not None:
        live = np.arange(ref.shape[1])[None, :] < n[:, None]
        assert (got[~live] == 0).all(), what
        got, ref, squares = got[live], ref[live], squares[live]
    if dtype == 0:
        return check(got, ref, 0, what)
    check(got, ref, 1, what, l2=(2 if what == "g" else 1) * L2[1], element=np.inf)
    floor = F32_ELEMENT * np.maximum(np.abs(ref), np.sqrt(np.mean(ref ** 2)))
    allowed = 6 * BF16 / np.sqrt(3) * np.sqrt(squares) + BF16 * np.abs(ref) + floor
    most = float((np.abs(got - ref) / allowed).max())
    assert most <= 1, (what, most)


def run(shape, dtype, seed=0, decays="both", resets=False, lengths=False, state=True, strides=False, shift=0, scale=0.3):
    import torch
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
    names = [k for k in ("q", "k", "v", "g") if v[k] is not None]
    p = {k: Placed(v[k].shape, dtype, st[k], v[k], shift) for k in names}
    grads = {k: Placed(v[k].shape, dtype, st[k], shift=shift) for k in names}
    py, pdy = Placed(v["v"].shape, dtype, st["y"], shift=shift), Placed(v["dy"].shape, dtype, st["y"], v["dy"], shift)
    d, dlen = {k: device(v[k]) for k in ("decay", "state", "dstate")}, device(n)
    last, dfirst = (torch.full((B, H, Dk, Dv), float("nan"), device="cuda:0") for _ in range(2))
    saved, saved_bytes, saved_check = workspace(seq.ucd_linear_attention_saved_size(desc))
    ws, ws_bytes, ws_check = workspace(seq.ucd_linear_attention_workspace_size(desc, seq.FWD))
    given, more = [p[k].ptr() for k in "qkv"], dict(g=p["g"].ptr() if "g" in p else None, decay=d["decay"], lengths=dlen, saved_bytes=saved_bytes)
    seq.ucd_linear_attention_fwd(desc, *given, py.ptr(), state_in=d["state"], state_out=last, saved=saved, ws=ws, ws_bytes=ws_bytes, **more)
    ws_check()
    back, back_bytes, back_check = workspace(seq.ucd_linear_attention_workspace_size(desc, seq.BWD))
    seq.ucd_linear_attention_bwd(desc, *given, pdy.ptr(), saved, *(grads[k].ptr() for k in "qkv"), dg=grads["g"].ptr() if "g" in grads else None,
                                 dstate_out=d["dstate"], dstate_in=dfirst, ws=back, ws_bytes=back_bytes, **more)
    saved_check(), back_check()
    with np.errstate(all="ignore"):
        ref, ref_state = os_.attention_fwd(v["q"], v["k"], v["v"], scale, v["g"], v["decay"], n, v["state"])
        want = os_.attention_bwd(v["q"], v["k"], v["v"], scale, v["dy"], v["g"], v["decay"], n, v["state"], v["dstate"])
    want["y"] = ref
    values, squares = forms(v, scale, n)
    for name in ["y"] + names:
        apart = float(np.linalg.norm(values[name] - want[name]) / np.linalg.norm(want[name]))
        assert apart <= 1e-9, (name, apart)      # the terms are those of the oracle's values
        off((py if name == "y" else grads[name]).get().astype(np.float64), want[name], squares[name], dtype, name, n)
    if resets:
        forgotten = np.isneginf(v["g"])
        assert forgotten.any() and not grads["g"].get()[forgotten].any()
    check(last.cpu().numpy(), ref_state, 0, "state", F32_L2)
    check(dfirst.cpu().numpy(), want["state"], 0, "dstate", F32_L2)


def plan(shape, dtype):
    """Segments and chunks of a call: Forward keeps a state for every segment."""
    B, L, H, Hk, Dk, Dv = shape
    desc = seq.linear_attention(B, L, H, Dk, Dv, Hk, dtype=dtype)
    segments = seq.ucd_linear_attention_saved_size(desc) // (B * H * Dk * Dv * 4)
    return segments, (L + 63) // 64


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("shape", SEQUENCES, ids=str)
def test_whole_sequences(shape, dtype):
    segments, chunks = plan(shape, dtype)
    assert segments == 1 and chunks > 1
    run(shape, dtype, sum(shape))


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("shape", SEGMENTS, ids=str)
def test_segments_of_chunks(shape, dtype):
    segments, chunks = plan(shape, dtype)
    assert 1 < segments <= chunks // 2
    run(shape, dtype, sum(shape))


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("shape", [SEQUENCES[0], SEQUENCES[2], SEGMENTS[0], SEGMENTS[3]], ids=str)
def test_resets_and_lengths(shape, dtype):
    """Sequences that end within a chunk, within a segment and before one, and documents that end within a row."""
    segments, chunks = plan(shape, dtype)
    assert segments < chunks
    run(shape, dtype, 1, "both", resets=True, lengths=True)
    run(shape, dtype, 2, "token", resets=True, lengths=True, state=False)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("decays", ["none", "head", "strong"])
@pytest.mark.parametrize("shape", [(5, 150, 53, 53, 40, 17), (4, 500, 25, 25, 17, 40)], ids=str)
def test_decays(shape, decays, dtype):
    segments, chunks = plan(shape, dtype)
    assert segments < chunks
    run(shape, dtype, 3, decays)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("strides, shift", [(True, 1), ("tokens first", 0), (None, 1)], ids=str)
def test_strides(strides, shift, dtype):
    for shape in ((5, 150, 53, 53, 24, 9), (4, 500, 25, 5, 9, 24)):
        segments, chunks = plan(shape, dtype)
        assert segments < chunks
        run(shape, dtype, 4, strides=strides, shift=shift)
