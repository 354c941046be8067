"""Short causal convolution against the 64-bit oracle: every filter length, single tokens to long sequences, odd channels,
strides, lengths with empty sequences, states in pools, idle sequences, gradients through the states."""
import numpy as np
import pytest

from oracle import seq as os_
from paper_1804_04806_amd import seq
from seq_helpers import Placed, check, device, kind_of, lengths_for, values, workspace

pytestmark = pytest.mark.gpu

# B, L, D, K
SHAPES = [(1, 1, 64, 4), (2, 3, 64, 4), (3, 64, 128, 4), (2, 257, 40, 3), (1, 1000, 33, 2), (5, 31, 509, 4), (2, 100, 24, 8), (3, 10, 16, 1),
          (2, 65, 8, 5), (4, 130, 1032, 6), (1, 4099, 8, 4), (2, 16, 7, 7), (1, 2, 72, 8), (300, 5, 16, 4)]


def inputs(shape, dtype, seed):
    B, L, D, K = shape
    rng = np.random.default_rng(seed)
    return {"x": values(rng, B, L, D, dtype=dtype), "w": values(rng, D, K, std=0.6, dtype=dtype), "bias": values(rng, D, std=0.3),
            "state": values(rng, B, K - 1, D, dtype=dtype), "dy": values(rng, B, L, D, std=0.3, dtype=dtype),
            "dstate": values(rng, B, K - 1, D, std=0.3, dtype=dtype)}, rng


def run(shape, dtype, silu=True, seed=0, lengths=False, state=True, bias=True, strides=False, beta=0.0, shift=0):
    B, L, D, K = shape
    v, rng = inputs(shape, dtype, seed)
    n = lengths_for(rng, B, L) if lengths else None
    if lengths:
        for b in range(B):
            v["x"][b, n[b]:] = v["dy"][b, n[b]:] = np.nan
    st = v["state"] if state else None
    bs = v["bias"] if bias else None
    xs = (L * (2 * D) + 6, 2 * D) if strides is True else (D, B * D) if strides == "tokens first" else None
    ys = (L * (D + 8), D + 8) if strides is True else None
    desc = seq.causal_conv(B, L, D, K, act=int(silu), dtype=dtype, x_stride=xs or (0, 0), y_stride=ys or (0, 0))
    px, py = Placed(v["x"].shape, dtype, xs, v["x"], shift), Placed(v["x"].shape, dtype, ys, shift=shift)
    pdy, pdx = Placed(v["x"].shape, dtype, ys, v["dy"], shift), Placed(v["x"].shape, dtype, xs, shift=shift)
    pst, pout = (Placed(v["state"].shape, dtype, data=v["state"]) if state else None), Placed(v["state"].shape, dtype)
    pds, pdin = Placed(v["state"].shape, dtype, data=v["dstate"]), Placed(v["state"].shape, dtype)
    w, dbs, ln = device(v["w"]).to(kind_of(dtype)), device(bs), device(n)
    old_w, old_b = rng.standard_normal((D, K)).astype(np.float32), rng.standard_normal(D).astype(np.float32)
    dw, dbias = device(old_w), device(old_b)
    st_ptr = pst.ptr() if state else None
    seq.ucd_causal_conv_fwd(desc, px.ptr(), w, dbs, py.ptr(), lengths=ln, state_in=st_ptr, state_out=pout.ptr())
    ws, nbytes, guard = workspace(seq.ucd_causal_conv_workspace_size(desc))
    seq.ucd_causal_conv_bwd(desc, px.ptr(), w, dbs, pdy.ptr(), pdx.ptr(), dw, dbias, lengths=ln, state_in=st_ptr, dstate_out=pds.ptr(),
                            dstate_in=pdin.ptr(), beta=beta, ws=ws, ws_bytes=nbytes)
    guard()
    y, out = os_.conv_fwd(v["x"], v["w"], bs, silu, n, st)
    dx, rw, rb, rs = os_.conv_bwd(v["x"], v["w"], bs, silu, v["dy"], n, st, v["dstate"])
    check(py.get(), y, dtype, "y")
    assert np.array_equal(pout.get(), out), "state"
    check(pdx.get(), dx, dtype, "dx")
    check(pdin.get(), rs, dtype, "dstate_in")
    check(dw.cpu().numpy(), rw + beta * old_w, 0, "dw")
    check(dbias.cpu().numpy(), rb + beta * old_b, 0, "dbias")
    if lengths:
        got_y, got_dx = py.get(), pdx.get()
        for b in range(B):
            assert not got_y[b, n[b]:].any() and not got_dx[b, n[b]:].any()


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_conv(shape, dtype):
    run(shape, dtype)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_conv_lengths(shape, dtype):
    run(shape, dtype, seed=1, lengths=True, state=shape[0] % 2 == 0)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("strides", [True, "tokens first"])
@pytest.mark.parametrize("shape", [SHAPES[2], SHAPES[3], SHAPES[5]], ids=str)
def test_conv_strides(shape, strides, dtype):
    run(shape, dtype, seed=2, strides=strides, lengths=True, shift=1 if strides is True else 0)


def test_conv_plain():
    run(SHAPES[3], 0, silu=False, state=False, bias=False)
    run(SHAPES[2], 0, beta=1.0)


@pytest.mark.parametrize("dtype", [0, 1])
def test_conv_wide_filters_values_stay_apart(dtype):
    """An infinite token reaches the K outputs that see it and no other; an infinite state the first K - 1."""
    import torch
    B, L, D, K = 1, 40, 16, 3
    desc = seq.causal_conv(B, L, D, K, dtype=dtype)
    x = torch.randn(B, L, D, device="cuda:0").to(kind_of(dtype))
    st = torch.zeros(B, K - 1, D, device="cuda:0").to(kind_of(dtype))
    x[0, 20, 5], st[0, 0, 6], st[0, 1, 7] = float("inf"), float("inf"), float("nan")
    w, y = torch.ones(D, K, device="cuda:0").to(kind_of(dtype)), torch.empty_like(x)
    seq.ucd_causal_conv_fwd(desc, x, w, None, y, state_in=st)
    bad = ~torch.isfinite(y[0].float()).cpu().numpy()
    want = np.zeros((L, D), bool)
    want[20:23, 5] = want[0, 6] = want[0:2, 7] = True
    assert np.array_equal(bad, want)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("shape", [(5, 1, 64, 4), (3, 1, 509, 3), (4, 1, 24, 1), (3, 1, 40, 8), (70, 1, 136, 2)], ids=str)
def test_conv_steps_follow_a_prompt(shape, dtype):
    """A prompt of ragged lengths into a pool, then single tokens: the same as whole sequences; idle sequences and the
    pool's other places stay as they are."""
    import torch
    B, _, D, K = shape
    L, steps = 6, 5
    rng = np.random.default_rng(3)
    x, w, bias = values(rng, B, L + steps, D, dtype=dtype), values(rng, D, K, std=0.6, dtype=dtype), values(rng, D, std=0.3)
    n = lengths_for(rng, B, L)
    pool = B + 4
    slots = rng.permutation(pool)[:B].astype(np.int32)
    slots[-1] = -1 if B % 2 else pool         # idle
    kd = kind_of(dtype)
    states = device(values(rng, pool, K - 1, D, dtype=dtype)).to(kd)
    before = states.clone()
    states[torch.from_numpy(slots[:-1].astype(np.int64)).to("cuda:0")] = 0
    dw, dbias, dslots, dn = device(w).to(kd), device(bias), device(slots), device(n)
    y = torch.full((B, L, D), float("nan"), device="cuda:0", dtype=kd)
    seq.ucd_causal_conv_fwd(seq.causal_conv(B, L, D, K, act=1, dtype=dtype, n_slots=pool), device(x[:, :L]).to(kd), dw, dbias, y,
                            lengths=dn, slots=dslots, state_in=states, state_out=states)
    seen = [x[b, :n[b]] for b in range(B)]
    step = seq.causal_conv(B, 1, D, K, act=1, dtype=dtype, n_slots=pool)
    for i in range(steps):
        new = x[:, L + i]
        y1 = torch.full((B, 1, D), float("nan"), device="cuda:0", dtype=kd)
        seq.ucd_causal_conv_step(step, device(new[:, None]).to(kd), dw, dbias, states, y1, slots=dslots)
        seen = [np.concatenate([s, new[b:b + 1]]) for b, s in enumerate(seen)]
        for b in range(B - 1):
            ref, tail = os_.conv_fwd(seen[b][None], w, bias, True)
            check(y1[b, 0].float().cpu().numpy(), ref[0, -1], dtype, (i, b))
            if K > 1:
                assert np.array_equal(states[int(slots[b])].float().cpu().numpy(), tail[0])
        assert not y1[B - 1].any()
    assert not y[B - 1].any()
    others = [p for p in range(pool) if p not in set(slots[:-1].tolist())]
    assert torch.equal(states[others], before[others])


def test_conv_no_tokens():
    """L = 0: the state is handed on, the gradients of the weights are 0."""
    import torch
    desc = seq.causal_conv(2, 0, 16, 4)
    st = torch.randn(2, 3, 16, device="cuda:0")
    out, w = torch.empty_like(st), torch.randn(16, 4, device="cuda:0")
    seq.ucd_causal_conv_fwd(desc, None, w, None, None, state_in=st, state_out=out)
    assert torch.equal(out, st)
    dw, dst = torch.full((16, 4), float("nan"), device="cuda:0"), torch.empty_like(st)
    ws, nbytes, _ = workspace(seq.ucd_causal_conv_workspace_size(desc))
    seq.ucd_causal_conv_bwd(desc, None, w, None, None, None, dw, None, state_in=st, dstate_out=out, dstate_in=dst, ws=ws, ws_bytes=nbytes)
    assert not dw.any() and torch.equal(dst, out)
