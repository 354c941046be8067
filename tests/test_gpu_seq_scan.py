"""Selective scan against the 64-bit oracle: one to 64 states, groups, single tokens to long sequences, odd channels, strides,
lengths with empty sequences, states in pools, gradients of everything, and what single tokens make of a prompt's state."""
import numpy as np
import pytest

from oracle import seq as os_
from paper_1804_04806_amd import seq
from seq_helpers import Placed, check, device, kind_of, lengths_for, values, workspace

pytestmark = pytest.mark.gpu

# B, L, D, N, G
SHAPES = [(1, 1, 64, 16, 1), (2, 5, 64, 16, 1), (3, 64, 128, 16, 2), (2, 33, 77, 13, 7), (1, 130, 96, 64, 1), (2, 17, 40, 1, 1), (1, 400, 16, 16, 1),
          (2, 70, 200, 32, 2), (1, 40, 12, 5, 4), (5, 31, 264, 8, 1), (1, 1300, 8, 16, 1), (2, 19, 3, 64, 3), (40, 9, 48, 16, 1), (1, 257, 130, 21, 1),
          (2, 16, 1, 2, 1)]


def inputs(shape, dtype, seed, scale=1.0):
    B, L, D, N, G = shape
    rng = np.random.default_rng(seed)
    step = np.exp(rng.uniform(np.log(1e-3), np.log(1e-1), D))
    v = {"u": values(rng, B, L, D, dtype=dtype), "dt": values(rng, B, L, D, std=0.5 * scale, dtype=dtype),
         "A": (-np.arange(1, N + 1) * rng.uniform(0.7, 1.3, (D, N))).astype(np.float32), "Bm": values(rng, B, L, G, N, dtype=dtype),
         "Cm": values(rng, B, L, G, N, dtype=dtype), "skip": values(rng, D), "z": values(rng, B, L, D, dtype=dtype),
         "dt_bias": (step + np.log(-np.expm1(-step))).astype(np.float32), "state": values(rng, B, D, N, std=0.5)}
    return v, values(rng, B, L, D, std=0.3, dtype=dtype), values(rng, B, D, N, std=0.3), rng


def run(shape, dtype, seed=0, lengths=False, state=True, without=(), softplus=True, strides=False, beta=0.0, scale=1.0, shift=0, l2=1e-5):
    B, L, D, N, G = shape
    v, dy, dstate, rng = inputs(shape, dtype, seed, scale)
    for name in without:
        v[name] = None
    if not softplus:
        v["dt"] = np.abs(v["dt"]) * np.float32(0.25)
        v["dt_bias"] = np.abs(v["dt_bias"]) * np.float32(0.01)   # steps are positive: a negative one times A grows beyond fp32
    n = lengths_for(rng, B, L) if lengths else None
    if lengths:
        for b in range(B):
            for name in ("u", "dt", "Bm", "Cm", "z"):
                if v[name] is not None:
                    v[name][b, n[b]:] = np.nan
            dy[b, n[b]:] = np.nan
    if not state:
        v["state"] = None
    width = {"u": D, "dt": D, "Bm": G * N, "Cm": G * N, "z": D, "y": D}
    st = {k: None for k in width}
    if strides is True:
        st = {k: (L * (w + 4 * i + 4) + 8, w + 4 * i + 4) for i, (k, w) in enumerate(width.items())}
    elif strides == "tokens first":
        st = {k: (w, B * w) for k, w in width.items()}
    desc = seq.scan(B, L, D, N, G, dtype=dtype, softplus=softplus, **{k + "_stride": s or (0, 0) for k, s in st.items()})
    p, grads = {}, {}
    for name in ("u", "dt", "Bm", "Cm", "z"):
        if v[name] is not None:
            p[name] = Placed(v[name].shape, dtype, st[name], v[name], shift)
            grads[name] = Placed(v[name].shape, dtype, st[name], shift=shift)
    py, pdy = Placed(dy.shape, dtype, st["y"], shift=shift), Placed(dy.shape, dtype, st["y"], dy, shift)
    old = {}
    for name in ("A", "skip", "dt_bias"):
        if v[name] is not None:
            old[name] = rng.standard_normal(v[name].shape).astype(np.float32)
            p[name], grads[name] = device(v[name]), device(old[name])
    given = {k: (t.ptr() if isinstance(t, Placed) else t) for k, t in p.items()}
    five = [given.pop(k) for k in ("u", "dt", "A", "Bm", "Cm")]
    given["lengths"] = device(n)
    pin, pout = device(v["state"]), Placed((B, D, N), 0)
    saved, saved_bytes, saved_guard = workspace(seq.ucd_scan_saved_size(desc))
    ws, nbytes, guard = workspace(seq.ucd_scan_workspace_size(desc, seq.FWD))
    seq.ucd_scan_fwd(desc, *five, py.ptr(), state_in=pin, state_out=pout.ptr(), saved=saved, saved_bytes=saved_bytes, ws=ws, ws_bytes=nbytes,
                     **given)
    guard(), saved_guard()
    ws, nbytes, guard = workspace(seq.ucd_scan_workspace_size(desc, seq.BWD))
    pds, pdin = Placed((B, D, N), 0, data=dstate), Placed((B, D, N), 0)
    out = {k: (t.ptr() if isinstance(t, Placed) else t) for k, t in grads.items()}
    seq.ucd_scan_bwd(desc, *five, pdy.ptr(), saved, out["u"], out["dt"], out["A"], out["Bm"], out["Cm"], dskip=out.get("skip"),
                     dz=out.get("z"), ddt_bias=out.get("dt_bias"), dstate_out=pds.ptr(), dstate_in=pdin.ptr(), beta=beta,
                     saved_bytes=saved_bytes, ws=ws, ws_bytes=nbytes, **given)
    guard()
    y, last = os_.scan_fwd(softplus=softplus, lengths=n, **v)
    ref = os_.scan_bwd(dy=dy, softplus=softplus, lengths=n, dstate_out=dstate, **v)
    check(py.get(), y, dtype, "y", l2=l2)
    check(pout.get(), last, 0, "state", l2=l2)
    for name in ("u", "dt", "Bm", "Cm", "z"):
        if name in grads:
            check(grads[name].get(), ref[name], dtype, "d" + name, l2=l2)
    for name in old:
        check(grads[name].cpu().numpy(), ref[name] + beta * old[name], 0, "d" + name, l2=l2)
    check(pdin.get(), ref["state"], 0, "dstate", l2=l2)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_scan(shape, dtype):
    run(shape, dtype)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_scan_lengths(shape, dtype):
    run(shape, dtype, seed=1, lengths=True, state=shape[0] % 2 == 0)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("strides", [True, "tokens first"])
@pytest.mark.parametrize("shape", [SHAPES[2], SHAPES[3], SHAPES[7]], ids=str)
def test_scan_strides(shape, strides, dtype):
    run(shape, dtype, seed=2, strides=strides, lengths=True, shift=1 if strides is True and dtype == 1 else 0)


@pytest.mark.parametrize("without", [("z",), ("skip",), ("dt_bias",), ("skip", "z", "dt_bias")], ids=str)
def test_scan_without(without):
    run(SHAPES[2], 0, seed=3, without=without, state=False)
    run(SHAPES[3], 1, seed=3, without=without)


def test_scan_plain_steps_and_accumulation():
    run(SHAPES[2], 0, seed=4, softplus=False)
    run(SHAPES[3], 0, seed=5, beta=1.0)


def test_scan_large_steps():
    """dt beyond softplus' bend on both sides: decays that underflow to 0, and steps that are all but 0."""
    run(SHAPES[2], 0, seed=6, scale=40.0)


def test_scan_not_finite_stays_in_its_channel():
    """A NaN in one channel's input, and what it leaves of the others."""
    import torch
    B, L, D, N, G = 2, 50, 70, 16, 1
    v, *_ = inputs((B, L, D, N, G), 0, 7)
    outs = []
    for bad in (False, True):
        t = {k: device(a) for k, a in v.items()}
        if bad:
            t["u"][0, 20, 33] = float("nan")
            t["dt"][1, 10, 5] = float("inf")
        y, last = torch.empty(B, L, D, device="cuda:0"), torch.empty(B, D, N, device="cuda:0")
        ws, nbytes, _ = workspace(seq.ucd_scan_workspace_size(seq.scan(B, L, D, N, G), seq.FWD))
        seq.ucd_scan_fwd(seq.scan(B, L, D, N, G), t["u"], t["dt"], t["A"], t["Bm"], t["Cm"], y, z=t["z"], state_in=t["state"], state_out=last,
                         ws=ws, ws_bytes=nbytes)
        outs.append((y.cpu().numpy(), last.cpu().numpy()))
    (y0, s0), (y1, s1) = outs
    mask = np.zeros((B, L, D), bool)
    mask[0, 20:, 33] = True
    assert np.isnan(y1[mask]).all()
    mask[1, 10:, 5] = True
    assert np.array_equal(y0[~mask], y1[~mask])
    keep = np.ones((B, D), bool)
    keep[0, 33] = keep[1, 5] = False
    assert np.array_equal(s0[keep], s1[keep])


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("shape", [(5, 1, 64, 16, 1), (3, 1, 77, 13, 7), (4, 1, 24, 1, 1), (3, 1, 40, 64, 2), (34, 1, 136, 8, 1), (2, 1, 130, 32, 1)],
                         ids=str)
def test_scan_steps_follow_a_prompt(shape, dtype):
    """A prompt of ragged lengths into a pool, then single tokens: the same as whole sequences; idle sequences and the pool's
    other places stay as they are."""
    import torch
    B, _, D, N, G = shape
    L, steps = 7, 4
    v, _, _, rng = inputs((B, L + steps, D, N, G), dtype, 8)
    v.pop("state")
    n = lengths_for(rng, B, L)
    pool = B + 4
    slots = rng.permutation(pool)[:B].astype(np.int32)
    slots[-1] = -7 if B % 2 else pool         # idle
    kd = kind_of(dtype)
    states = device(values(rng, pool, D, N))
    before = states.clone()
    states[torch.from_numpy(slots[:-1].astype(np.int64)).to("cuda:0")] = 0
    dslots = device(slots)
    tok = ("u", "dt", "Bm", "Cm", "z")
    w = {k: device(v[k]) for k in ("A", "skip", "dt_bias")}

    def call(part):
        t = {k: device(v[k][:, part]).to(kd) for k in tok}
        return [t["u"], t["dt"], w["A"], t["Bm"], t["Cm"]], dict(skip=w["skip"], dt_bias=w["dt_bias"], z=t["z"], slots=dslots)
    five, more = call(slice(0, L))
    desc = seq.scan(B, L, D, N, G, dtype=dtype, n_slots=pool)
    y = torch.full((B, L, D), float("nan"), device="cuda:0", dtype=kd)
    ws, nbytes, _ = workspace(seq.ucd_scan_workspace_size(desc, seq.FWD))
    seq.ucd_scan_fwd(desc, *five, y, state_in=states, state_out=states, lengths=device(n), ws=ws, ws_bytes=nbytes, **more)
    assert not y[B - 1].any()
    step = seq.scan(B, 1, D, N, G, dtype=dtype, n_slots=pool)
    for i in range(steps):
        five, more = call(slice(L + i, L + i + 1))
        y1 = torch.full((B, 1, D), float("nan"), device="cuda:0", dtype=kd)
        seq.ucd_scan_step(step, *five, states, y1, **more)
        for b in range(B - 1):
            at = list(range(n[b])) + list(range(L, L + i + 1))
            whole = {k: v[k][b:b + 1, at] if k in tok else v[k] for k in v}
            ref, last = os_.scan_fwd(**whole)
            check(y1[b, 0].float().cpu().numpy(), ref[0, -1], dtype, (i, b))
            check(states[int(slots[b])].cpu().numpy(), last[0], 0, (i, b))
        assert not y1[B - 1].any()
    others = [q for q in range(pool) if q not in set(slots[:-1].tolist())]
    assert torch.equal(states[others], before[others])


def test_scan_no_tokens():
    """L = 0: the state is handed on, its gradient handed back, the gradients of the weights are 0."""
    import torch
    desc = seq.scan(2, 0, 16, 8)
    st, A = torch.randn(2, 16, 8, device="cuda:0"), -torch.rand(16, 8, device="cuda:0")
    out = torch.empty_like(st)
    seq.ucd_scan_fwd(desc, None, None, A, None, None, None, state_in=st, state_out=out, ws=workspace(1 << 16)[0], ws_bytes=1 << 16)
    assert torch.equal(out, st)
    dA, dst = torch.full((16, 8), float("nan"), device="cuda:0"), torch.empty_like(st)
    saved, saved_bytes, _ = workspace(max(16, seq.ucd_scan_saved_size(desc)))
    ws, nbytes, _ = workspace(max(16, seq.ucd_scan_workspace_size(desc, seq.BWD)))
    seq.ucd_scan_bwd(desc, None, None, A, None, None, None, saved, None, None, dA, None, None, dstate_out=st, dstate_in=dst,
                     saved_bytes=saved_bytes, ws=ws, ws_bytes=nbytes)
    assert not dA.any() and torch.equal(dst, st)


@pytest.mark.parametrize("dtype", [0, 1])
def test_scan_gradients_repeat(dtype):
    """Sums are taken in a fixed order: the same bits each time."""
    import torch
    B, L, D, N, G = 3, 200, 300, 16, 2
    v, dy, _, _ = inputs((B, L, D, N, G), dtype, 9)
    kd = kind_of(dtype)
    t = {k: device(a).to(kd if k in ("u", "dt", "Bm", "Cm", "z") else torch.float32) for k, a in v.items()}
    desc, d = seq.scan(B, L, D, N, G, dtype=dtype), device(dy).to(kd)
    got = []
    for _ in range(3):
        y = torch.empty_like(d)
        saved, ws = (torch.full((max(16, n),), 255, dtype=torch.uint8, device="cuda:0") for n in
                     (seq.ucd_scan_saved_size(desc), max(seq.ucd_scan_workspace_size(desc, k) for k in (0, 1))))
        five = [t[k] for k in ("u", "dt", "A", "Bm", "Cm")]
        more = dict(skip=t["skip"], z=t["z"], dt_bias=t["dt_bias"])
        seq.ucd_scan_fwd(desc, *five, y, saved=saved, ws=ws, **more)
        out = [torch.empty_like(a) for a in five]
        extra = {"d" + k: torch.empty_like(a) for k, a in more.items()}
        seq.ucd_scan_bwd(desc, *five, d, saved, *out, ws=ws, **more, **extra)
        got.append([y] + out + list(extra.values()))
    assert all(torch.equal(a, b) for other in got[1:] for a, b in zip(got[0], other))
