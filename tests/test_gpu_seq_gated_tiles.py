"""Gated projection: every kind of tile that its three products take, in both types, over many steps and with ragged ends, against the formulas in 64 bits."""
import numpy as np
import pytest

from paper_1804_04806_amd import seq
from seq_helpers import BF16, F32_ELEMENT, F32_L2, Placed, kind_of, workspace
from test_seq_gated_plan import SIDES

pytestmark = pytest.mark.gpu


def close(got, ref, squares, dtype, what):
    """fp32 as elsewhere.  bf16: an element's own rounding, 2^-8 of it, and where dgate and dup were rounded before their products, which is 2^-8 of each at
    most and independent of one another, a variance of 2^-16 / 3 of its terms' squares: none of some ten million elements is six standard
    deviations off.  In the 2-norm 2^-8 for each."""
    import torch
    got = torch.from_numpy(got).cuda().double().reshape(ref.shape)
    assert bool(torch.isfinite(got).all()), what
    norm, rms = float(ref.norm()), float(ref.square().mean().sqrt())
    roundings = 0 if dtype == 0 else 1 if squares is None else 2
    apart = float((got - ref).norm()) / norm
    assert apart <= F32_L2 + roundings * BF16, (what, apart)
    allowed = F32_ELEMENT * ref.abs().clamp(min=rms)
    if dtype == 1:
        allowed += BF16 * ref.abs()
        if squares is not None:
            allowed += 6 * BF16 / np.sqrt(3) * squares.sqrt()
    most = float(((got - ref).abs() / allowed).max())
    assert most <= 1, (what, most)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("shape", SIDES, ids=str)
def test_tiles(shape, dtype):
    import torch
    M, D, F = shape
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(sum(shape))

    def new(*s, std):
        return (torch.randn(s, device="cuda:0", generator=gen) * std).to(kind_of(dtype))
    x, dy, wg, wu = new(M, D, std=1.0), new(M, F, std=0.3), new(F, D, std=1.5 * D ** -0.5), new(F, D, std=1.5 * D ** -0.5)
    old = [new(F, D, std=M ** 0.5) for _ in range(2)]
    desc = seq.gated_projection(M, D, F, seq.ACT_SILU, dtype)
    y, dx = Placed((1, M, F), dtype), Placed((1, M, D), dtype)
    saved, saved_bytes, saved_check = workspace(seq.ucd_gated_projection_saved_size(desc))
    ws, ws_bytes, ws_check = workspace(max(seq.ucd_gated_projection_workspace_size(desc, d) for d in (seq.FWD, seq.BWD)))
    x64, wg64, wu64, dy64 = (t.double() for t in (x, wg, wu, dy))
    gate, up = x64 @ wg64.t(), x64 @ wu64.t()
    s = torch.sigmoid(gate)
    value, slope = gate * s, s * (1 + gate * (1 - s))
    for kept in (None, saved):
        y.t.fill_(Placed.POISON)
        seq.ucd_gated_projection_fwd(desc, x, wg, wu, y.ptr(), saved=kept, saved_bytes=saved_bytes if kept else None, ws=ws, ws_bytes=ws_bytes)
        close(y.get(), value * up, None, dtype, "y")
    dgate, dup = dy64 * up * slope, dy64 * value
    for beta in (0.0, 1.0):
        dwg, dwu = Placed((1, F, D), dtype), Placed((1, F, D), dtype)
        if beta:
            dwg.t.copy_(old[0]), dwu.t.copy_(old[1])
        seq.ucd_gated_projection_bwd(desc, x, wg, wu, dy, saved, dx.ptr(), dwg.ptr(), dwu.ptr(), beta=beta, saved_bytes=saved_bytes, ws=ws,
                                     ws_bytes=ws_bytes)
        close(dx.get(), dgate @ wg64 + dup @ wu64, dgate ** 2 @ wg64 ** 2 + dup ** 2 @ wu64 ** 2, dtype, "dx")
        for got, side, before, what in ((dwg, dgate, old[0], "dw_gate"), (dwu, dup, old[1], "dw_up")):
            close(got.get(), side.t() @ x64 + beta * before.double(), (side.t() ** 2) @ x64 ** 2, dtype, what)
    saved_check(), ws_check()
