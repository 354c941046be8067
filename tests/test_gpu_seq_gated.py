"""Gated projection against the 64-bit oracle: single tokens to hundreds, rows of odd lengths, both types, all activations, strides and
addresses, gradients, gradients in parts, no tokens."""
import numpy as np
import pytest

from oracle import seq as os_
from paper_1804_04806_amd import seq
from seq_helpers import BF16, F32_ELEMENT, F32_L2, Placed, check, values, workspace

pytestmark = pytest.mark.gpu

# M, D, F
SHAPES = [(1, 1, 1), (1, 64, 128), (3, 40, 24), (16, 200, 33), (17, 512, 48), (64, 96, 130), (65, 64, 64), (70, 33, 35), (128, 128, 128), (200, 72, 300),
          (129, 257, 65), (300, 1000, 40), (1000, 24, 520), (512, 640, 1152)]

# y in bf16 is rounded once, its sums are fp32.  Gradients: dgate and dup are rounded once to bf16 (fp32: three parts of bf16, 2^-24) before their
# products; those errors are independent, 2^-8 of their terms at most, so that in the 2-norm they are 2^-8 of the result, and for an element at
# most six standard deviations, 6 * 2^-8 / sqrt(3) < 4 * 2^-8 of the rms, beside its own rounding.
L2, ELEMENT = {0: F32_L2, 1: BF16}, {0: F32_ELEMENT, 1: 4 * BF16}


def run(shape, dtype, act=1, seed=0, stride=0, shift=0, w_shift=0, beta=0.0):
    M, D, F = shape
    rng = np.random.default_rng(seed)
    x, dy = values(rng, M, D, dtype=dtype), values(rng, M, F, std=0.3, dtype=dtype)
    wg, wu = (values(rng, F, D, std=1.5 * D ** -0.5, dtype=dtype) for _ in range(2))
    old = [values(rng, F, D, std=float(M) ** 0.5, dtype=dtype) for _ in range(2)]
    xs, ys = ((M * (D + stride), D + stride), (M * (F + stride), F + stride)) if stride else (None, None)
    px, pdx = Placed((1, M, D), dtype, xs, x[None], shift), Placed((1, M, D), dtype, xs, shift=shift)
    py, pdy = Placed((1, M, F), dtype, ys, shift=shift), Placed((1, M, F), dtype, ys, dy[None], shift)
    pg, pu = (Placed((1, F, D), dtype, None, w[None], w_shift) for w in (wg, wu))
    dg, du = (Placed((1, F, D), dtype, shift=w_shift) for _ in range(2))
    if beta:
        import torch
        for p, o in zip((dg, du), old):
            p.t.copy_(torch.from_numpy(o[None]))
    desc = seq.gated_projection(M, D, F, act, dtype, D + stride if stride else 0, F + stride if stride else 0)
    ws, ws_bytes, ws_check = workspace(seq.ucd_gated_projection_workspace_size(desc, seq.FWD))
    saved, saved_bytes, saved_check = workspace(seq.ucd_gated_projection_saved_size(desc))
    ref = os_.gated_fwd(x, wg, wu, act)
    for kept in (None, saved):
        py.t.fill_(Placed.POISON)
        seq.ucd_gated_projection_fwd(desc, px.ptr(), pg.ptr(), pu.ptr(), py.ptr(), saved=kept, saved_bytes=saved_bytes if kept else None, ws=ws,
                                     ws_bytes=ws_bytes)
        check(py.get()[0], ref, dtype, "y")
    ws_check(), saved_check()
    ws, ws_bytes, ws_check = workspace(seq.ucd_gated_projection_workspace_size(desc, seq.BWD))
    seq.ucd_gated_projection_bwd(desc, px.ptr(), pg.ptr(), pu.ptr(), pdy.ptr(), saved, pdx.ptr(), dg.ptr(), du.ptr(), beta=beta,
                                 saved_bytes=saved_bytes, ws=ws, ws_bytes=ws_bytes)
    ws_check()
    dx, dwg, dwu = os_.gated_bwd(x, wg, wu, act, dy)
    check(pdx.get()[0], dx, dtype, "dx", L2[dtype], ELEMENT[dtype])
    # An element of a weight's gradient is a sum over the tokens: where they are few its error is not that of the mean element, but at most 2^-8 of
    # sum |dG| |x| (each term's dG rounded once), which holds for every element whatever the tokens are, beside its own
    # rounding (1.01: of one by the other, and sums in fp32); the 2-norm's share is that of many.
    value, slope = os_.gate_act(x.astype(np.float64) @ wg.T.astype(np.float64), act)
    sides = dy * (x.astype(np.float64) @ wu.T.astype(np.float64)) * slope, dy * value
    for got, want, before, side, what in ((dg, dwg, old[0], sides[0], "dw_gate"), (du, dwu, old[1], sides[1], "dw_up")):
        want, got = want + beta * before, got.get()[0]
        if M > 64 or dtype == 0:
            check(got, want, dtype, what, L2[dtype], ELEMENT[dtype])
            continue
        check(got, want, dtype, what, L2[dtype], np.inf)
        room = BF16 * (np.abs(side).T @ np.abs(x)) + BF16 * np.abs(want)
        assert (np.abs(got - want) <= 1.01 * room + F32_ELEMENT).all(), what


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_against_oracle(shape, dtype):
    run(shape, dtype, seed=sum(shape))


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("act", [0, 2])
@pytest.mark.parametrize("shape", [(7, 64, 40), (150, 96, 72)], ids=str)
def test_activations(shape, act, dtype):
    run(shape, dtype, act, 1)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("stride,shift,w_shift", [(8, 0, 0), (3, 0, 0), (0, 1, 0), (0, 0, 1), (5, 3, 1)])
@pytest.mark.parametrize("M", [5, 140])
def test_strides_and_addresses(M, stride, shift, w_shift, dtype):
    run((M, 64, 72), dtype, 1, 2, stride, shift, w_shift)


@pytest.mark.parametrize("dtype", [0, 1])
def test_gradients_in_parts(dtype):
    run((150, 72, 136), dtype, 1, 3, beta=1.0)
    run((40, 33, 35), dtype, 1, 3, beta=1.0)


@pytest.mark.parametrize("dtype", [0, 1])
def test_large_tiles(dtype):
    """Enough tiles for those of 256 by 256 in all three products, the last of each ragged."""
    run((4100, 4104, 2080), dtype, 1, 4) if dtype == 1 else run((4100, 1032, 2080), dtype, 1, 4)


@pytest.mark.parametrize("M, D, F, act", [(17, 4096, 8192, 1), (33, 2048, 8200, 2), (64, 8192, 2050, 1)])
def test_few_tokens_of_large_weights(M, D, F, act):
    """Tiles of 64 tokens, with and without parts of the reduction; and rows that lie askew, which are read as they are, without a workspace's use."""
    run((M, D, F), 1, act, 6)
    run((M, D, F), 1, act, 7, shift=1, w_shift=1)


@pytest.mark.parametrize("dtype", [0, 1])
def test_no_tokens(dtype):
    import torch
    kind = torch.bfloat16 if dtype == 1 else torch.float32
    D, F = 24, 40
    desc = seq.gated_projection(0, D, F, dtype=dtype)
    w = torch.ones(F, D, dtype=kind, device="cuda:0")
    seq.ucd_gated_projection_fwd(desc, None, w, w, None)
    for beta, want in ((1.0, 3.0), (0.0, 0.0)):
        dg, du = (torch.full((F, D), 3.0, dtype=kind, device="cuda:0") for _ in range(2))
        seq.ucd_gated_projection_bwd(desc, None, w, w, None, None, None, dg, du, beta=beta)
        assert bool((dg == want).all()) and bool((du == want).all())


def test_saturated_gates():
    """Gates whose sigmoid is 0 or 1, and cubes beyond the type's range."""
    import torch
    for act in (1, 2):
        x = torch.tensor([[1e4], [-1e4], [3e15], [-3e15], [0.0]], device="cuda:0")
        one = torch.ones(1, 1, device="cuda:0")
        desc = seq.gated_projection(5, 1, 1, act, 0)
        y, saved = torch.empty(5, 1, device="cuda:0"), torch.empty(seq.ucd_gated_projection_saved_size(desc), dtype=torch.uint8, device="cuda:0")
        ws = torch.empty(max(16, *(seq.ucd_gated_projection_workspace_size(desc, d) for d in (seq.FWD, seq.BWD))), dtype=torch.uint8, device="cuda:0")
        seq.ucd_gated_projection_fwd(desc, x, one, one, y, saved=saved, ws=ws)
        want = torch.tensor([[1e8], [0.0], [9e30], [0.0], [0.0]], device="cuda:0")
        assert torch.allclose(y, want, rtol=1e-5, atol=0)
        dx, dg, du = torch.empty_like(x), torch.empty_like(one), torch.empty_like(one)
        seq.ucd_gated_projection_bwd(desc, x, one, one, torch.ones_like(y), saved, dx, dg, du, ws=ws)
        # y = x act(x): its derivative is 2 x where the gate is open and 0 where it is shut
        want = torch.tensor([[2e4], [0.0], [6e15], [0.0], [0.0]], device="cuda:0")
        assert torch.allclose(dx, want, rtol=1e-5, atol=0)
