"""Rows that are no whole packs, or begin between their multiples: the packs at the rows' ends reach back into other lanes', waves', groups' or
workgroups' channels, which have to stay theirs.  Against the 64-bit oracle, with the other tests' inputs and tolerances."""
import numpy as np
import pytest

import test_gpu_seq_conv as conv
import test_gpu_seq_norm as norm
import test_gpu_seq_scan as scan
from oracle import seq as os_
from paper_1804_04806_amd import seq
from seq_helpers import check, device, kind_of, values

pytestmark = pytest.mark.gpu

# N, S, C, G: single positions with one pack to a lane, with several, too many for a wave; slabs of several groups, of one; parts of a group, of positions
NORMS = [(3, 1, 33, 3), (5, 1, 682, 2), (3, 1, 2047, 1), (2, 1, 4101, 1), (3, 1, 8190, 2), (3, 40, 34, 2), (2, 1024, 51, 3), (2, 100, 511, 1),
         (3, 50, 4001, 1), (1, 3, 20001, 1), (1, 9000, 27, 1), (1, 5000, 2051, 1), (2, 300, 100, 4)]


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("shape", NORMS, ids=str)
def test_norm_groups_of_no_whole_packs(shape, dtype):
    norm.compare(*norm.run(shape, dtype, True, seed=11), dtype)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("shape", [NORMS[1], NORMS[2], NORMS[5], NORMS[8], (2, 1, 64, 2), (2, 49, 64, 4), (1, 9000, 64, 2)], ids=str)
def test_norm_rows_anywhere(shape, dtype):
    norm.compare(*norm.run(shape, dtype, True, seed=12, strides=True, shift=1), dtype)


# B, L, D, K: a last pack of one channel in a wave, a workgroup and a run of its own
CONVS = [(2, 50, 9, 4), (2, 50, 15, 3), (3, 33, 257, 4), (2, 40, 2049, 2), (1, 70, 2055, 4), (2, 30, 129, 8), (2, 20, 3, 4)]


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("shape", CONVS, ids=str)
def test_conv_rows_of_no_whole_packs(shape, dtype):
    conv.run(shape, dtype, seed=11, lengths=True)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("shape", [CONVS[2], CONVS[4], (2, 50, 64, 4)], ids=str)
def test_conv_rows_anywhere(shape, dtype):
    conv.run(shape, dtype, seed=12, strides=True, shift=1)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("shape", CONVS + [(64, 1, 2049, 4), (64, 1, 515, 3)], ids=str)
def test_conv_state_in_place(shape, dtype):
    """Prompts and single tokens that replace the state they began with."""
    import torch
    B, L, D, K = shape
    v, _ = conv.inputs(shape, dtype, 13)
    kd = kind_of(dtype)
    x, w, bias, state = device(v["x"]).to(kd), device(v["w"]).to(kd), device(v["bias"]), device(v["state"]).to(kd)
    y = torch.full_like(x, float("nan"))
    seq.ucd_causal_conv_fwd(seq.causal_conv(B, L, D, K, act=1, dtype=dtype), x, w, bias, y, state_in=state, state_out=state)
    ref, tail = os_.conv_fwd(v["x"], v["w"], v["bias"], True, None, v["state"])
    check(y.float().cpu().numpy(), ref, dtype, "y")
    assert np.array_equal(state.float().cpu().numpy(), tail)
    new = values(np.random.default_rng(14), B, 1, D, dtype=dtype)
    y1 = torch.full((B, 1, D), float("nan"), device="cuda:0", dtype=kd)
    seq.ucd_causal_conv_step(seq.causal_conv(B, 1, D, K, act=1, dtype=dtype), device(new).to(kd), w, bias, state, y1)
    ref, tail = os_.conv_fwd(new, v["w"], v["bias"], True, None, tail)
    check(y1.float().cpu().numpy(), ref, dtype, "step")
    assert np.array_equal(state.float().cpu().numpy(), tail)


# B, L, D, N, G: groups of 4 to 6 channels, of a wave's and one, two or three more, of a workgroup's and one more; states between 5 and 63
SCANS = [(2, 37, 4, 16, 1), (2, 37, 20, 13, 4), (2, 50, 17, 16, 1), (1, 70, 36, 9, 2), (2, 33, 19, 16, 1), (1, 90, 65, 16, 1), (2, 40, 130, 6, 2),
         (1, 70, 41, 30, 1), (2, 33, 21, 63, 1), (1, 600, 35, 14, 1), (2, 48, 64, 15, 1), (1, 33, 66, 3, 2)]


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("shape", SCANS, ids=str)
def test_scan_rows_of_no_whole_packs(shape, dtype):
    scan.run(shape, dtype, seed=11)
    scan.run(shape, dtype, seed=12, lengths=True)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("shape", [SCANS[3], SCANS[5], (2, 64, 64, 16, 1), (1, 40, 64, 8, 2)], ids=str)
def test_scan_rows_anywhere(shape, dtype):
    scan.run(shape, dtype, seed=13, strides=True, shift=1)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("silu", [False, True])
@pytest.mark.parametrize("shape", [(1, 1, 1, 1), (700, 1, 33, 33), (3, 1, 100, 100)], ids=str)
def test_norm_of_single_elements_has_no_gradient(shape, silu, dtype):
    """dx is a difference of equal terms: exactly 0, not what rounding them differently would leave of it."""
    got, _ = norm.run(shape, dtype, silu, seed=15)
    assert not got["dx"].any() and not got["dgamma"].any()
