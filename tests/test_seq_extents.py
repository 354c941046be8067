"""The sequence operators' largest extents, on the host: what a descriptor may not have is refused by every entry point, and the
sizes of the largest that it may have are those of the formulas, not of sums that ran over."""
import pytest

from paper_1804_04806_amd import seq, ucd

P, MOST = 1 << 20, 1 << 30        # an aligned address that is never read; the largest extent
WS = dict(ws=P, ws_bytes=(1 << 64) - 1, stream=0)


def refused(call, *args, **kw):
    with pytest.raises(ucd.UcdError) as e:
        call(*args, **kw)
    assert e.value.status == ucd.E_INVALID, e.value.status


BEYOND = [MOST + 1, (1 << 31) - 33, (1 << 31) - 16, (1 << 31) - 1]


@pytest.mark.parametrize("n", BEYOND)
@pytest.mark.parametrize("name", ["N", "S"])
def test_norm_beyond(name, n):
    desc = seq.group_norm(**{**dict(N=1, S=1, C=1, G=1), name: n})
    assert seq.ucd_group_norm_workspace_size(desc, seq.FWD) == seq.ucd_group_norm_workspace_size(desc, seq.BWD) == ucd.WS_NA
    refused(seq.ucd_group_norm_fwd, desc, P, P, P, P, **WS)
    refused(seq.ucd_group_norm_bwd, desc, P, P, P, P, P, P, P, P, **WS)


@pytest.mark.parametrize("n", BEYOND)
@pytest.mark.parametrize("name", ["B", "L"])
def test_conv_beyond(name, n):
    desc = seq.causal_conv(**{**dict(B=1, L=1, D=4, K=4), name: n})
    assert seq.ucd_causal_conv_workspace_size(desc) == ucd.WS_NA
    refused(seq.ucd_causal_conv_fwd, desc, P, P, P, P, stream=0)
    refused(seq.ucd_causal_conv_bwd, desc, P, P, P, P, P, P, P, **WS)
    refused(seq.ucd_causal_conv_step, desc, P, P, P, P, P, stream=0)


@pytest.mark.parametrize("n", BEYOND)
@pytest.mark.parametrize("name", ["B", "L"])
def test_scan_beyond(name, n):
    desc = seq.scan(**{**dict(B=1, L=1, D=4, N=4), name: n})
    assert {seq.ucd_scan_workspace_size(desc, seq.FWD), seq.ucd_scan_workspace_size(desc, seq.BWD),
            seq.ucd_scan_saved_size(desc)} == {ucd.WS_NA}
    refused(seq.ucd_scan_fwd, desc, P, P, P, P, P, P, saved=P, saved_bytes=(1 << 64) - 1, **WS)
    refused(seq.ucd_scan_bwd, desc, P, P, P, P, P, P, P, P, P, P, P, P, saved_bytes=(1 << 64) - 1, **WS)
    refused(seq.ucd_scan_step, desc, P, P, P, P, P, P, P, stream=0)


@pytest.mark.parametrize("n", [MOST, MOST - 1, MOST - 31])
def test_the_largest(n):
    # partial sums of dw and dbias by 2048 rows of workgroups, which half as many tokens fill as well
    size = seq.ucd_causal_conv_workspace_size
    assert size(seq.causal_conv(1, n, 4, 4)) == size(seq.causal_conv(1, n // 2, 4, 4)) == 4 * 2048 * 5 * 4
    # states every eight tokens, two to a tile of 16
    assert seq.ucd_scan_saved_size(seq.scan(1, n, 4, 4)) == 4 * ((n + 15) // 16) * 2 * 4 * 4
    # sums of dBm and dCm of every tile, 64 segments' states, steps and sums of weights
    need = 4 * ((n + 15) // 16) * 16 * 2 * 4
    assert need < seq.ucd_scan_workspace_size(seq.scan(1, n, 4, 4), seq.BWD) < need + 65 * 4 * (4 * 4 + 4 + 4 * 6)
    assert seq.ucd_group_norm_workspace_size(seq.group_norm(n, 1, 1, 1), seq.FWD) == 0


ANY = [1, 1 << 26, 1 << 41, 1 << 62]       # strides that an extent of one never takes


@pytest.mark.parametrize("inner", [1] + ANY)
def test_channels_beyond(inner):
    """2^25 channels are the most, also where there is a single token whose stride says nothing about them."""
    n = (1 << 25) + 64
    desc = seq.group_norm(1, 1, n, 1, x_stride=(0, inner), y_stride=(0, inner))
    assert seq.ucd_group_norm_workspace_size(desc, seq.FWD) == ucd.WS_NA
    refused(seq.ucd_group_norm_fwd, desc, P, P, P, P, **WS)
    desc = seq.causal_conv(1, 1, n, 4, x_stride=(0, inner), y_stride=(0, inner))
    assert seq.ucd_causal_conv_workspace_size(desc) == ucd.WS_NA
    refused(seq.ucd_causal_conv_step, desc, P, P, P, P, P, stream=0)
    for D, N, G in ((n, 4, 1), (1 << 20, 64, 1 << 20)):
        desc = seq.scan(1, 1, D, N, G, **{k + "_stride": (0, inner) for k in ("u", "dt", "Bm", "Cm", "z", "y")})
        assert seq.ucd_scan_saved_size(desc) == ucd.WS_NA
        refused(seq.ucd_scan_step, desc, P, P, P, P, P, P, P, stream=0)


@pytest.mark.parametrize("any", ANY)
def test_strides_of_an_extent_of_one(any):
    size = seq.ucd_group_norm_workspace_size
    assert size(seq.group_norm(5, 1, 64, 4, x_stride=(64, any), y_stride=(96, any)), seq.BWD) == size(seq.group_norm(5, 1, 64, 4), seq.BWD)
    assert size(seq.group_norm(1, 5, 64, 4, x_stride=(any, 64)), seq.BWD) == size(seq.group_norm(1, 5, 64, 4), seq.BWD)
    size = seq.ucd_causal_conv_workspace_size
    assert size(seq.causal_conv(5, 1, 64, 4, x_stride=(64, any))) == size(seq.causal_conv(5, 1, 64, 4))
    assert size(seq.causal_conv(1, 5, 64, 4, y_stride=(any, 64))) == size(seq.causal_conv(1, 5, 64, 4))
    size, names = seq.ucd_scan_saved_size, ("u", "dt", "Bm", "Cm", "z", "y")
    assert size(seq.scan(5, 1, 64, 16, **{k + "_stride": (64, any) for k in names})) == size(seq.scan(5, 1, 64, 16))
    assert size(seq.scan(1, 5, 64, 16, **{k + "_stride": (any, 64) for k in names})) == size(seq.scan(1, 5, 64, 16))


def test_pools_of_no_sequences():
    """A pool beside no sequences: the places, a tensor of no elements, have no address."""
    conv, one = seq.causal_conv(0, 3, 8, 4, n_slots=5), seq.causal_conv(0, 1, 8, 4, n_slots=5)
    for slots in (None, P):
        seq.ucd_causal_conv_fwd(conv, None, P, P, None, slots=slots, state_in=P, state_out=P, stream=0)
        seq.ucd_causal_conv_step(one, None, P, P, P, None, slots=slots, stream=0)
        seq.ucd_scan_fwd(seq.scan(0, 3, 8, 4, n_slots=5), None, None, P, None, None, None, slots=slots, state_in=P, state_out=P, **WS)
        seq.ucd_scan_step(seq.scan(0, 1, 8, 4, n_slots=5), None, None, P, None, None, P, None, slots=slots, stream=0)


def test_too_many_workgroups():
    """Extents that are allowed each, in calls that are too large to be counted."""
    def unsupported(call, *args, **kw):
        with pytest.raises(ucd.UcdError) as e:
            call(*args, **kw)
        assert e.value.status == ucd.E_UNSUPPORTED, e.value.status
    conv = seq.causal_conv(MOST, 8, 1, 4)
    unsupported(seq.ucd_causal_conv_fwd, conv, P, P, P, P, stream=0)
    unsupported(seq.ucd_causal_conv_bwd, conv, P, P, P, P, P, P, P, **WS)
    scan = seq.scan(MOST, 1, 16, 4)
    unsupported(seq.ucd_scan_fwd, scan, P, P, P, P, P, P, **WS)
    unsupported(seq.ucd_scan_step, scan, P, P, P, P, P, P, P, stream=0)
