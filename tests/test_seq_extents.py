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
