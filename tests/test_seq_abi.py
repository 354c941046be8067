"""include/ucd_seq.h and its binding without a GPU: exported names, workspace queries, and what the entry points refuse
(every refusal happens on the host, before anything is launched; the addresses below are never read)."""
import ctypes
import os
import re

import pytest

from paper_1804_04806_amd import seq, ucd

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 20   # an aligned address


def test_every_declared_symbol_is_exported():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "ucd_seq.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(ucd_[a-z_0-9]+)\s*\(", text)))
    assert names == sorted(seq.EXPORTS)
    lib = ctypes.CDLL(ucd.LIB_PATH)
    assert all(hasattr(lib, n) and hasattr(seq, n) for n in names)


def refused(status, call, *args, **kw):
    with pytest.raises(ucd.UcdError) as e:
        call(*args, **kw)
    assert e.value.status == status, (e.value.status, status)


NORM = dict(N=2, S=3, C=8, G=2)
CONV = dict(B=2, L=3, D=8, K=4)
SCAN = dict(B=2, L=3, D=8, N=16, G=2)


def norm_fwd(desc, x=P, gamma=P, beta=P, y=P, **kw):
    kw.setdefault("ws", P)
    kw.setdefault("ws_bytes", 1 << 30)
    seq.ucd_group_norm_fwd(desc, x, gamma, beta, y, stream=0, **kw)


def conv_fwd(desc, x=P, w=P, y=P, **kw):
    seq.ucd_causal_conv_fwd(desc, x, w, P, y, stream=0, **kw)


def scan_fwd(desc, u=P, A=P, y=P, **kw):
    kw.setdefault("ws", P)
    kw.setdefault("ws_bytes", 1 << 30)
    seq.ucd_scan_fwd(desc, u, P, A, P, P, y, stream=0, **kw)


@pytest.mark.parametrize("bad", [dict(N=0), dict(S=0), dict(C=9), dict(G=0), dict(G=3), dict(act=2), dict(act=-1), dict(dtype=2),
                                 dict(eps=-1e-5), dict(eps=float("nan")), dict(eps=float("inf")), dict(x_stride=(0, 7)),
                                 dict(x_stride=(23, 8)), dict(y_stride=(-24, 8)), dict(y_stride=(0, -8)), dict(x_stride=(1 << 41, 0)),
                                 dict(N=1 << 20, S=1 << 20, C=1 << 20)], ids=str)
def test_norm_descriptors(bad):
    desc = seq.group_norm(**{**NORM, **bad})
    assert seq.ucd_group_norm_workspace_size(desc, seq.FWD) == ucd.WS_NA
    refused(ucd.E_INVALID, norm_fwd, desc)


@pytest.mark.parametrize("bad", [dict(B=-1), dict(L=-1), dict(D=0), dict(K=0), dict(K=9), dict(act=2), dict(dtype=-1), dict(n_slots=-1),
                                 dict(x_stride=(0, 7)), dict(x_stride=(8, 8)), dict(y_stride=(8, 15))], ids=str)
def test_conv_descriptors(bad):
    desc = seq.causal_conv(**{**CONV, **bad})
    assert seq.ucd_causal_conv_workspace_size(desc) == ucd.WS_NA
    refused(ucd.E_INVALID, conv_fwd, desc)


@pytest.mark.parametrize("bad", [dict(B=-1), dict(L=-1), dict(D=0), dict(D=9), dict(N=0), dict(N=65), dict(G=0), dict(G=3), dict(dtype=2),
                                 dict(softplus=2), dict(n_slots=-1), dict(u_stride=(0, 7)), dict(Bm_stride=(0, 31)),
                                 dict(Cm_stride=(95, 32)), dict(z_stride=(8, 8)), dict(y_stride=(1, 0))], ids=str)
def test_scan_descriptors(bad):
    desc = seq.scan(**{**SCAN, **bad})
    assert seq.ucd_scan_workspace_size(desc, seq.FWD) == ucd.WS_NA and seq.ucd_scan_saved_size(desc) == ucd.WS_NA
    refused(ucd.E_INVALID, scan_fwd, desc)


def test_directions():
    for n in (-1, 2):
        assert seq.ucd_group_norm_workspace_size(seq.group_norm(**NORM), n) == ucd.WS_NA
        assert seq.ucd_scan_workspace_size(seq.scan(**SCAN), n) == ucd.WS_NA


def test_pointers():
    norm, conv, scan = seq.group_norm(**NORM), seq.causal_conv(**CONV), seq.scan(**SCAN)
    for name in ("x", "gamma", "beta", "y"):
        refused(ucd.E_NULLPTR, norm_fwd, norm, **{name: None})
    for name in ("x", "w", "y"):
        refused(ucd.E_NULLPTR, conv_fwd, conv, **{name: None})
    for name in ("u", "A", "y"):
        refused(ucd.E_NULLPTR, scan_fwd, scan, **{name: None})
    # alignment to the element
    refused(ucd.E_INVALID, norm_fwd, norm, x=P + 2)
    refused(ucd.E_INVALID, norm_fwd, seq.group_norm(**NORM, dtype=1), x=P + 1)
    refused(ucd.E_INVALID, conv_fwd, conv, y=P + 2)
    refused(ucd.E_INVALID, conv_fwd, conv, state_out=P + 2)
    refused(ucd.E_INVALID, scan_fwd, scan, A=P + 2)
    refused(ucd.E_INVALID, scan_fwd, scan, lengths=P + 1)
    refused(ucd.E_INVALID, scan_fwd, scan, state_in=P + 1)
    for call in (seq.ucd_group_norm_bwd,):
        refused(ucd.E_NULLPTR, call, norm, P, P, P, None, P, P, P, P, ws=P, ws_bytes=1 << 30, stream=0)
        refused(ucd.E_INVALID, call, norm, P, P, P, P, P, P, P, P, beta=0.5, ws=P, ws_bytes=1 << 30, stream=0)
    refused(ucd.E_NULLPTR, seq.ucd_causal_conv_bwd, conv, P, P, P, P, P, None, P, ws=P, ws_bytes=1 << 30, stream=0)
    refused(ucd.E_INVALID, seq.ucd_causal_conv_bwd, conv, P, P, P, P, P, P, P, beta=2.0, ws=P, ws_bytes=1 << 30, stream=0)


def test_slots_and_pools_go_together():
    refused(ucd.E_INVALID, conv_fwd, seq.causal_conv(**CONV), slots=P)
    refused(ucd.E_INVALID, conv_fwd, seq.causal_conv(**CONV, n_slots=5))
    refused(ucd.E_INVALID, scan_fwd, seq.scan(**SCAN), slots=P)
    refused(ucd.E_INVALID, scan_fwd, seq.scan(**SCAN, n_slots=5))
    # Backward has no pools
    refused(ucd.E_INVALID, seq.ucd_causal_conv_bwd, seq.causal_conv(**CONV, n_slots=5), P, P, P, P, P, P, P, ws=P, ws_bytes=1 << 30,
            stream=0)
    refused(ucd.E_INVALID, seq.ucd_scan_bwd, seq.scan(**SCAN, n_slots=5), P, P, P, P, P, P, P, P, P, P, P, P, saved_bytes=1 << 30,
            ws=P, ws_bytes=1 << 30, stream=0)


def test_steps_are_single_tokens():
    refused(ucd.E_INVALID, seq.ucd_causal_conv_step, seq.causal_conv(**CONV), P, P, P, P, P, stream=0)
    refused(ucd.E_INVALID, seq.ucd_scan_step, seq.scan(**SCAN), P, P, P, P, P, P, P, stream=0)
    conv, scan = seq.causal_conv(**{**CONV, "L": 1}), seq.scan(**{**SCAN, "L": 1})
    refused(ucd.E_NULLPTR, seq.ucd_causal_conv_step, conv, P, P, P, None, P, stream=0)
    refused(ucd.E_NULLPTR, seq.ucd_scan_step, scan, P, P, P, P, P, None, P, stream=0)


def test_workspaces():
    # a prompt's states and Backward's partial sums
    scan = seq.scan(B=1, L=16384, D=64, N=16)
    saved, need = seq.ucd_scan_saved_size(scan), seq.ucd_scan_workspace_size(scan, seq.BWD)
    assert saved > 0 and need > 0

    def bwd(saved_bytes=saved, ws=P, ws_bytes=need, **kw):
        seq.ucd_scan_bwd(scan, P, P, P, P, P, P, P, P, P, P, P, P, saved_bytes=saved_bytes, ws=ws, ws_bytes=ws_bytes, stream=0, **kw)
    refused(ucd.E_WS_TOO_SMALL, bwd, saved_bytes=saved - 1)
    refused(ucd.E_WS_TOO_SMALL, bwd, ws_bytes=need - 1)
    refused(ucd.E_NULLPTR, bwd, ws=None)
    refused(ucd.E_INVALID, bwd, ws=P + 4)
    refused(ucd.E_NULLPTR, bwd, z=P)              # z without dz
    refused(ucd.E_NULLPTR, bwd, skip=P)
    refused(ucd.E_NULLPTR, bwd, dt_bias=P)
    refused(ucd.E_INVALID, bwd, beta=0.5)
    refused(ucd.E_WS_TOO_SMALL, scan_fwd, scan, saved=P, saved_bytes=saved - 1)


def test_no_token_at_all():
    """Tensors of no elements have no address: nothing is read, nothing is refused."""
    conv_fwd(seq.causal_conv(**{**CONV, "B": 0}), x=None, y=None)
    scan_fwd(seq.scan(**{**SCAN, "B": 0}), u=None, y=None)
