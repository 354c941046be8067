"""Linear attention and gated projection without a GPU: what the entry points refuse (on the host, before anything is launched; the
addresses below are never read), the sizes that they ask for, and the oracle's gradients against differences."""
import ctypes
import os
import re

import numpy as np
import pytest

from oracle import seq as os_
from paper_1804_04806_amd import seq, ucd

P = 1 << 20   # an aligned address
ATTENTION = dict(B=2, L=3, H=4, Hk=2, Dk=8, Dv=16)
GATED = dict(M=100, D=16, F=24)
BIG = dict(saved_bytes=1 << 40, ws=P, ws_bytes=1 << 40)


def test_every_declared_symbol_is_exported():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(root, "include", "ucd_mix.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(ucd_[a-z_0-9]+)\s*\(", text)))
    assert names == sorted(seq.MIX_EXPORTS)
    lib = ctypes.CDLL(ucd.LIB_PATH)
    assert all(hasattr(lib, n) and hasattr(seq, n) for n in names)


def refused(status, call, *args, **kw):
    with pytest.raises(ucd.UcdError) as e:
        call(*args, **kw)
    assert e.value.status == status, (e.value.status, status)


def attention_fwd(desc, q=P, k=P, v=P, y=P, **kw):
    seq.ucd_linear_attention_fwd(desc, q, k, v, y, **{**BIG, **kw}, stream=0)


def attention_bwd(desc, q=P, k=P, v=P, dy=P, saved=P, dq=P, dk=P, dv=P, **kw):
    seq.ucd_linear_attention_bwd(desc, q, k, v, dy, saved, dq, dk, dv, **{**BIG, **kw}, stream=0)


def gated_fwd(desc, x=P, wg=P, wu=P, y=P, **kw):
    seq.ucd_gated_projection_fwd(desc, x, wg, wu, y, **{**BIG, **kw}, stream=0)


def gated_bwd(desc, x=P, wg=P, wu=P, dy=P, saved=P, dx=P, dwg=P, dwu=P, **kw):
    seq.ucd_gated_projection_bwd(desc, x, wg, wu, dy, saved, dx, dwg, dwu, **{**BIG, **kw}, stream=0)


@pytest.mark.parametrize("bad", [dict(B=-1), dict(L=-1), dict(H=0), dict(Hk=0), dict(Hk=3), dict(Hk=8), dict(Dk=0), dict(Dk=129), dict(Dv=0),
                                 dict(Dv=129), dict(dtype=2), dict(n_slots=-1), dict(scale=float("nan")), dict(scale=float("inf")),
                                 dict(q_stride=(0, 15)), dict(k_stride=(47, 16)), dict(v_stride=(0, 63)), dict(g_stride=(0, 3)),
                                 dict(y_stride=(-1, 64)), dict(L=(1 << 30) + 1), dict(B=1 << 20, L=1 << 20, H=1 << 10, Hk=1)], ids=str)
def test_attention_descriptors(bad):
    desc = seq.linear_attention(**{**ATTENTION, **bad})
    assert seq.ucd_linear_attention_workspace_size(desc, seq.FWD) == ucd.WS_NA and seq.ucd_linear_attention_saved_size(desc) == ucd.WS_NA
    refused(ucd.E_INVALID, attention_fwd, desc)
    refused(ucd.E_INVALID, attention_bwd, desc)


@pytest.mark.parametrize("bad", [dict(M=-1), dict(D=0), dict(F=0), dict(D=(1 << 20) + 1), dict(F=(1 << 20) + 1), dict(act=3), dict(act=-1), dict(dtype=2),
                                 dict(x_stride=15), dict(y_stride=23), dict(x_stride=(1 << 21) + 1), dict(x_stride=-16)], ids=str)
def test_gated_descriptors(bad):
    desc = seq.gated_projection(**{**GATED, **bad})
    assert seq.ucd_gated_projection_workspace_size(desc, seq.FWD) == ucd.WS_NA and seq.ucd_gated_projection_saved_size(desc) == ucd.WS_NA
    refused(ucd.E_INVALID, gated_fwd, desc)
    refused(ucd.E_INVALID, gated_bwd, desc)


def test_directions():
    for n in (-1, 2):
        assert seq.ucd_linear_attention_workspace_size(seq.linear_attention(**ATTENTION), n) == ucd.WS_NA
        assert seq.ucd_gated_projection_workspace_size(seq.gated_projection(**GATED), n) == ucd.WS_NA


def test_attention_pointers():
    desc, half = seq.linear_attention(**ATTENTION), seq.linear_attention(**ATTENTION, dtype=1)
    for name in ("q", "k", "v", "y"):
        refused(ucd.E_NULLPTR, attention_fwd, desc, **{name: None})
        refused(ucd.E_INVALID, attention_fwd, desc, **{name: P + 2})
        refused(ucd.E_INVALID, attention_fwd, half, **{name: P + 1})
    for name in ("g", "decay", "lengths", "state_in", "state_out"):
        refused(ucd.E_INVALID, attention_fwd, desc, **{name: P + 2})
    for name in ("q", "k", "v", "dy", "dq", "dk", "dv", "saved"):
        refused(ucd.E_NULLPTR, attention_bwd, desc, **{name: None})
        refused(ucd.E_INVALID, attention_bwd, desc, **{name: P + 2})
    for name in ("dstate_out", "dstate_in"):
        refused(ucd.E_INVALID, attention_bwd, desc, **{name: P + 2})
    refused(ucd.E_INVALID, attention_bwd, desc, dg=P)          # a gradient of what is not there
    refused(ucd.E_INVALID, attention_bwd, desc, g=P, dg=P + 2)


def test_attention_slots():
    refused(ucd.E_INVALID, attention_fwd, seq.linear_attention(**ATTENTION), slots=P)
    refused(ucd.E_INVALID, attention_fwd, seq.linear_attention(**ATTENTION, n_slots=5))
    refused(ucd.E_INVALID, attention_bwd, seq.linear_attention(**ATTENTION, n_slots=5))
    step = seq.ucd_linear_attention_step
    refused(ucd.E_INVALID, step, seq.linear_attention(**ATTENTION), P, P, P, P, P, stream=0)
    one = seq.linear_attention(**{**ATTENTION, "L": 1})
    refused(ucd.E_NULLPTR, step, one, P, P, P, None, P, stream=0)
    refused(ucd.E_NULLPTR, step, one, P, None, P, P, P, stream=0)
    refused(ucd.E_INVALID, step, one, P, P, P, P, P, slots=P, stream=0)
    refused(ucd.E_INVALID, step, one, P, P, P, P + 2, P, stream=0)


def test_attention_buffers():
    desc = seq.linear_attention(B=1, L=16384, H=2, Dk=64, Dv=64)        # in segments
    for d, call in ((seq.FWD, attention_fwd), (seq.BWD, attention_bwd)):
        need, saved = seq.ucd_linear_attention_workspace_size(desc, d), seq.ucd_linear_attention_saved_size(desc)
        assert need > 0 and saved > 0
        refused(ucd.E_WS_TOO_SMALL, call, desc, ws_bytes=need - 1)
        refused(ucd.E_NULLPTR, call, desc, ws=None)
        refused(ucd.E_INVALID, call, desc, ws=P + 4)
        refused(ucd.E_WS_TOO_SMALL, call, desc, saved=P, saved_bytes=saved - 1)
        refused(ucd.E_INVALID, call, desc, saved=P + 4)


def test_gated_pointers():
    desc, half = seq.gated_projection(**GATED), seq.gated_projection(**GATED, dtype=1)
    for name in ("x", "wg", "wu", "y"):
        refused(ucd.E_NULLPTR, gated_fwd, desc, **{name: None})
        refused(ucd.E_INVALID, gated_fwd, desc, **{name: P + 2})
        refused(ucd.E_INVALID, gated_fwd, half, **{name: P + 1})
    for name in ("x", "wg", "wu", "dy", "saved", "dx", "dwg", "dwu"):
        refused(ucd.E_NULLPTR, gated_bwd, desc, **{name: None})
        refused(ucd.E_INVALID, gated_bwd, desc, **{name: P + 2})
    refused(ucd.E_INVALID, gated_bwd, desc, beta=0.5)
    for d, call in ((seq.FWD, gated_fwd), (seq.BWD, gated_bwd)):
        need, saved = seq.ucd_gated_projection_workspace_size(desc, d), seq.ucd_gated_projection_saved_size(desc)
        assert need > 0 and saved >= 100 * 2 * 24 * 4
        refused(ucd.E_WS_TOO_SMALL, call, desc, ws_bytes=need - 1)
        refused(ucd.E_NULLPTR, call, desc, ws=None)
        refused(ucd.E_WS_TOO_SMALL, call, desc, saved=P, saved_bytes=saved - 1)


def test_too_many_workgroups():
    refused(ucd.E_UNSUPPORTED, attention_fwd, seq.linear_attention(B=1 << 22, L=1, H=4, Dk=8, Dv=8))
    refused(ucd.E_UNSUPPORTED, attention_bwd, seq.linear_attention(B=1 << 22, L=1, H=4, Dk=8, Dv=8))
    refused(ucd.E_UNSUPPORTED, gated_fwd, seq.gated_projection(M=1 << 30, D=16, F=128))


def test_no_token_at_all():
    attention_fwd(seq.linear_attention(**{**ATTENTION, "B": 0}), q=None, k=None, v=None, y=None)
    attention_bwd(seq.linear_attention(**{**ATTENTION, "B": 0}), q=None, k=None, v=None, dy=None, dq=None, dk=None, dv=None)
    gated_fwd(seq.gated_projection(**{**GATED, "M": 0}), x=None, y=None)


def test_oracle_attention_gradients():
    rng = np.random.default_rng(0)
    B, L, H, Hk, Dk, Dv = 2, 6, 4, 2, 3, 5
    n, decay, dstate = np.array([6, 4]), -rng.uniform(0.1, 0.5, H), rng.standard_normal((B, H, Dk, Dv))
    dy = rng.standard_normal((B, L, H, Dv))
    given = {"q": rng.standard_normal((B, L, Hk, Dk)), "k": rng.standard_normal((B, L, Hk, Dk)), "v": rng.standard_normal((B, L, H, Dv)),
             "g": -rng.uniform(0.1, 1, (B, L, H)), "state": rng.standard_normal((B, H, Dk, Dv))}

    def loss(q, k, v, g, state):
        y, s = os_.attention_fwd(q, k, v, 0.3, g, decay, n, state)
        return (y * dy).sum() + (s * dstate).sum()
    grads = os_.attention_bwd(given["q"], given["k"], given["v"], 0.3, dy, given["g"], decay, n, given["state"], dstate)
    for name, value in given.items():
        d = rng.standard_normal(value.shape)
        up, down = ({**given, name: value + s * 1e-5 * d} for s in (1, -1))
        # differences of 1e-5: second-order terms 1e-10, rounding 1e-16 * 100 / 1e-5
        assert abs((loss(**up) - loss(**down)) / 2e-5 - (grads[name] * d).sum()) < 1e-7


@pytest.mark.parametrize("act", [0, 1, 2])
def test_oracle_gated_gradients(act):
    rng = np.random.default_rng(1)
    given, dy = [rng.standard_normal(s) for s in ((4, 3), (5, 3), (5, 3))], rng.standard_normal((4, 5))
    grads = os_.gated_bwd(*given, act, dy)
    for i in range(3):
        d = rng.standard_normal(given[i].shape)
        up, down = ([a + s * 1e-5 * d if j == i else a for j, a in enumerate(given)] for s in (1, -1))
        difference = ((os_.gated_fwd(*up, act) - os_.gated_fwd(*down, act)) * dy).sum() / 2e-5
        assert abs(difference - (grads[i] * d).sum()) < 1e-7
