"""So many channels that a launch with a thread for each piece of work would have 2^32 threads and more, which is no valid grid."""
import pytest

from paper_1804_04806_amd import seq

pytestmark = pytest.mark.gpu


def fresh(*shape, dtype=None):
    """Memory that no kernel has written: NaN."""
    import torch
    return torch.full(shape, float("nan"), device="cuda:0", dtype=dtype or torch.float32)


def room(nbytes):
    import torch
    return torch.empty(max(16, nbytes), dtype=torch.uint8, device="cuda:0")


def near(got, want):
    import torch
    assert bool(torch.isfinite(got).all())
    assert float((got - want).abs().max()) <= 1e-5 * float(want.abs().max())


def test_conv_gradients_of_many_channels():
    """One token of 2^25 channels with eight taps: 9 * 2^25 sums, 64 to a workgroup of 1024."""
    import torch
    D, K = 1 << 25, 8
    desc = seq.causal_conv(1, 1, D, K, dtype=1)
    x, dy = (torch.randn(1, 1, D, device="cuda:0").bfloat16() for _ in range(2))
    w = torch.ones(D, K, device="cuda:0", dtype=torch.bfloat16)
    dx, dw, dbias = fresh(1, 1, D, dtype=torch.bfloat16), fresh(D, K), fresh(D)
    seq.ucd_causal_conv_bwd(desc, x, w, None, dy, dx, dw, dbias, ws=room(seq.ucd_causal_conv_workspace_size(desc)))
    assert torch.equal(dx, dy) and torch.equal(dbias, dy.float().view(-1))
    assert torch.equal(dw[:, K - 1], (x.float() * dy.float()).view(-1)) and not dw[:, :K - 1].any()


def test_scan_gradients_of_many_channels():
    """One token of 2^22 channels with 64 states: 66 * 2^22 sums."""
    import torch
    D, N = 1 << 22, 64
    desc = seq.scan(1, 1, D, N, softplus=False)
    u, dt, dy = (torch.randn(1, 1, D, device="cuda:0") for _ in range(3))
    Bm, Cm = torch.randn(1, 1, N, device="cuda:0"), torch.randn(1, 1, N, device="cuda:0")
    A, skip, bias = -torch.ones(D, N, device="cuda:0"), torch.ones(D, device="cuda:0"), torch.zeros(D, device="cuda:0")
    y, du, ddt, dA = fresh(1, 1, D), fresh(1, 1, D), fresh(1, 1, D), fresh(D, N)
    dB, dC, dskip, dbias = fresh(1, 1, N), fresh(1, 1, N), fresh(D), fresh(D)
    saved, ws = room(seq.ucd_scan_saved_size(desc)), room(max(seq.ucd_scan_workspace_size(desc, k) for k in (seq.FWD, seq.BWD)))
    seq.ucd_scan_fwd(desc, u, dt, A, Bm, Cm, y, skip=skip, dt_bias=bias, saved=saved, ws=ws)
    seq.ucd_scan_bwd(desc, u, dt, A, Bm, Cm, dy, saved, du, ddt, dA, dB, dC, skip=skip, dskip=dskip, dt_bias=bias, ddt_bias=dbias, ws=ws)
    both = (Bm.double() * Cm.double()).sum().float()
    near(y, u * dt * both + u)
    near(du, dy * dt * both + dy)
    near(dbias, (dy * u * both).view(-1))
    assert torch.equal(dskip, (dy * u).view(-1)) and torch.equal(ddt.view(-1), dbias) and not dA.any()


def test_norm_of_many_strips():
    """65 positions of 2^25 channels in as many groups: 2^19 strips of 64 groups, each with 1024 threads, in rounds of eight samples."""
    import torch
    S, C = 65, 1 << 25
    x = torch.empty(1, S, C, device="cuda:0", dtype=torch.bfloat16)
    x.normal_()
    gamma, beta = torch.randn(C, device="cuda:0"), torch.randn(C, device="cuda:0")
    desc = seq.group_norm(1, S, C, C, dtype=1)
    y, stats = fresh(1, S, C, dtype=torch.bfloat16), fresh(2, 1, C)
    seq.ucd_group_norm_fwd(desc, x, gamma, beta, y, stats, ws=room(seq.ucd_group_norm_workspace_size(desc, seq.FWD)))
    for part in (slice(0, 4096), slice(C // 2 - 2048, C // 2 + 2048), slice(C - 4096, C)):
        v = x[0, :, part].double()
        var, mean = torch.var_mean(v, 0, correction=0)
        want = (v - mean) * (var + 1e-5).rsqrt() * gamma[part] + beta[part]
        off = (y[0, :, part].double() - want).abs()
        assert bool((off <= 2.0 ** -8 * want.abs() + 1e-5).all())
        near(stats[0, 0, part], mean.float())
    # every strip was written: sums of a column of positions are NaN where one was not
    assert bool(torch.isfinite(y[0].float().sum(0)).all()) and bool(torch.isfinite(stats).all())
    dy = y.normal_()
    dx, dgamma, dbeta = fresh(1, S, C, dtype=torch.bfloat16), fresh(C), fresh(C)
    seq.ucd_group_norm_bwd(desc, x, gamma, beta, stats, dy, dx, dgamma, dbeta, ws=room(seq.ucd_group_norm_workspace_size(desc, seq.BWD)))
    for part in (slice(0, 2048), slice(C - 2048, C)):
        g, v = dy[0, :, part].double(), x[0, :, part].double()
        var, mean = torch.var_mean(v, 0, correction=0)
        rstd = (var + 1e-5).rsqrt()
        xhat = (v - mean) * rstd
        near(dbeta[part], g.sum(0).float())
        near(dgamma[part], (g * xhat).sum(0).float())
        g = g * gamma[part]
        want = rstd * (g - g.mean(0) - xhat * (g * xhat).mean(0))
        assert bool(((dx[0, :, part].double() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-5 * want.abs().max()).all())
    assert bool(torch.isfinite(dx[0].float().sum(0)).all()) and bool(torch.isfinite(dgamma + dbeta).all())
