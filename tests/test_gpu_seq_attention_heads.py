"""Linear attention of many heads to one of q and k: gradients that are sums over all of them, H * Dk beyond 2^23 elements."""
import pytest

from paper_1804_04806_amd import seq

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("L, H, Dk", [(2, 2 ** 17, 128), (70, 2 ** 17, 128), (66, 2 ** 17, 72), (5, 2 ** 17, 65)])
def test_gradients_of_many_heads(L, H, Dk, dtype):
    """One channel of v to a head, so that the formulas in 64 bits are products of tokens:  M[t, s] = sum over heads of D dy_t v_s,
    dq = scale M k, dk = scale M^T q, dg_u = scale sum of (M of a head) (q k^T) over the pairs that u lies between.

    bf16: the pairs' weights and the state, operands of dq and dk, are rounded, 2^-8 of a term at most in the 2-norm for each, and the gradients once
    more, 2^-8: three of them.  fp32: a few 1e-7, 1e-5 allowed, as the other tests of these operators.  dg: four parts of which three have a
    rounded operand, 6 * 2^-8, and its own rounding."""
    import torch
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(L + Dk)
    kind, scale = (torch.float32, torch.bfloat16)[dtype], 0.2

    def new(*shape, std=1.0):
        return (torch.randn(shape, device="cuda:0", generator=gen) * std).to(kind)
    q, k, v, dy = new(1, L, 1, Dk), new(1, L, 1, Dk, std=Dk ** -0.25), new(1, L, H, 1), new(1, L, H, 1)
    # part of every pair of rows is the same for all heads, so that sums over them do not vanish
    v, dy = (v.float() + 0.5).to(kind), (dy.float() + 0.5).to(kind)
    g = (-0.2 * torch.rand((1, L, H), device="cuda:0", generator=gen)).to(kind)
    desc = seq.linear_attention(1, L, H, Dk, 1, 1, scale, dtype)

    def room(nbytes):
        return torch.full((max(4, (nbytes + 3) // 4),), float("nan"), device="cuda:0")
    y, (dq, dk, dv, dg) = torch.empty_like(v), (torch.full_like(t, float("nan")) for t in (q, k, v, g))
    saved = room(seq.ucd_linear_attention_saved_size(desc))
    seq.ucd_linear_attention_fwd(desc, q, k, v, y, g=g, saved=saved, ws=room(seq.ucd_linear_attention_workspace_size(desc, seq.FWD)))
    seq.ucd_linear_attention_bwd(desc, q, k, v, dy, saved, dq, dk, dv, g=g, dg=dg, ws=room(seq.ucd_linear_attention_workspace_size(desc, seq.BWD)))
    want = {"y": torch.zeros(L, H, dtype=torch.float64, device="cuda:0"), "dv": torch.zeros(L, H, dtype=torch.float64, device="cuda:0"),
            "dg": torch.zeros(L, H, dtype=torch.float64, device="cuda:0"), "M": torch.zeros(L, L, dtype=torch.float64, device="cuda:0")}
    q2, k2 = q[0, :, 0].double(), k[0, :, 0].double()
    pairs = scale * (q2 @ k2.t())
    unseen = torch.arange(L, device="cuda:0")[:, None] < torch.arange(L, device="cuda:0")[None, :]
    for h in range(0, H, 1 << 13):      # some heads at a time
        part = slice(h, h + (1 << 13))
        vh, dyh, gh = (t[0, :, part].reshape(L, -1).double().t() for t in (v, dy, g))
        total = gh.cumsum(1)
        seen = (total[:, :, None] - total[:, None, :]).masked_fill(unseen, float("-inf")).exp()
        want["y"][:, part] = ((seen * pairs) * vh[:, None, :]).sum(2).t()
        want["dv"][:, part] = ((seen * pairs) * dyh[:, :, None]).sum(1).t()
        moved = seen * dyh[:, :, None] * vh[:, None, :]
        want["M"] += moved.sum(0)
        crossing = moved * pairs
        # what lies between s and t: rows from u on, columns before u
        both = crossing.flip(1).cumsum(1).flip(1).cumsum(2)
        want["dg"][1:, part] = torch.diagonal(both, offset=-1, dim1=1, dim2=2).t()
    want["dq"], want["dk"] = scale * (want["M"] @ k2), scale * (want["M"].t() @ q2)
    for name, got in (("y", y), ("dv", dv), ("dq", dq), ("dk", dk), ("dg", dg)):
        got, ref = got.double().reshape(want[name].shape), want[name]
        assert bool(torch.isfinite(got).all()), name
        allowed = 1e-5 if dtype == 0 else (7 if name == "dg" else 3) * 2.0 ** -8
        assert float((got - ref).norm()) <= allowed * float(ref.norm()), (name, float((got - ref).norm() / ref.norm()))
