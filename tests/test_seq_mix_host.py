"""What the attention and feed-forward blocks hand to linear attention and the gated projection, without a GPU."""
import pytest
import torch

from paper_1804_04806_amd import sequence_block as sb
from paper_1804_04806_amd import ucd

B, L, H, HK, DK, DV, F = 2, 3, 4, 2, 8, 6, 10


def arguments(kind=torch.float32):
    """(function, arguments): tensors of one type, the heads' decays in fp32."""
    q, v = torch.randn(B, L, HK, DK, dtype=kind), torch.randn(B, L, H, DV, dtype=kind)
    x, w = torch.randn(B, L, DK, dtype=kind), torch.randn(DK, 2 * F, dtype=kind)
    return [(sb.LinearAttention, [q, torch.randn_like(q), v, -torch.rand(B, L, H).to(kind), -torch.rand(2 * H)[::2], 0.5]),
            (sb.GatedProjection, [x, w.t()[:F], w.t()[F:]])]


@pytest.fixture
def host(monkeypatch):
    """Calls are written down instead of made, and the host's memory is taken for the device's."""
    calls = []
    monkeypatch.setattr(sb, "_DEVICE", "cpu")
    for name in sb.seq.EXPORTS + sb.seq.MIX_EXPORTS:
        if not name.endswith("_size"):
            monkeypatch.setattr(sb.seq, name, lambda *a, _name=name, **k: calls.append((_name, a, k)))
    return calls


def test_weights_reach_the_operators_dense(host):
    for (function, args), places in zip(arguments(), ((4,), (1, 2))):
        function.apply(*args)
        got = [t for t in [*host[-1][1], *host[-1][2].values()] if isinstance(t, torch.Tensor)]
        for i in places:
            assert any(t.is_contiguous() and t.shape == args[i].shape and torch.equal(t, args[i]) for t in got), i


def views(shape):
    b, l, c = shape
    dense = torch.randn(shape)
    return {"dense": dense, "half": torch.randn(b, l, 2 * c)[..., c:], "tokens first": torch.randn(l, b, c).transpose(0, 1),
            "fewer tokens": torch.randn(b, 2 * l, c)[:, 1:l + 1], "every other": torch.randn(b, 2 * l, c)[:, ::2],
            "over sequences": torch.randn(1, l, c).expand(shape), "over tokens": torch.randn(b, 1, c).expand(shape),
            "channels first": torch.randn(b, c, l).transpose(1, 2), "one token": torch.randn(b, l, c)[:, 1:2], "one sequence": dense[1:]}


@pytest.mark.parametrize("name", views((B, L, DK)))
def test_rows_of_a_projection_are_where_the_descriptor_says(name, host):
    x = views((B, L, DK))[name]
    sb.GatedProjection.apply(x, *arguments()[1][1][1:])
    (desc, given, *_), m = host[-1][1], x.shape[0] * x.shape[1]
    assert (desc.M, desc.D, desc.F) == (m, DK, F)
    stride = desc.x_m or DK
    assert stride >= DK and torch.equal(given.as_strided((m, DK), (stride, 1)), x.reshape(m, DK))


@pytest.mark.parametrize("name", views((B, L, HK * DK)))
def test_heads_are_where_the_descriptor_says(name, host):
    q = views((B, L, HK * DK))[name].unflatten(-1, (HK, DK))
    b, l = q.shape[:2]
    sb.LinearAttention.apply(q, torch.randn(b, l, HK, DK), torch.randn(b, l, H, DV))
    desc, given = host[-1][1][:2]
    inner = desc.q_l or HK * DK
    assert torch.equal(given.as_strided(q.shape, (desc.q_b or inner * l, inner, DK, 1)), q)


def test_foreign_types_and_shapes_are_refused():
    """A tensor of another type or shape is refused before anything is launched, and so is the host's memory."""
    for function, args in arguments():
        with pytest.raises(ValueError, match="device"):
            function.apply(*args)
        for kind in (torch.float64, torch.float16, torch.int32):
            with pytest.raises(TypeError):
                function.apply(args[0].to(kind), *args[1:])
        for i, t in enumerate(args):
            if not isinstance(t, torch.Tensor):
                continue
            with pytest.raises(TypeError):
                function.apply(*args[:i], t.bfloat16(), *args[i + 1:])
            for cut in (t[:-1], t[..., :-1], t[0], t[None]):
                with pytest.raises(ValueError):
                    function.apply(*args[:i], cut, *args[i + 1:])
    (attention, args), _ = arguments()
    with pytest.raises(ValueError, match="constants"):
        attention.apply(*args[:4], args[4].clone().requires_grad_())


def test_refused_descriptors_raise_the_librarys_error(monkeypatch):
    monkeypatch.setattr(sb, "_DEVICE", "cpu")
    monkeypatch.setattr(sb.seq, "_raw_stream", lambda: 0)
    wide, (attention, _), (gated, args) = torch.randn(B, L, 1, 129), *arguments()
    for function, bad in ((attention, [wide, wide, wide]), (attention, [torch.randn(B, L, 3, 8)] * 2 + [torch.randn(B, L, 4, 8)]),
                          (attention, [torch.randn(B, L, 1, 8)] * 3 + [None, None, float("nan")]), (gated, args + [3]),
                          (gated, [torch.randn(B, L, 0), torch.randn(F, 0), torch.randn(F, 0)])):
        with pytest.raises(ucd.UcdError) as e:
            function.apply(*bad)
        assert e.value.status == (ucd.E_INVALID if bad[0].numel() else ucd.E_NULLPTR)      # tensors of nothing are nowhere


def test_second_derivatives_are_refused(host):
    for function, args in arguments():
        args = [t.clone().requires_grad_(i != 4) if isinstance(t, torch.Tensor) else t for i, t in enumerate(args)]
        leaves = [t for t in args if isinstance(t, torch.Tensor) and t.requires_grad]
        y = function.apply(*args)
        first = torch.autograd.grad(y, leaves, torch.ones_like(y) * leaves[0].sum(), create_graph=True)
        penalty = sum(g.square().sum() for g in first) + leaves[0].pow(3).sum()
        with pytest.raises(RuntimeError, match="differentiat"):
            torch.autograd.grad(penalty, leaves, allow_unused=True)


def test_what_is_not_kept_has_no_gradient(host):
    _, (gated, args) = arguments()
    args = [t.clone().requires_grad_() for t in args]
    y = gated.apply(*args, sb.seq.ACT_GELU, False)
    assert host[-1][2]["saved"] is None and host[-1][1][0].act == sb.seq.ACT_GELU
    with pytest.raises(RuntimeError, match="kept"):
        y.sum().backward()
    block, x = sb.FeedForward(DK, F, device="cpu"), torch.randn(B, L, DK)
    block(x)
    assert host[-1][2]["saved"] is not None
    with torch.no_grad():
        block(x)
    assert host[-1][2]["saved"] is None


def test_states_and_places_are_checked(host):
    """Decoding: places and lengths are int32, states of the type and extents that the kernels move on in place."""
    block = sb.AttentionBlock(16, heads=4, size=8, key_heads=2, device="cpu")
    x, slots, lengths = torch.randn(2, 3, 16), torch.tensor([1, 0], dtype=torch.int32), torch.tensor([3, 1], dtype=torch.int32)
    pools = block.pools(5)
    assert block.extend(x, pools, slots, lengths).shape == x.shape and any(n == "ucd_linear_attention_fwd" for n, _, _ in host)
    del host[:]
    assert block.extend(x[:, :1], pools, slots).shape == (2, 1, 16) and any(n == "ucd_linear_attention_step" for n, _, _ in host)
    good = dict(x=x, pools=pools, slots=slots, lengths=lengths)
    for bad in (dict(slots=slots.long()), dict(lengths=lengths.long()), dict(pools=(pools[0].bfloat16(),))):
        with pytest.raises(TypeError):
            block.extend(**{**good, **bad})
    for bad in (dict(slots=slots[:1]), dict(lengths=lengths[:1]), dict(pools=(pools[0][:, 1:],)), dict(pools=(pools[0].transpose(2, 3),)),
                dict(pools=()), dict(x=x[0])):
        with pytest.raises(ValueError):
            block.extend(**{**good, **bad})
    with pytest.raises(ValueError):
        sb.AttentionBlock(16, heads=4, size=8, key_heads=3, device="cpu")
