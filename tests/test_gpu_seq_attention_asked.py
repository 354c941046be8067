"""Linear attention: what a caller asks for beside them does not change the bits of the outputs."""
import pytest

from paper_1804_04806_amd import seq

pytestmark = pytest.mark.gpu

# B, L, H, Hk, Dk, Dv: segments of one chunk, segments of several, walks over whole sequences
SHAPES = [(2, 300, 8, 4, 64, 128), (3, 1500, 16, 16, 40, 33), (33, 150, 16, 4, 24, 16)]


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_bits_of_what_is_asked_for(shape, dtype):
    """y with and without the last state and with and without what Backward reads; dv, dq and dk with and without the gradient of the first state."""
    import torch
    B, L, H, Hk, Dk, Dv = shape
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(sum(shape))
    kind = (torch.float32, torch.bfloat16)[dtype]

    def new(*s):
        return torch.randn(s, device="cuda:0", generator=gen).to(kind)
    q, k, v, dy, g = new(B, L, Hk, Dk), new(B, L, Hk, Dk), new(B, L, H, Dv), new(B, L, H, Dv), -0.1 * new(B, L, H).abs()
    first = torch.randn(B, H, Dk, Dv, device="cuda:0", generator=gen)
    desc = seq.linear_attention(B, L, H, Dk, Dv, Hk, 0.1, dtype)
    ws = torch.empty(max(16, *(seq.ucd_linear_attention_workspace_size(desc, d) for d in (seq.FWD, seq.BWD))), dtype=torch.uint8, device="cuda:0")
    saved = torch.empty(seq.ucd_linear_attention_saved_size(desc), dtype=torch.uint8, device="cuda:0")
    got = []
    for last in (None, torch.empty_like(first)):
        for kept in (None, saved):
            y = torch.empty_like(v)
            seq.ucd_linear_attention_fwd(desc, q, k, v, y, g=g, state_in=first, state_out=last, saved=kept, ws=ws)
            got.append(y)
    assert all(torch.equal(got[0], t) for t in got[1:])
    got = []
    for dfirst in (None, torch.empty_like(first)):
        grads = [torch.empty_like(t) for t in (q, k, v, g)]
        seq.ucd_linear_attention_bwd(desc, q, k, v, dy, saved, *grads[:3], g=g, dg=grads[3], dstate_in=dfirst, ws=ws)
        got.append(grads)
    assert all(torch.equal(a, b) for a, b in zip(*got))
