"""Shared helpers of the sequence operators' tests: inputs of the values that the operators meet, tensors with strides of
their own inside a poisoned buffer, comparison with the oracle."""
import numpy as np

from paper_1804_04806_amd import synth

# fp32: sums of up to some thousand terms, each rounding 6e-8 of its result, and decays whose errors add up over the tokens
# that a state remembers: a few 1e-7 in the 2-norm, 1e-5 allowed; one element within 1e-4 of the largest of itself and
# the tensor's rms.  bf16 results are rounded once more, to 8 significant
# bits: 2^-8 of an element at most.
F32_L2, F32_ELEMENT, BF16 = 1e-5, 1e-4, 2.0 ** -8


def values(rng, *shape, std=1.0, dtype=0):
    """Normal values that the type holds."""
    v = (rng.standard_normal(shape) * std).astype(np.float32)
    return synth.from_bf16_bits(synth.to_bf16_bits(v)) if dtype == 1 else v


def kind_of(dtype):
    import torch
    return torch.bfloat16 if dtype == 1 else torch.float32


class Placed:
    """A (outer, inner, ...) array on the device with strides of its own; what lies between its rows and around it is poison
    that must stay (an output) and is not taken for a value (an input)."""
    POISON = -7.8125e18
    EDGE = 64

    def __init__(self, shape, dtype, strides=None, data=None, shift=0):
        import torch
        self.shape, width = tuple(shape), int(np.prod(shape[2:], dtype=np.int64))
        outer, inner = strides or (shape[1] * width, width)
        size = max(0, (shape[0] - 1) * outer + (shape[1] - 1) * inner + width) if min(shape[:2]) > 0 else 0
        self.buf = torch.full((2 * self.EDGE + shift + size,), self.POISON, dtype=kind_of(dtype), device="cuda:0")
        self.strides = (outer, inner)
        self.t = self._view(self.buf[self.EDGE + shift:], width)
        if data is not None:
            self.t.copy_(torch.from_numpy(np.ascontiguousarray(data).reshape(self.t.shape)))
            if strides is not None:
                self.buf[self._outside()] = float("nan")

    def _view(self, flat, width):
        return flat.as_strided((self.shape[0], self.shape[1], width), self.strides + (1,))

    def _outside(self):
        import torch
        mark = torch.ones_like(self.buf, dtype=torch.bool)
        off = self.t.storage_offset()
        mark[off:].as_strided(self.t.shape, self.t.stride()).fill_(False)
        return mark

    def ptr(self):
        return self.t.data_ptr()

    def get(self):
        """The values, after a check that nothing else was written."""
        assert bool((self.buf[self._outside()] == self.POISON).all()), "written outside the tensor"
        return self.t.float().cpu().numpy().reshape(self.shape)


def workspace(nbytes):
    """A buffer of exactly nbytes, poisoned, and a check that what follows it stays."""
    import torch
    buf = torch.full((nbytes // 4 + 64,), float("nan"), device="cuda:0")

    def check():
        assert bool(torch.isnan(buf[(nbytes + 3) // 4:]).all()), "workspace written behind its end"
    return buf.data_ptr(), nbytes, check


def device(a):
    import torch
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to("cuda:0")


def check(got, ref, dtype, what="", l2=F32_L2, element=F32_ELEMENT):
    got, ref = np.asarray(got, np.float64), np.asarray(ref, np.float64)
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    if not ref.size:
        return
    assert np.isfinite(got).all(), what
    norm, rms = np.linalg.norm(ref), np.sqrt(np.mean(ref ** 2))
    off = np.linalg.norm(got - ref)
    assert off <= (l2 + (BF16 if dtype == 1 else 0)) * norm, (what, off / max(norm, 1e-300))
    allowed = element * np.maximum(np.abs(ref), rms) + (BF16 * np.abs(ref) if dtype == 1 else 0)
    assert (np.abs(got - ref) <= allowed).all(), (what, float((np.abs(got - ref) - allowed).max()), rms)


def lengths_for(rng, B, L):
    """Full, empty and single-token sequences among others."""
    n = ([L, 0, min(1, L)] + [int(rng.integers(0, L + 1)) for _ in range(B)])[:B]
    return np.array(n, dtype=np.int32)

