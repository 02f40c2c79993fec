"""What the GPU tests of the operators inside a layer share: buffers with guards, and units of rounding."""
import numpy as np

FP32, FP16, BF16 = 0, 1, 2
U = 2.0 ** -24                                            # half a step of binary32
UNIT = {FP32: U, FP16: 2.0 ** -11, BF16: 2.0 ** -8}       # of a rounding to a type, relative
TINY = {FP32: 2.0 ** -149, FP16: 2.0 ** -25, BF16: 2.0 ** -134}
GUARD = 7.0


def lib():
    import torch
    import paper_2006_15704_amd as d
    return torch, d


def torch_type(dt):
    import torch
    return {FP32: torch.float32, FP16: torch.float16, BF16: torch.bfloat16}[dt]


class Rows:
    """values[T, D] on the GPU, `gap` elements between rows, `shift` in front, guards everywhere else.  `held` is
    what its type holds of the values, in 64 bits."""

    def __init__(self, values, dt, gap=0, shift=0):
        import torch
        values = np.asarray(values, dtype=np.float64)
        self.dt, self.shape, self.stride, self.shift = dt, values.shape, values.shape[1] + gap, shift
        T = values.shape[0]
        self.buf = torch.full((shift + T * self.stride + 16,), GUARD, dtype=torch_type(dt), device="cuda")
        self.view = self._view(self.buf)
        self.view.copy_(torch.from_numpy(values))
        self.held = self.view.double().cpu().numpy()

    def _view(self, buf):
        T, D = self.shape
        return buf[self.shift:self.shift + T * self.stride].view(T, self.stride)[:, :D]

    @property
    def ptr(self):
        return self.buf.data_ptr() + self.shift * self.buf.element_size()

    def get(self):
        return self.view.double().cpu().numpy()

    def check_guards(self):
        keep = self.buf.clone()
        self._view(keep).fill_(GUARD)
        assert (keep == GUARD).all(), "wrote outside its rows"


def vector(values, dt):
    import torch
    x = torch.from_numpy(np.asarray(values, dtype=np.float64)).to("cuda", torch_type(dt))
    return x, x.double().cpu().numpy()


def close(got, want, bound, what):
    """Every element within its own bound (first-order errors: one per cent for the products of errors)."""
    bad = ~(np.abs(got - want) <= 1.01 * bound)
    assert not bad.any(), (what, int(bad.sum()), np.argwhere(bad)[:3].tolist(), got[bad][:3], want[bad][:3], bound[bad][:3])
