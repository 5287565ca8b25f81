"""Matrices inside wider buffers, for tests of strides, alignment and of what a call leaves alone."""
import torch

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
MARK = 77.0


def half(dtype):
    """Half a step of the storage type, relative to the value."""
    return torch.finfo(DT[dtype]).eps / 2


class Matrix:
    """A [rows, H] matrix inside a wider buffer whose rest is filled with a mark."""

    def __init__(self, rows, H, dtype, pad=0, front=0, data=None):
        self.buf = torch.full((front + rows * (H + pad) + 3,), MARK, dtype=DT[dtype], device="cuda")
        self.view = self.buf[front:front + rows * (H + pad)].view(rows, H + pad)[:, :H]
        if data is None:
            self.view.fill_(float("nan"))   # outputs must be overwritten
        else:
            self.view.copy_(torch.from_numpy(data))

    def assert_around_untouched(self):
        inside = self.view.clone()
        self.view.fill_(MARK)
        assert (self.buf == MARK).all(), "written outside the rows"
        self.view.copy_(inside)


def rounded(a, dtype):
    return torch.from_numpy(a).to(DT[dtype]).double().numpy()
