"""Tensors for the operators on a caller's device memory: rows of any distance
inside a larger buffer whose other elements are known, so that a test sees what
a call wrote beside its output."""
import torch

MARK = 7.25  # a value that bf16 holds


class Rows:
    """[rows, cols] at element `lead` of a buffer, rows cols + pad apart."""

    def __init__(self, rows, cols, dtype, pad=0, lead=0, data=None, tail=64):
        self.rows, self.cols, self.ld, self.lead = rows, cols, cols + pad, lead
        fill = MARK if dtype.is_floating_point else 77
        self.buf = torch.full((lead + rows * self.ld + tail,), fill, dtype=dtype, device="cuda")
        self.view = self.buf[lead:lead + rows * self.ld].view(rows, self.ld)[:, :cols]
        if data is not None:
            self.view.copy_(data)

    @property
    def ptr(self):
        return self.buf.data_ptr() + self.lead * self.buf.element_size()

    def numpy(self):
        v = self.view.detach().cpu()
        return (v.float() if v.dtype == torch.bfloat16 else v).numpy()

    def untouched(self):
        """Whether everything beside the rows still holds the mark."""
        b = self.buf.clone()
        b[self.lead:self.lead + self.rows * self.ld].view(self.rows, self.ld)[:, :self.cols] = self.mark()
        return bool((b == self.mark()).all())

    def mark(self):
        return MARK if self.buf.dtype.is_floating_point else 77


def dtype_of(prec):
    return torch.bfloat16 if prec else torch.float32


def stream():
    return torch.cuda.current_stream().cuda_stream
