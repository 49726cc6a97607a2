"""Arrays of rows on the GPU whose every other element is a mark or NaN."""
import math

import torch

MARK = 77.0


class Rows:
    """Rows [total, width] in a larger array: `pad` elements between rows, `shift` before the first; everything else holds `fill`."""

    def __init__(self, values, pad=0, shift=0, fill=math.nan):
        self.total, self.width = values.shape
        self.ld, self.shift, self.dtype, self.fill = self.width + pad, shift, values.dtype, fill
        self.values = values
        flat = torch.full((shift + max(self.total, 1) * self.ld + 8,), fill, dtype=values.dtype)
        self.view(flat)[:] = values
        self.flat = flat.cuda()

    @classmethod
    def empty(cls, total, width, dtype, pad=0, shift=0):
        return cls(torch.full((total, width), MARK, dtype=dtype), pad, shift, MARK)

    def view(self, flat):
        return flat[self.shift:self.shift + self.total * self.ld].view(self.total, self.ld)[:, :self.width]

    @property
    def arg(self):
        return self.flat[self.shift:]

    def result(self, what=""):
        """The rows, after a look at everything around them."""
        got = self.flat.cpu()
        around = torch.ones_like(got, dtype=torch.bool)
        self.view(around)[:] = False
        rest = got[around].float()
        assert (torch.isnan(rest) if math.isnan(self.fill) else rest == self.fill).all(), f"{what}: written beyond the rows"
        return self.view(got)


def activations(g, total, width, dtype, offset=0.0):
    """Rows of sizes between 2^-4 and 2^4, a few columns larger than the others."""
    x = torch.randn(total, width, generator=g) * torch.exp2(torch.rand(total, 1, generator=g) * 8 - 4) + offset
    x[:, torch.randint(0, width, (1 + width // 100,), generator=g)] *= 8
    return x.to(dtype)


def some(g, total, share=0.3):
    """A mask that leaves out about this share of the rows."""
    return (torch.rand(total, generator=g) >= share).to(torch.uint8)
