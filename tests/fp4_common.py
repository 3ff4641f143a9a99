"""Pages of 4-bit numbers for the tests: the format in 64 bits, and ragged batches over such pages."""
import torch

from paged_common import Batch

GRID = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)
BORDERS = (GRID[1:] + GRID[:-1]) / 2
LIMITS = 7 * 2.0 ** torch.arange(-125, 125, dtype=torch.float64)      # the largest magnitudes that scales 2^-125 .. 2^124 are enough for


def quantised64(x):
    """(codes, scales) of rows of multiples of 32 numbers, by trying every scale."""
    b = x.double().unflatten(-1, (-1, 32))
    most = b.abs().amax(-1, keepdim=True)
    e = (most > LIMITS).sum(-1, keepdim=True).double() - 125
    y = b / 2.0 ** e
    at = torch.searchsorted(BORDERS, y.abs().contiguous())             # of two equally near ones the lower
    at = torch.where((at < 7) & (y.abs() == BORDERS[at.clamp(max=6)]), at + at % 2, at)
    code = at + 8 * torch.signbit(y)
    bad = ~torch.isfinite(b).all(-1, keepdim=True)
    code, scale = torch.where(bad, 0, code).flatten(-2), torch.where(bad, 255, e + 127)[..., 0]
    return (code[..., ::2] + 16 * code[..., 1::2]).to(torch.uint8), scale.to(torch.uint8)


def values64(codes, scales):
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).long()
    v = GRID[c & 7] * torch.where(c >= 8, -1.0, 1.0)
    s = torch.where(scales >= 253, torch.nan, 2.0 ** (scales.double() - 127))
    return (v.unflatten(-1, (-1, 32)) * s[..., None]).flatten(-2)


NAMES = ("k_codes", "v_codes", "k_scales", "v_scales")


class Batch4(Batch):
    """k_cache, v_cache: the values of the codes and scales, in 64 bits (on the host)."""

    def __init__(self, *args, layout="phkd", scale_layout=None, **kw):
        super().__init__(*args, layout=layout, **kw)
        for c in "kv":
            codes, scales = quantised64(getattr(self, c + "_cache"))
            for name, t, order in (("_codes", codes, layout), ("_scales", scales, scale_layout or layout)):
                dims = ["pkhd".index(x) for x in order]
                setattr(self, c + name, t.permute(dims).contiguous().permute([dims.index(i) for i in range(4)]))
        self.renew()

    def renew(self):
        self.k_cache, self.v_cache = values64(self.k_codes, self.k_scales), values64(self.v_codes, self.v_scales)

    def cuda(self):
        b = super().cuda()
        b.__class__ = Batch4
        b.k_cache = b.v_cache = None
        return b

    def pool(self):
        return self.k_codes, self.k_scales, self.v_codes, self.v_scales
