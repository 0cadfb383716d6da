"""Products with weights of 4 bits whose arithmetic is exact: x are small whole numbers, scales powers of two, and no sum has more than 24 bits, so that
the one rounding of the result is all there is, and a lost or doubled element, a group's wrong scale or a neighbour's shows in every bit."""
import pytest
import torch

from paper_2411_01830_amd import binding as ft

pytestmark = pytest.mark.gpu

SLAB = 4096
BF16, FP16 = torch.bfloat16, torch.float16


def ops():
    from paper_2411_01830_amd import operators
    return operators


class Exact:
    """Random codes, zeros up to 15, scales of 1, 1/2, 1/4 and 1/8 with either sign, `by` times as large; whatever else the pool holds are the bytes of NaN."""

    def __init__(self, ni, no, group, dtype, zeros=True, seed=0, shift=0, by=1.0):
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        groups, row = -(-ni // group), (ni + 1) // 2
        n = 2 * SLAB * 4 + no * row + 3 * no * groups
        self.mem = torch.full((-(-n // SLAB) * SLAB,), 0xFF, dtype=torch.uint8, device="cuda")
        self.pool = ft.pool_create(self.mem.data_ptr(), self.mem.numel(), SLAB, 0)
        self.ni, self.no, self.group, self.dtype = ni, no, group, dtype
        codes = self.ints(256, no, row).to(torch.uint8)
        scales = (torch.exp2(-self.ints(4, no, groups).float()) * (1 - 2 * self.ints(2, no, groups)) * by).to(dtype)
        zero = self.ints(16, no, groups).to(torch.uint8)
        at = [self.put(codes, shift), self.put(scales, 2 * shift), self.put(zero, shift) if zeros else None]
        self.handle = ops().Linear4(self.pool, at[0], at[1], ni, no, group, dtype, zeros_off=at[2])
        k = torch.arange(ni, device="cuda")
        self.weights = (codes[:, k // 2] >> (4 * (k % 2)).to(torch.uint8) & 15).double()
        self.weights -= zero.double()[:, k // group] if zeros else 8
        self.weights *= scales.double()[:, k // group]

    def __del__(self):
        torch.cuda.synchronize()
        ft.pool_destroy(self.pool)

    def ints(self, hi, *shape):
        return torch.randint(hi, shape, device="cuda", generator=self.gen)

    def put(self, t, shift):
        raw = t.contiguous().view(-1).view(torch.uint8)
        at = ft.slab_alloc(self.pool, raw.numel() + shift) + shift
        self.mem[at:at + raw.numel()] = raw
        return at

    def x(self, rows, by=1.0):
        return ((self.ints(9, rows, self.ni) - 4).float() * by).to(self.dtype)

    def base(self, rows):
        return ((self.ints(33, rows, self.no) - 16).float() / 8).to(self.dtype)

    def product(self, x, base=None):
        """The result: in 64 bits no sum of these is rounded, and in 32 none has to be."""
        y = x.double() @ self.weights.t().contiguous()
        if base is not None:
            y += base.double()
        assert torch.equal(y, y.float().double())
        return y.to(self.dtype)


@pytest.mark.parametrize("rows,ni,no,group", [(1, 512, 200, 128), (9, 328, 90, 64), (16, 296, 64, 40), (2, 21, 30, 8), (20, 384, 11008, 128), (64, 640, 17000, 128),
                                              (64, 2112, 5000, 64), (40, 1320, 16400, 40)])
def test_scales_next_to_the_largest_number(rows, ni, no, group):
    """Scales of up to 2^123: no weight is beyond 2^127, but a scale times 128, and what the code counts from, is."""
    w = Exact(ni, no, group, BF16, seed=1, by=2.0 ** 123)
    x = w.x(rows, by=2.0 ** -110)
    out = ops().linear4_apply(w.handle, x)
    assert torch.isfinite(out).all() and torch.equal(out, w.product(x))
