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


# (rows, width in, width out, group): the kernel that its sizes ask for on 256 compute units - for up to 2, 8 or 16 rows at a time; with 1, 2 or 4 tiles of 16
# rows, the work along the rows shared out or not, and how often a workgroup brings scales -, which test_linear4_plans.py compares with the library's rule
KINDS = {
    # few rows: groups of every kind, widths that end anywhere, up to as many groups as shared memory has room for
    (1, 8192, 512, 32): "narrow 2", (1, 12346, 512, 32): "narrow 2", (1, 20001, 333, 64): "narrow 2", (2, 20001, 333, 128): "narrow 2", (1, 4097, 600, 128): "narrow 2",
    (2, 513, 70, 40): "narrow 2", (1, 31001, 100, 32): "narrow 2", (2, 32768, 100, 32): "narrow 2",
    (3, 2047, 333, 40): "narrow 8", (7, 9001, 1000, 64): "narrow 8", (8, 9001, 1000, 128): "narrow 8", (8, 20001, 3333, 32): "narrow 8", (5, 17000, 2000, 32): "narrow 8",
    (4, 32768, 4096, 32): "narrow 8", (4, 12000, 700, 40): "narrow 8",
    (17, 700, 100, 32): "narrow 16", (33, 600, 200, 64): "narrow 16", (16, 2000, 4096, 128): "narrow 16", (16, 3001, 2001, 64): "narrow 16", (10, 8192, 4096, 32): "narrow 16",
    (16, 9001, 2000, 32): "narrow 16", (16, 9000, 3000, 128): "narrow 16", (9, 7003, 1500, 40): "narrow 16",
    # a tile of 16 rows
    (16, 1001, 40001, 128): "wide 1 whole 1", (16, 1001, 40001, 64): "wide 1 whole 1", (16, 3001, 40001, 32): "wide 1 whole 2",
    (64, 4100, 3001, 64): "wide 1 whole 2", (16, 8192, 8200, 128): "wide 1 shared 1", (9, 6000, 8000, 64): "wide 1 shared 1", (16, 20001, 8001, 32): "wide 1 shared 3",
    (41, 12345, 2000, 384): "wide 1 shared 1", (48, 20000, 2100, 1024): "wide 1 shared 1", (3, 32768, 1000, 32): "wide 1 shared 1", (16, 5000, 9001, 48): "wide 1 shared 1",
    # two
    (24, 1001, 20001, 128): "wide 2 whole 1", (24, 1501, 20001, 64): "wide 2 whole 1", (20, 2501, 17001, 40): "wide 2 whole 1", (32, 4201, 20001, 32): "wide 2 whole 3",
    (32, 9001, 20001, 64): "wide 2 whole 3", (32, 10001, 20001, 128): "wide 2 whole 2", (32, 8200, 2600, 128): "wide 2 shared 1", (24, 16001, 4000, 64): "wide 2 shared 1",
    (20, 4400, 5100, 72): "wide 2 shared 1", (70, 1000, 4100, 256): "wide 2 whole 1",
    # four
    (33, 1290, 32700, 40): "wide 4 whole 1",
    (64, 1100, 32000, 128): "wide 4 whole 1", (50, 1300, 31000, 64): "wide 4 whole 1", (64, 8191, 32001, 32): "wide 4 whole 4", (64, 8191, 32001, 64): "wide 4 whole 2",
    (64, 9001, 32000, 128): "wide 4 whole 2", (50, 3001, 32000, 40): "wide 4 whole 2", (100, 20001, 1000, 128): "wide 4 shared 1", (128, 20001, 4001, 64): "wide 4 shared 2",
    (128, 20001, 4000, 32): "wide 4 shared 3", (130, 16001, 4100, 40): "wide 4 shared 4", (64, 200, 60000, 128): "wide 4 whole 1",
    # the plain one
    (5, 1001, 77, 8): "any", (19, 333, 50, 24): "any", (2, 32801, 20, 32): "any", (9, 31, 40, 32): "any", (3, 40, 5, 32): "any",
}
CASES = list(KINDS)


def apart(rows, width, gap, at, dtype):
    """Rows of a larger tensor whose other elements are 7."""
    home = torch.full((rows, width + gap), 7.0, dtype=dtype, device="cuda")
    return home, home[:, at:at + width]


@pytest.mark.parametrize("dtype", [BF16, FP16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
def test_products_to_the_last_bit(case, dtype):
    """Whole tensors; rows apart at odd places, onto themselves, with nothing else written; rows beside one that is not finite."""
    rows, ni, no, group = case
    w = Exact(ni, no, group, dtype, zeros=ni % 3 != 1, seed=rows + ni, shift=ni % 2)
    x = w.x(rows)
    want = w.product(x)
    assert torch.equal(ops().linear4_apply(w.handle, x), want)

    base = w.base(rows)
    x_home, x_in = apart(rows, ni, 9, 5, dtype)
    home, out = apart(rows, no, 11, 3, dtype)
    x_in.copy_(x)
    out.copy_(base)
    assert ops().linear4_apply(w.handle, x_in, base=out, out=out) is out
    onto = w.product(x, base)
    assert torch.equal(out, onto)
    assert (home[:, :3] == 7).all() and (home[:, 3 + no:] == 7).all()
    other_home, other = apart(rows, no, 2, 1, dtype)
    ops().linear4_apply(w.handle, x_in, base=base, out=other)
    assert torch.equal(other, onto) and (other_home[:, 0] == 7).all() and (other_home[:, 1 + no:] == 7).all()

    bad = x.clone()
    where = {0: ni - 1, rows // 2: 0, rows - 1: ni // 2}
    for r, at in where.items():
        bad[r, at] = float("inf") if r % 2 else float("nan")
    got = ops().linear4_apply(w.handle, bad)
    fine = [r for r in range(rows) if r not in where]
    assert torch.equal(got[fine], want[fine]) and not torch.isfinite(got[list(where)]).any()


@pytest.mark.parametrize("dtype", [BF16, FP16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("rows,ni,no,group,stride", [(2, 515, 200, 64, 1 << 24), (17, 300, 90, 128, (1 << 24) + 3), (2, 515, 200, 64, (1 << 24) - 1),
                                                     (16, 3001, 301, 64, (1 << 24) - 1), (64, 1100, 32000, 128, (1 << 24) - 1), (24, 1501, 20001, 64, (1 << 24) - 1)])
def test_rows_of_x_far_apart(rows, ni, no, group, stride, dtype):
    """On either side of the strides whose offsets in a tile of rows 32 bits hold."""
    w = Exact(ni, no, group, dtype, seed=stride % 100)
    x = w.x(rows)
    far = torch.empty((rows - 1) * stride + ni, dtype=dtype, device="cuda").as_strided((rows, ni), (stride, 1))
    far.copy_(x)
    assert torch.equal(ops().linear4_apply(w.handle, far), w.product(x))


@pytest.mark.parametrize("rows,ni,no,group", [(140, 300, 40, 32), (140, 300, 24000, 128), (140, 16001, 200, 64)])
def test_rows_of_results_far_apart(rows, ni, no, group):
    """Beyond 2^31 elements and 2^32 bytes from the first one, onto what they hold."""
    stride = (1 << 24) + 1
    w = Exact(ni, no, group, BF16, seed=3)
    x, base = w.x(rows), w.base(rows)
    far = torch.empty((rows - 1) * stride + no, dtype=BF16, device="cuda").as_strided((rows, no), (stride, 1))
    far.copy_(base)
    ops().linear4_apply(w.handle, x, base=far, out=far)
    assert torch.equal(far, w.product(x, base))
