"""Weights of 4 bits, norms and rotations of heads, and drafted tokens judged, against plain 64-bit implementations.

Bounds come from the types and the order of sums alone. u is the unit roundoff of the tensors' type (bfloat16 2^-8, float16 2^-11), e that of
the 32 bits in between, 2^-24. What is decided - which rows stand, which token comes next - has to be equal."""
import math
import random

import pytest
import torch

from paper_2411_01830_amd import binding as ft

pytestmark = pytest.mark.gpu

SLAB = 4096
BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32
U = {BF16: 2.0 ** -8, FP16: 2.0 ** -11}
TINY = {BF16: 0.0, FP16: 2.0 ** -25}   # half the smallest float16
E = 2.0 ** -24


def ops():
    from paper_2411_01830_amd import operators
    return operators


class Memory:
    """A pool over one device tensor, filled with the bytes of NaN."""

    def __init__(self, nbytes):
        n = (nbytes + SLAB - 1) // SLAB * SLAB + 8 * SLAB
        self.mem = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
        self.pool = ft.pool_create(self.mem.data_ptr(), n, SLAB, 0)

    def put(self, t, shift=0):
        """An allocation that holds the tensor, `shift` bytes behind its beginning."""
        raw = t.contiguous().view(-1).view(torch.uint8)
        at = ft.slab_alloc(self.pool, max(1, raw.numel() + shift)) + shift
        self.mem[at:at + raw.numel()] = raw
        return at

    def __del__(self):
        torch.cuda.synchronize()
        ft.pool_destroy(self.pool)


def gpu(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device="cuda")


def within(got, want, bound):
    """Every element is off by at most its bound, and finite where the wanted one is."""
    got = got.double()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    share = torch.nan_to_num((got - want).abs() / bound, nan=0.0)
    assert float(share.max() if share.numel() else 0.0) <= 1, float(share.max())


# ---- weights of 4 bits ------------------------------------------------------------------------------

class Weights:
    def __init__(self, ni, no, group, dtype, zeros, seed, shift=0, wild=False):
        g = torch.Generator(device="cuda").manual_seed(seed)
        groups, row = -(-ni // group), (ni + 1) // 2
        self.codes = torch.randint(256, (no, row), dtype=torch.uint8, device="cuda", generator=g)
        self.scales = ((0.5 + torch.rand(no, groups, device="cuda", generator=g)) * (-1) ** torch.randint(2, (no, groups), device="cuda", generator=g)
                       * (0.2 * ni ** -0.5)).to(dtype)
        self.zeros = torch.randint(256 if wild else 16, (no, groups), dtype=torch.uint8, device="cuda", generator=g) if zeros else None
        self.m = Memory(no * row + 3 * no * groups + 4 * SLAB)
        at = self.m.put(self.codes, shift), self.m.put(self.scales, 2 * shift), self.m.put(self.zeros, shift) if zeros else None
        self.scales_off = at[1]
        self.handle = ops().Linear4(self.m.pool, at[0], at[1], ni, no, group, dtype, zeros_off=at[2])
        k = torch.arange(ni, device="cuda")
        self.scale = self.scales.double()[:, k // group]
        self.zero = self.zeros.double()[:, k // group] if zeros else torch.full((no, ni), 8.0, dtype=torch.float64, device="cuda")
        code = (self.codes[:, k // 2] >> (4 * (k % 2)).to(torch.uint8)) & 15
        self.off = code.double() - self.zero
        self.group, self.groups, self.dtype = group, groups, dtype

    def product(self, x, base=None):
        """The result and how far it may be off. Kernels may multiply with 128 + code and take away (128 + zero) times the sum of a group's x:
        sums of at most a group's elements then have terms of up to |x| (143 + 128 + zero). Groups are added behind that."""
        x = x.double()
        y = x @ (self.off * self.scale).t()
        terms = x.abs() @ ((271 + self.zero) * self.scale.abs()).t()
        direct = x.abs() @ (self.off.abs() * self.scale.abs()).t()
        if base is not None:
            y, direct = y + base.double(), direct + base.double().abs()
        return y, 1.001 * U[self.dtype] * y.abs() + TINY[self.dtype] + E * ((min(self.group, x.shape[1]) + 16) * terms + (self.groups + 32) * direct)


LINEAR = [
    # rows, width in, width out, group, zeros, base, shift in bytes
    (1, 8, 1, 8, False, False, 0), (1, 1, 1, 8, True, True, 0), (3, 7, 5, 8, True, False, 0), (2, 2, 3, 8, False, True, 1), (1, 4096, 4096, 128, False, False, 0),
    (1, 4096, 1000, 64, True, True, 0), (2, 1024, 129, 32, True, False, 0), (5, 1000, 777, 40, True, False, 0), (16, 2048, 512, 128, True, True, 0),
    (17, 1023, 65, 32, True, False, 0), (15, 640, 48, 64, False, False, 1), (33, 896, 272, 128, True, True, 0), (64, 1536, 640, 64, False, False, 0),
    (65, 512, 96, 32, True, True, 0), (200, 768, 80, 256, True, False, 0), (7, 8192, 96, 8192, True, False, 0), (9, 520, 100, 1024, True, False, 3),
    (4, 11008, 64, 128, False, False, 0), (1, 14336, 256, 64, True, False, 0), (31, 264, 33, 24, True, True, 5), (64, 96, 2048, 32, True, False, 0),
    # as many groups as shared memory has room for, and one more; widths and rows on either side of the rules that choose
    (16, 32768, 20, 32, True, True, 0), (3, 32776, 20, 32, True, False, 1), (2, 33000, 40, 32, False, False, 0), (24, 5000, 3001, 40, True, True, 1),
    (48, 4100, 2500, 96, True, False, 0), (64, 8192, 1111, 64, True, True, 0), (40, 2304, 5000, 32, False, True, 2), (12, 2100, 20001, 64, True, True, 1),
    (130, 3333, 700, 128, True, True, 3), (17, 513, 16400, 136, True, False, 0),
    # large enough for tiles that share rows of x: of 16, 32 and 64 rows, groups of every kind, work along the rows shared out or not, rows that end anywhere
    (16, 8192, 8200, 128, False, True, 0), (9, 6000, 8000, 64, True, False, 1), (16, 5000, 9001, 48, True, True, 2), (32, 8200, 2600, 128, True, False, 1),
    (17, 5000, 5003, 64, True, True, 0), (20, 4400, 5100, 72, True, False, 5), (64, 8192, 2000, 128, True, True, 0), (64, 4100, 3001, 64, True, False, 1),
    (50, 3000, 4999, 40, True, True, 3), (33, 2500, 6000, 32, False, False, 0), (64, 300, 40000, 256, True, False, 0), (64, 200, 60000, 128, True, True, 0),
    (300, 1024, 4096, 512, True, True, 0), (48, 20000, 2100, 1024, True, False, 0), (41, 12345, 2000, 384, True, True, 1),
    (64, 1100, 32000, 128, True, True, 1), (50, 1300, 31000, 64, True, False, 0), (33, 1290, 32700, 40, False, True, 3), (128, 14000, 4000, 64, True, True, 0),
    (256, 4096, 4000, 128, True, False, 0), (70, 1000, 4100, 256, False, False, 2),
]


@pytest.mark.parametrize("dtype", [BF16, FP16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("case", LINEAR, ids=lambda c: "-".join(map(str, c)))
def test_products_with_weights_of_four_bits(case, dtype):
    rows, ni, no, group, zeros, base, shift = case
    w = Weights(ni, no, group, dtype, zeros, rows + ni, shift)
    g = torch.Generator(device="cuda").manual_seed(no)
    x = torch.randn(rows, ni, device="cuda", generator=g).to(dtype)
    b = torch.randn(rows, no, device="cuda", generator=g).to(dtype) if base else None
    want, bound = w.product(x, b)
    out = ops().linear4_apply(w.handle, x, base=b)
    within(out, want, bound)
    again = ops().linear4_apply(w.handle, x, base=b)
    assert torch.equal(out, again)                                        # whatever order its workgroups ran in


@pytest.mark.parametrize("dtype", [BF16, FP16], ids=["bf16", "fp16"])
def test_products_of_rows_apart_in_place_and_beside_other_things(dtype):
    w = Weights(512, 200, 64, dtype, True, 1, wild=True)                     # zeros of any byte
    g = torch.Generator(device="cuda").manual_seed(2)
    wide = torch.randn(19, 600, device="cuda", generator=g).to(dtype)
    x = wide[:, 41:553]
    home = torch.randn(19, 211, device="cuda", generator=g).to(dtype)
    before = home.clone()
    out = home[:, 5:205]
    want, bound = w.product(x, out)
    assert ops().linear4_apply(w.handle, x, base=out, out=out) is out
    within(out, want, bound)
    assert torch.equal(home[:, :5], before[:, :5]) and torch.equal(home[:, 205:], before[:, 205:])
    base = before[:, 5:205]
    other = torch.full((19, 300), 7.0, dtype=dtype, device="cuda")
    ops().linear4_apply(w.handle, x, base=base, out=other[:, 100:])
    assert torch.equal(other[:, 100:], out) and (other[:, :100] == 7).all()


@pytest.mark.parametrize("dtype", [BF16, FP16], ids=["bf16", "fp16"])
def test_rows_and_columns_of_infinities_keep_to_themselves(dtype):
    w = Weights(384, 144, 32, dtype, True, 3)
    x = torch.randn(20, 384, device="cuda", generator=torch.Generator(device="cuda").manual_seed(4)).to(dtype)
    clean = ops().linear4_apply(w.handle, x)
    bad = x.clone()
    bad[3, 100], bad[17, 0], bad[18, 383] = math.inf, math.nan, -math.inf
    out = ops().linear4_apply(w.handle, bad)
    fine = [r for r in range(20) if r not in (3, 17, 18)]
    assert torch.equal(out[fine], clean[fine])
    assert not torch.isfinite(out[[3, 17, 18]]).any()
    b = clean.clone()
    b[5, 7] = math.nan
    out = ops().linear4_apply(w.handle, x, base=b)
    assert torch.isnan(out[5, 7]) and torch.isnan(out).sum() == 1


@pytest.mark.parametrize("rows,ni,no,group", [(1, 640, 300, 128), (9, 328, 90, 64), (16, 296, 64, 40), (2, 21, 30, 8), (20, 384, 11008, 128), (64, 640, 17000, 128),
                                              (64, 2112, 5000, 64), (40, 1320, 16400, 40), (70, 1290, 9001, 32)])
@pytest.mark.parametrize("dtype", [BF16, FP16], ids=["bf16", "fp16"])
def test_columns_whose_scales_are_not_finite_keep_to_themselves(rows, ni, no, group, dtype):
    w = Weights(ni, no, group, dtype, True, 6)
    x = torch.randn(rows, ni, device="cuda", generator=torch.Generator(device="cuda").manual_seed(7)).to(dtype)
    clean = ops().linear4_apply(w.handle, x)
    scales = w.m.mem[w.scales_off:][:2 * no * w.groups].view(dtype).view(no, w.groups)
    assert torch.equal(scales, w.scales)
    wild = torch.arange(4, no, 5, device="cuda")                              # (the rows before and behind them are not)
    scales[wild, 0], scales[wild[::2], 0] = math.inf, math.nan
    out = ops().linear4_apply(w.handle, x)
    fine = torch.ones(no, dtype=torch.bool, device="cuda")
    fine[wild] = False
    assert torch.equal(out[:, fine], clean[:, fine])
    assert not torch.isfinite(out[:, wild]).any()


def test_no_rows_have_no_products():
    w = Weights(64, 32, 32, BF16, False, 5)
    assert ops().linear4_apply(w.handle, torch.zeros(0, 64, dtype=BF16, device="cuda")).shape == (0, 32)


# ---- norms and rotations --------------------------------------------------------------------------------

def rotated(x, positions, freqs, axis, neighbours, eps, weight):
    """The definition in 64 bits, and the size that errors are relative to."""
    half = len(freqs)
    y = x.double()
    if eps is not None:
        y = y / (y.square().mean(-1, keepdim=True) + eps).sqrt() * (1 if weight is None else weight.double())
    angle = positions.double()[:, axis] * freqs.double()[None]
    c, s = angle.cos()[:, None], angle.sin()[:, None]
    first = torch.arange(half, device="cuda") * (2 if neighbours else 1)
    second = first + (1 if neighbours else half)
    out, size = y.clone(), y.abs()
    a, b = y[..., first], y[..., second]
    out[..., first], out[..., second] = a * c - b * s, a * s + b * c
    size[..., first] = size[..., second] = a.abs() + b.abs()
    return out, size


ROTATE = [
    # tokens, heads, key heads, dim, rot, axes, neighbours, norm, weights, furthest position, elements between heads
    (1, 1, 1, 8, 8, 1, False, False, False, 100, 0), (1, 32, 8, 128, 128, 1, False, True, True, 131072, 0), (3, 4, 0, 64, 64, 1, True, True, False, 2 ** 31, 0),
    (77, 5, 1, 80, 80, 3, True, True, True, 512, 0), (64, 6, 2, 96, 96, 1, False, False, False, 9000, 3), (33, 3, 3, 72, 34, 2, False, True, True, 4096, 1),
    (50, 2, 1, 128, 64, 1, True, False, False, 1 << 20, 0), (19, 4, 4, 256, 256, 4, False, True, True, 70000, 0), (20, 1, 2, 256, 2, 1, True, True, True, 50, 5),
    (40, 7, 7, 64, 0, 1, False, True, True, 10, 0), (11, 3, 1, 64, 30, 1, False, True, False, 5000, 0), (129, 8, 2, 128, 96, 3, False, True, True, 60000, 0),
    (4099, 4, 1, 128, 128, 1, False, True, True, 32768, 0), (513, 16, 16, 80, 40, 2, True, True, True, 2000, 8), (21, 5, 5, 24, 24, 1, False, True, True, 99, 0),
    (6, 40, 8, 128, 128, 1, True, False, False, 1 << 24, 0), (260, 3, 2, 40, 16, 1, True, True, False, 300, 0),
    # fewer pairs than eight, and several tokens to a workgroup
    (30, 4, 2, 256, 14, 2, False, True, True, 8000, 1), (9, 2, 1, 64, 2, 1, False, False, False, 1 << 20, 0), (5000, 1, 1, 64, 64, 1, False, True, True, 9000, 0),
    (2061, 3, 2, 256, 256, 2, False, True, False, 40000, 0), (6001, 2, 0, 48, 40, 1, False, True, True, 6001, 3),
]


@pytest.mark.parametrize("dtype", [BF16, FP16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("case", ROTATE, ids=lambda c: "-".join(map(str, c)))
def test_heads_normed_and_rotated(case, dtype):
    tokens, heads, kv, dim, rot, axes, neighbours, norm, weighted, far, gap = case
    g = torch.Generator(device="cuda").manual_seed(tokens + dim)
    rng = random.Random(str(case))
    m = Memory(SLAB)
    wide = torch.randn(tokens, heads + kv, dim + gap, device="cuda", generator=g).mul_(3).to(dtype)
    q, k = wide[:, :heads, gap:], wide[:, heads:, gap:]
    positions = torch.randint(-far, far, (tokens, axes), device="cuda", generator=g, dtype=torch.int64).clamp(-2 ** 31, 2 ** 31 - 1).to(torch.int32)
    positions[0] = min(far, 2 ** 31 - 1)
    freqs = torch.tensor([10000.0 ** (-2 * i / max(rot, 1)) for i in range(rot // 2)], device="cuda")
    axis = [rng.randrange(axes) for _ in range(rot // 2)]
    if axes > 1:
        axis[0] = axes - 1
    rotation = ops().Rotation(m.pool, freqs, dim, axes=axis if axes > 1 else None, neighbours=neighbours)
    eps = 1e-5 if norm else None
    weights = [(1 + 0.3 * torch.randn(dim, device="cuda", generator=g)).to(dtype) if weighted else None for _ in range(2)]
    given = wide.clone()
    got = ops().rotate_heads(rotation, q, k if kv else None, positions if axes > 1 or tokens % 2 else positions[:, 0].contiguous(),
                             q_weight=weights[0], k_weight=weights[1] if kv else None, eps=eps)
    assert torch.equal(wide, given)
    at = torch.tensor(axis, dtype=torch.int64, device="cuda")
    for x, y, w in ((q, got[0], weights[0]), (k, got[1], weights[1])):
        if x.shape[1] == 0:
            assert y is None
            continue
        want, size = rotated(x, positions, freqs, at, neighbours, eps, w)
        # the norm's sum of squares, root and products: below 12 e together; sine and cosine 3 e of their own and 2 of the angle; two products
        # and a sum. Positions of 31 bits: angles of 2^31 in 53 bits are off by 2^-21.
        within(y, want, 1.001 * U[dtype] * want.abs() + (20 * E + (2.0 ** -20 if far > 2 ** 28 else 0)) * size + TINY[dtype])
    # in place: the same bits
    ops().rotate_heads(rotation, q, k if kv else None, positions, q_weight=weights[0], k_weight=weights[1] if kv else None, eps=eps, q_out=q,
                       k_out=k if kv else None)
    assert torch.equal(q, got[0]) and (not kv or torch.equal(k, got[1]))
    assert torch.equal(wide[..., :gap], given[..., :gap])                   # what lies between the heads stays


def test_position_zero_and_heads_without_a_norm_are_copies():
    m = Memory(SLAB)
    x = torch.randn(9, 6, 128, device="cuda").to(BF16)
    rotation = ops().Rotation(m.pool, [1.0 / (i + 1) for i in range(64)], 128)
    q, k = ops().rotate_heads(rotation, x[:, :4], x[:, 4:], torch.zeros(9, dtype=torch.int32, device="cuda"))
    assert torch.equal(q, x[:, :4]) and torch.equal(k, x[:, 4:])


def test_turning_back_and_forth_keeps_products():
    """Products of rotated queries and keys depend on the distance of their positions alone."""
    m = Memory(SLAB)
    g = torch.Generator(device="cuda").manual_seed(0)
    q, k = torch.randn(1, 1, 128, device="cuda", generator=g).to(FP16), torch.randn(1, 1, 128, device="cuda", generator=g).to(FP16)
    rotation = ops().Rotation(m.pool, [10000.0 ** (-i / 64) for i in range(64)], 128)
    at = [0, 5, 1000, 65536, 10 ** 6, -77]
    qs, ks = ops().rotate_heads(rotation, q.expand(6, 1, 128), k.expand(6, 1, 128), gpu([a + 13 for a in at]), eps=0.0)[0], \
        ops().rotate_heads(rotation, k.expand(6, 1, 128), None, gpu(at), eps=0.0)[0]
    s = (qs.double() * ks.double()).sum(-1)[:, 0]
    # 128 products of two rounded numbers each: the root of the sum of squares is 128 for either side
    assert float((s - s[0]).abs().max()) <= 128 * 4 * U[FP16]


@pytest.mark.parametrize("dim,rot,neighbours", [(128, 128, False), (80, 80, True), (72, 34, False)])
def test_heads_of_infinities_keep_to_themselves(dim, rot, neighbours):
    m = Memory(SLAB)
    x = torch.randn(12, 5, dim, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).to(FP16)
    rotation = ops().Rotation(m.pool, [0.5 ** i for i in range(rot // 2)], dim, neighbours=neighbours)
    at = torch.arange(12, dtype=torch.int32, device="cuda")
    clean = ops().rotate_heads(rotation, x[:, :3], x[:, 3:], at, eps=1e-6)
    bad = x.clone()
    bad[2, 1, 7], bad[5, 4, dim - 1], bad[7, 0, 0] = math.inf, math.nan, -math.inf
    zero = bad[9, 2].zero_()
    got = ops().rotate_heads(rotation, bad[:, :3], bad[:, 3:], at, eps=1e-6)
    for t in range(12):
        for h in range(5):
            a, b = (clean[0][t, h], got[0][t, h]) if h < 3 else (clean[1][t, h - 3], got[1][t, h - 3])
            if (t, h) == (9, 2):
                assert (b == 0).all() and zero.numel() == dim
            elif (t, h) in ((2, 1), (5, 4), (7, 0)):
                assert torch.isnan(b).any()
            else:
                assert torch.equal(a, b)


# ---- drafted tokens judged ----------------------------------------------------------------------------------

def judged(tokens, starts, drafts, target, draft, accept, pick, parent):
    """The definition, row by row, in 64 bits on the CPU."""
    target, draft = target.double().cpu(), None if draft is None else draft.double().cpu()
    rest = lambda t: torch.where(t > 0, t, 0)  # noqa: E731  (of NaN nothing is left)
    vocab = target.shape[1]
    keep, last, after = [0] * len(tokens), [], []
    for r, (a, b) in enumerate(zip(starts, starts[1:])):
        b = min(b, a + drafts)
        if b <= a:
            last.append(-1)
            after.append(-1)
            continue
        row, keep[a] = a, 1
        while True:
            p = rest(target[row])
            left, mass, taken = p.clone(), 1.0, 0.0
            found = None
            for t in range(row + 1, b):
                if (parent[t] if parent is not None else t - a - 1) != row - a or (parent is not None and parent[t] >= t - a):
                    continue
                c = tokens[t]
                inside = 0 <= c < vocab
                here = float(left[c]) if inside else 0.0
                q = 1.0 if draft is None else (float(draft[row][c]) if inside else 0.0)
                if accept[t] * mass * q < here:
                    found = t
                    break
                if draft is None:
                    if inside:
                        left[c] = 0
                    mass = max(mass - here, 0.0)
                else:
                    taken += mass
                    left = rest(target[row] - taken * draft[row])
                    mass = float(left.sum())
            if found is None:
                break
            row, keep[found] = found, 1
        if float(left.sum()) == 0:
            left = p
        sums = left.cumsum(0)
        over = torch.nonzero((sums > pick[r] * float(sums[-1])) & (left > 0))[:, 0]
        some = torch.nonzero(left > 0)[:, 0]
        after.append(int(over[0]) if len(over) else int(some[-1]) if len(some) else -1)
        last.append(row)
    return keep, last, after


def drafted(rng, gen, counts, vocab, tree, drawn, dtype, spread=3.0, noise=0.7, lead=0, tail=0):
    """Trees (or chains) of tokens drawn from a draft that is near the target."""
    starts = [lead]
    for n in counts:
        starts.append(starts[-1] + n)
    rows = starts[-1] + tail
    parent = [0] * rows
    for a, b in zip(starts, starts[1:]):
        for i in range(b - a):
            parent[a + i] = -1 if i == 0 else rng.randrange(max(0, i - 3), i) if tree else i - 1
    logits = torch.randn(rows, vocab, device="cuda", generator=gen) * spread
    target = torch.softmax(logits, -1).to(dtype)
    draft = torch.softmax(logits + noise * torch.randn(rows, vocab, device="cuda", generator=gen), -1).to(dtype)
    first = [0] * rows
    for a, b in zip(starts, starts[1:]):
        for t in range(a, b):
            first[t] = a
    of = draft[gpu([f + max(p, 0) for f, p in zip(first, parent)], torch.int64)].float() if rows else draft.float()
    tokens = (of / torch.empty_like(of).exponential_(generator=gen)).argmax(-1) if rows else torch.zeros(0, dtype=torch.int64, device="cuda")
    if not drawn:
        draft = None
    accept = torch.rand(rows, device="cuda", generator=gen)
    pick = torch.rand(len(counts), device="cuda", generator=gen)
    return starts, rows, parent if tree else None, target, draft, tokens, accept, pick


def judge(m, starts, drafts, parent, target, draft, tokens, accept, pick):
    """The operator's answer, which has to be the definition's."""
    got = ops().tree_verify(m.pool, tokens, gpu(starts), drafts, target, accept, pick, draft=draft, parent=None if parent is None else gpu(parent))
    want = judged(tokens.tolist(), starts, drafts, target, draft, accept.tolist(), pick.tolist(), parent)
    assert got[0].tolist() == want[0]
    assert got[1].tolist() == want[1]
    assert got[2].tolist() == want[2]
    return got


VERIFY = [
    # requests, rows of a request up to, vocabulary, tree
    (1, 1, 1, False), (1, 1, 5000, False), (1, 5, 32768, False), (3, 4, 2, True), (40, 8, 7, True), (17, 12, 1023, True), (17, 12, 1024, False), (9, 6, 1025, True),
    (64, 8, 2048, False), (5, 70, 3001, True), (2, 200, 515, True), (300, 5, 100, True), (6, 9, 70001, True), (2, 3, 262144, False), (1, 1024, 40, True),
    (1, 16, 131072, True), (3, 0, 64, True), (30, 3, 33000, True), (85, 2, 32769, True), (90, 3, 34000, False),
]


@pytest.mark.parametrize("dtype", [BF16, FP16, FP32], ids=["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("drawn", [True, False], ids=["drawn", "chosen"])
@pytest.mark.parametrize("case", VERIFY, ids=lambda c: "-".join(map(str, c)))
def test_drafted_tokens_judged(case, drawn, dtype):
    requests, most, vocab, tree = case
    rng = random.Random(str((case, drawn, dtype)))
    gen = torch.Generator(device="cuda").manual_seed(vocab + most)
    counts = [most] + [rng.choice([most, rng.randint(0, most)]) for _ in range(requests - 1)]
    lead, tail = rng.choice([(0, 0), (3, 5)])
    m = Memory(SLAB)
    starts, rows, parent, target, draft, tokens, accept, pick = drafted(rng, gen, counts, vocab, tree, drawn, dtype, lead=lead, tail=tail)
    judge(m, starts, max(most, 1), parent, target, draft, tokens, accept, pick)


@pytest.mark.parametrize("drawn", [True, False], ids=["drawn", "chosen"])
def test_many_siblings_that_fall(drawn):
    """Draft and target disagree: nearly all siblings fall, and what is left is cut down once for each."""
    rng, gen = random.Random(7), torch.Generator(device="cuda").manual_seed(7)
    m = Memory(SLAB)
    starts, rows, parent, target, draft, tokens, accept, pick = drafted(rng, gen, [40] * 12, 3000, True, drawn, FP32, spread=2.0, noise=4.0)
    for a in starts[:-1]:
        for i in range(1, 40):
            parent[a + i] = 0 if i < 30 else rng.randrange(30)
    kept = judge(m, starts, 40, parent, target, draft, tokens, accept * 0.5 + 0.5, pick)[0]
    assert kept.sum() < 60


def test_alike_siblings_and_tokens_that_there_are_not():
    m = Memory(SLAB)
    gen = torch.Generator(device="cuda").manual_seed(3)
    target = torch.softmax(torch.randn(24, 50, device="cuda", generator=gen), -1)
    draft = torch.softmax(torch.randn(24, 50, device="cuda", generator=gen), -1)
    tokens = gpu([4, 9, 9, 9, -1, 50, 2 ** 40, 9] * 3, torch.int64)
    parent = [-1, 0, 0, 0, 0, 0, 0, 0] * 3
    for accept in (0.999, 0.5, 0.0):
        for d in (draft, None):
            judge(m, [0, 8, 16, 24], 8, parent, target, d, tokens, torch.full((24,), accept, device="cuda"), gpu([0.0, 0.4, 0.99999], FP32))


def test_parents_of_any_kind_are_looked_at_between_their_bounds():
    m = Memory(SLAB)
    rng, gen = random.Random(5), torch.Generator(device="cuda").manual_seed(5)
    starts, rows, parent, target, draft, tokens, accept, pick = drafted(rng, gen, [9, 30, 1, 64], 300, True, True, FP32)
    for t in range(rows):
        if rng.random() < 0.4:
            parent[t] = rng.choice([-2 ** 31, -5, 2 ** 31 - 1, 77, 8, 29, 63, t])
    judge(m, starts, 64, parent, target, draft, tokens, accept, pick)
    for bad in ([-9, 50, 20, 2 ** 31 - 1, 104], [104, 30, 2, -2 ** 31, 9]):   # starts that descend or leave the rows: in bounds, whatever comes of it
        got = ops().tree_verify(m.pool, tokens, gpu(bad), 64, target, accept, pick, draft=draft, parent=gpu(parent))
        assert ((got[1] >= -1) & (got[1] < rows)).all() and ((got[2] >= -1) & (got[2] < 300)).all()


def test_rows_beyond_the_drafts_are_not_judged():
    m = Memory(SLAB)
    rng, gen = random.Random(6), torch.Generator(device="cuda").manual_seed(6)
    starts, rows, parent, target, draft, tokens, accept, pick = drafted(rng, gen, [9, 12, 3], 500, True, True, BF16)
    for drafts in (1, 5, 11, 1024, 5000):
        judge(m, starts, drafts, parent, target, draft, tokens, accept, pick)


def test_probabilities_that_are_none_count_as_nothing():
    """NaN and negative numbers of either side, infinities of the draft, rows of zeros, a draft that is the target."""
    m = Memory(SLAB)
    rng, gen = random.Random(8), torch.Generator(device="cuda").manual_seed(8)
    starts, rows, parent, target, draft, tokens, accept, pick = drafted(rng, gen, [6] * 20, 1500, True, True, FP32)
    wild = torch.rand(rows, 1500, device="cuda", generator=gen)
    target[wild < 0.02], target[(wild > 0.6) & (wild < 0.61)] = math.nan, -0.3
    wild = torch.rand(rows, 1500, device="cuda", generator=gen)
    draft[wild < 0.02], draft[(wild > 0.5) & (wild < 0.51)], draft[(wild > 0.6) & (wild < 0.61)] = math.nan, math.inf, -0.3
    target[6:12] = 0
    target[12:18] = draft[12:18]
    draft[18:24] = 0
    target[24:30], draft[24:30] = math.nan, math.nan
    target[30:36] = 0
    target[30:36, 1499] = 1e-42                                            # denormal
    token = judge(m, starts, 6, parent, target, draft, tokens, accept, pick)[2]
    judge(m, starts, 6, parent, target, None, tokens, accept, pick)
    judge(m, starts, 6, None, target, draft, tokens, gpu([math.nan, 2.0, -1.0] * 40, FP32), gpu([math.nan, 1.0, 7.0, -1.0] * 5, FP32))
    target[60:] = math.inf                                                 # what comes of these is a token, or none
    got = ops().tree_verify(m.pool, tokens, gpu(starts), 6, target, accept, pick, draft=draft, parent=gpu(parent))
    assert torch.equal(got[2][:10], token[:10]) and ((got[2] >= -1) & (got[2] < 1500)).all()


@pytest.mark.parametrize("drawn", [True, False], ids=["drawn", "chosen"])
def test_rows_of_which_nothing_is_left(drawn):
    """A target of zeros has no token; one that is the draft's equal, or below it, is gone after its first fall, and is taken whole then."""
    m = Memory(SLAB)
    rng, gen = random.Random(10), torch.Generator(device="cuda").manual_seed(10)
    starts, rows, parent, target, draft, tokens, accept, pick = drafted(rng, gen, [5] * 8, 3000, True, True, FP32)
    target[0:5] = 0
    target[5:10] = draft[5:10] * 0.5
    target[10:15] = draft[10:15]
    target[15:20] = 0
    target[15:20, 2999] = 1e-42                                            # denormal
    accept[5:10] = 0.9
    token = judge(m, starts, 5, parent, target, draft if drawn else None, tokens, accept, pick)[2]
    assert token[0] == -1 and token[1] >= 0 and token[3] == 2999


@pytest.mark.parametrize("dtype", [BF16, FP16, FP32], ids=["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("drawn", [True, False], ids=["drawn", "chosen"])
def test_rows_of_probabilities_apart_and_at_odd_places(drawn, dtype):
    m = Memory(SLAB)
    rng, gen = random.Random(9), torch.Generator(device="cuda").manual_seed(9)
    starts, rows, parent, target, draft, tokens, accept, pick = drafted(rng, gen, [7, 0, 9], 2051, True, drawn, dtype)
    wide = torch.full((rows, 2, 2060), math.nan, dtype=dtype, device="cuda")
    wide[:, 0, 3:2054] = target
    if drawn:
        wide[:, 1, 1:2052] = draft
    want = judge(m, starts, 9, parent, target, draft, tokens, accept, pick)
    got = ops().tree_verify(m.pool, tokens, gpu(starts), 9, wide[:, 0, 3:2054], accept, pick, draft=wide[:, 1, 1:2052] if drawn else None, parent=gpu(parent))
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("drawn", [True, False], ids=["drawn", "chosen"])
def test_what_comes_out_is_distributed_as_the_target(drawn):
    """A node with three siblings and a child behind the first: the token behind the first row follows its row of the target, whatever the draft.
    With n requests the count of a token of probability p has a deviation of sqrt(n p (1 - p)); of six counts none is further than five of them
    in more than one of 10^5 seeds, and the seed is fixed."""
    n, vocab = 40000, 6
    m = Memory(SLAB)
    gen = torch.Generator(device="cuda").manual_seed(11)
    p = torch.tensor([0.4, 0.25, 0.15, 0.1, 0.07, 0.03], device="cuda")
    q = torch.tensor([0.1, 0.1, 0.2, 0.2, 0.2, 0.2], device="cuda")
    target, draft = p.expand(4 * n, vocab).contiguous(), q.expand(4 * n, vocab).contiguous()
    tokens = torch.multinomial(q, 4 * n, replacement=True, generator=gen) if drawn else gpu([0, 3, 1, 3] * n, torch.int64)
    starts = torch.arange(0, 4 * n + 1, 4, dtype=torch.int32, device="cuda")
    parent = gpu([-1, 0, 0, 0] * n)
    kept, last, token = ops().tree_verify(m.pool, tokens, starts, 4, target, torch.rand(4 * n, device="cuda", generator=gen), torch.rand(n, device="cuda", generator=gen),
                                          draft=draft if drawn else None, parent=parent)
    kept = kept.view(n, 4)
    first = torch.where(kept[:, 1:].sum(-1) > 0, tokens[last.long()], token)
    assert (kept.sum(-1) <= 2).all()
    for c in range(vocab):
        expect = n * float(p[c])
        assert abs(int((first == c).sum()) - expect) <= 5 * math.sqrt(expect * (1 - float(p[c]))), c


# ---- streams and graphs -------------------------------------------------------------------------------------

def test_calls_of_a_step_in_a_graph_and_on_another_stream():
    """The three together, captured once and replayed with other inputs, eager work between the replays; and on two streams at once."""
    w = Weights(256, 192, 64, BF16, True, 12)
    gen = torch.Generator(device="cuda").manual_seed(12)
    rng = random.Random(12)
    rotation = ops().Rotation(w.m.pool, [0.9 ** i for i in range(16)], 32)
    starts, rows, parent, target, draft, tokens, accept, pick = drafted(rng, gen, [5, 3, 8], 2000, True, True, FP32)
    x = torch.randn(rows, 256, device="cuda", generator=gen).to(BF16)
    at, begin, hangs = torch.arange(rows, dtype=torch.int32, device="cuda"), gpu(starts), gpu(parent)

    def step():
        qkv = ops().linear4_apply(w.handle, x).view(rows, 6, 32)
        q, k = ops().rotate_heads(rotation, qkv[:, :4], qkv[:, 4:], at, eps=1e-6)
        return (q, k, *ops().tree_verify(w.m.pool, tokens, begin, 8, target, accept, pick, draft=draft, parent=hangs))

    eager = [t.clone() for t in step()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = step()
    here = step()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) and torch.equal(a, c) for a, b, c in zip(eager, other, here))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for _ in range(4):
        x.copy_(torch.randn(rows, 256, device="cuda", generator=gen))
        accept.copy_(torch.rand(rows, device="cuda", generator=gen))
        pick.copy_(torch.rand(3, device="cuda", generator=gen))
        at.add_(1000)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured, step()))
        judge(w.m, starts, 8, parent, target, draft, tokens, accept, pick)


def test_calls_with_workspaces_in_two_graphs_at_once():
    """Products shared out along the rows and sums by many workgroups, both with workspaces: two captured steps replayed on two streams together."""
    w = Weights(4096, 4000, 64, FP16, True, 14)
    rng = random.Random(14)

    class Step:
        def __init__(self, seed, stream):
            self.gen, self.stream = torch.Generator(device="cuda").manual_seed(seed), stream
            starts, rows, parent, self.target, self.draft, self.tokens, self.accept, self.pick = drafted(rng, self.gen, [9, 1, 12, 18], 40001, True, True, BF16)
            self.starts, self.parent, self.rows = gpu(starts), gpu(parent), rows
            self.x = torch.randn(rows, 4096, device="cuda", generator=self.gen).to(FP16)

        def run(self):
            return (ops().linear4_apply(w.handle, self.x), *ops().tree_verify(w.m.pool, self.tokens, self.starts, 18, self.target, self.accept, self.pick,
                                                                             draft=self.draft, parent=self.parent))

    steps = [Step(1, torch.cuda.Stream()), Step(2, torch.cuda.Stream())]
    for s in steps:
        assert s.rows == 40
        s.run()
        torch.cuda.synchronize()
        s.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(s.graph):
            s.out = s.run()
    for _ in range(4):
        for s in steps:
            s.x.copy_(torch.randn(s.rows, 4096, device="cuda", generator=s.gen))
            s.accept.copy_(torch.rand(s.rows, device="cuda", generator=s.gen))
        torch.cuda.synchronize()
        for s in steps:
            with torch.cuda.stream(s.stream):
                s.graph.replay()
        torch.cuda.synchronize()
        for s in steps:
            assert all(torch.equal(a, b) for a, b in zip(s.out, s.run()))
    want, bound = w.product(steps[0].x)
    within(steps[0].out[0], want, bound)


def test_tensors_that_ask_for_gradients_or_lie_elsewhere_are_refused():
    w = Weights(64, 32, 32, BF16, False, 13)
    rotation = ops().Rotation(w.m.pool, [1.0] * 4, 8)
    x = torch.zeros(2, 64, dtype=BF16, device="cuda")
    h = torch.zeros(2, 1, 8, dtype=BF16, device="cuda")
    at = gpu([0, 1])
    p, t, r = torch.ones(2, 5, device="cuda"), gpu([0, 1], torch.int64), torch.zeros(2, device="cuda")
    calls = [
        lambda: ops().linear4_apply(w.handle, x.clone().requires_grad_()), lambda: ops().linear4_apply(w.handle, x.float()), lambda: ops().linear4_apply(w.handle, x.cpu()),
        lambda: ops().linear4_apply(w.handle, x[:, :63]), lambda: ops().linear4_apply(w.handle, x, base=x), lambda: ops().linear4_apply(w.handle, x, out=x[:1, :32]),
        lambda: ops().rotate_heads(rotation, h.clone().requires_grad_(), None, at), lambda: ops().rotate_heads(rotation, h, h.float(), at),
        lambda: ops().rotate_heads(rotation, h, None, at.long()), lambda: ops().rotate_heads(rotation, h, None, at[:1]),
        lambda: ops().rotate_heads(rotation, h, None, at, q_weight=h[0, 0]), lambda: ops().rotate_heads(rotation, h, None, at, q_weight=h[0, 0, :7], eps=0.0),
        lambda: ops().rotate_heads(rotation, h, None, at, k_out=h), lambda: ops().rotate_heads(rotation, h, None, at, eps=-1.0),
        lambda: ops().rotate_heads(rotation, h, None, at, eps=1e300), lambda: ops().rotate_heads(rotation, h, None, at, eps=math.nan),
        lambda: ops().tree_verify(w.m.pool, t, gpu([0, 2]), -1, p, r, r[:1]), lambda: ops().tree_verify(w.m.pool, t, gpu([0, 2]), 1 << 40, p, r, r[:1]),
        lambda: ops().rotate_heads(rotation, h, None, at, q_out=h[:1].expand(2, 1, 8)), lambda: ops().rotate_heads(rotation, h.float(), None, at),
        lambda: ops().rotate_heads(ops().Rotation(w.m.pool, [1.0] * 4, 8, axes=[0, 0, 1, 1]), h, None, at),
        lambda: ops().tree_verify(w.m.pool, t, gpu([0, 2]), 2, p, r, r[:1], draft=p.half()), lambda: ops().tree_verify(w.m.pool, t, gpu([0, 2]), 2, p, r, r),
        lambda: ops().tree_verify(w.m.pool, t, gpu([0, 2]), 2, p, r[:1], r[:1]), lambda: ops().tree_verify(w.m.pool, t, gpu([0, 2]), 0, p, r, r[:1]),
        lambda: ops().tree_verify(w.m.pool, t, gpu([0, 2]), 2, p.double(), r, r[:1]), lambda: ops().tree_verify(w.m.pool, t, gpu([0, 2]), 2, p.t(), r, r[:1]),
        lambda: ops().tree_verify(w.m.pool, t, gpu([0, 2]), 2, p, r, r[:1], parent=gpu([0])), lambda: ops().tree_verify(w.m.pool, t.int(), gpu([0, 2]), 2, p, r, r[:1]),
        lambda: ops().tree_verify(w.m.pool, t, gpu([0, 2]), 2, p.clone().requires_grad_(), r, r[:1]),
    ]
    for i, call in enumerate(calls):
        with pytest.raises(ft.FtError) as err:
            call()
        assert err.value.code == -1, i
    with torch.no_grad():
        ops().linear4_apply(w.handle, x.clone().requires_grad_())
