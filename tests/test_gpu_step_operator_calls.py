"""Calls of the operators between projections and next tokens that are made in other ways than a step makes them."""
import pytest
import torch

from paper_2411_01830_amd import binding as ft

pytestmark = pytest.mark.gpu

SLAB = 4096
BF16, FP32 = torch.bfloat16, torch.float32


def ops():
    from paper_2411_01830_amd import operators
    return operators


@pytest.fixture()
def pool():
    mem = torch.zeros(64 * SLAB, dtype=torch.uint8, device="cuda")
    p = ft.pool_create(mem.data_ptr(), mem.numel(), SLAB, 0)
    yield p
    torch.cuda.synchronize()
    ft.pool_destroy(p)


def ints(*values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device="cuda")


@pytest.mark.parametrize("given", ["float32", "float64", "strided", "list"])
def test_a_rotation_keeps_the_frequencies_that_it_was_given(pool, given):
    """What becomes of the caller's tensor afterwards does not change it."""
    freqs = torch.linspace(1.0, 0.1, 64, device="cuda", dtype=torch.float64 if given == "float64" else FP32)
    freqs = freqs[::2] if given == "strided" else freqs[:32]
    q = torch.randn(7, 3, 64, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).to(BF16)
    at = torch.arange(7, dtype=torch.int32, device="cuda") * 100
    rotation = ops().Rotation(pool, freqs.tolist() if given == "list" else freqs, 64)
    before = ops().rotate_heads(rotation, q, None, at)[0]
    freqs.zero_()
    assert torch.equal(ops().rotate_heads(rotation, q, None, at)[0], before)
    assert not torch.equal(before, q)


@pytest.mark.parametrize("what", [None, 3, [0, 1]], ids=str)
def test_what_is_no_tensor_is_refused_as_everything_else_is(pool, what):
    o = ops()
    dtype = dict(dtype=BF16, device="cuda")
    rotation = o.Rotation(pool, [1.0] * 4, 8)
    weights = o.Linear4(pool, ft.slab_alloc(pool, SLAB), ft.slab_alloc(pool, SLAB), 64, 32, 32, BF16)
    cache = o.KvCache(pool, ft.slab_alloc(pool, SLAB), ft.slab_alloc(pool, SLAB), 2, 4, 1, 64, BF16)
    x, h, kv = torch.zeros(2, 64, **dtype), torch.zeros(2, 1, 8, **dtype), torch.zeros(2, 1, 64, **dtype)
    two, one, table, free, state = ints(0, 2), ints(1), ints(0)[None], ints(1, 0), ints(1, 0, 0, 0)
    t, p, r = ints(0, 1, dtype=torch.int64), torch.ones(2, 5, device="cuda"), torch.zeros(2, device="cuda")
    calls = {
        "x": lambda v: o.linear4_apply(weights, v), "base": lambda v: o.linear4_apply(weights, x, base=v), "out": lambda v: o.linear4_apply(weights, x, out=v),
        "q": lambda v: o.rotate_heads(rotation, v, None, two), "k": lambda v: o.rotate_heads(rotation, h, v, two), "positions": lambda v: o.rotate_heads(rotation, h, None, v),
        "q_weight": lambda v: o.rotate_heads(rotation, h, None, two, q_weight=v, eps=0.0), "k_weight": lambda v: o.rotate_heads(rotation, h, h, two, k_weight=v, eps=0.0),
        "q_out": lambda v: o.rotate_heads(rotation, h, None, two, q_out=v), "k_out": lambda v: o.rotate_heads(rotation, h, h, two, k_out=v),
        "tokens": lambda v: o.tree_verify(pool, v, two, 2, p, r, r[:1]), "starts": lambda v: o.tree_verify(pool, t, v, 2, p, r, r[:1]),
        "target": lambda v: o.tree_verify(pool, t, two, 2, v, r, r[:1]), "accept": lambda v: o.tree_verify(pool, t, two, 2, p, v, r[:1]),
        "pick": lambda v: o.tree_verify(pool, t, two, 2, p, r, v), "draft": lambda v: o.tree_verify(pool, t, two, 2, p, r, r[:1], draft=v),
        "parent": lambda v: o.tree_verify(pool, t, two, 2, p, r, r[:1], parent=v),
        "keep": lambda v: o.kv_grow(pool, one, two, 2, table, free, state, 4, keep=v), "done": lambda v: o.kv_release(pool, v, one, table, free, state, 4),
        "mask": lambda v: o.tree_attention(cache, kv, kv, kv, two, one, table, 2, mask=v),
    }
    optional = {"base", "out", "k", "q_weight", "k_weight", "q_out", "k_out", "draft", "parent", "keep", "mask"}
    for name, call in calls.items():
        if what is None and name in optional:
            continue
        with pytest.raises(ft.FtError) as err:
            call(what)
        assert err.value.code == -1, name


def defined(tokens, counts, target, accept, pick, draft):
    """Chains judged by the definition, row by row, in 64 bits."""
    keep, last, after, a = [], [], [], 0
    for r, n in enumerate(counts):
        row, left, keep_here = a, None, [1] + [0] * (n - 1)
        while True:
            p = target[row].double()
            left = p
            if row + 1 == a + n:
                break
            c = int(tokens[row + 1])
            q = draft[row].double() if draft is not None else None
            if float(accept[row + 1]) * (1.0 if q is None else float(q[c])) < float(p[c]):
                row += 1
                keep_here[row - a] = 1
                continue
            if q is None:
                left = p.clone()
                left[c] = 0
            else:
                left = (p - q).clamp(min=0)
            break
        left = left if float(left.sum()) > 0 else p
        sums = left.cumsum(0)
        after.append(int(torch.nonzero(sums > float(pick[r]) * float(sums[-1]))[0]))
        keep += keep_here
        last.append(row)
        a += n
    return keep, last, after


@pytest.mark.parametrize("requests,vocab,dtype,drawn,spread", [
    (128, 131072, FP32, True, True), (160, 131072, FP32, True, True), (161, 131072, FP32, True, False), (128, 262144, BF16, True, True), (90, 131072, FP32, False, False),
    (90, 262144, FP32, False, True), (90, 131071, FP32, True, False), (85, 131071, FP32, True, True), (86, 65536, BF16, False, False),
], ids=str)
def test_first_sums_are_spread_where_rows_are_long(pool, requests, vocab, dtype, drawn, spread):
    """Requests beyond a third of the compute units, on either side of the rule's 1 MiB a request, judged alike in one launch and in two."""
    units = torch.cuda.get_device_properties(0).multi_processor_count
    if units != 256:
        pytest.skip("the counts are for 256 compute units")
    gen = torch.Generator(device="cuda").manual_seed(requests + vocab)
    counts = [1 + r % 3 for r in range(requests)]
    starts = [0]
    for n in counts:
        starts.append(starts[-1] + n)
    rows = starts[-1]
    target, draft = torch.empty(rows, vocab, dtype=dtype, device="cuda"), torch.empty(rows, vocab, dtype=dtype, device="cuda")
    for a in range(0, rows, 64):
        logits = 3 * torch.randn(min(64, rows - a), vocab, device="cuda", generator=gen)
        target[a:a + 64] = torch.softmax(logits, -1)
        draft[a:a + 64] = torch.softmax(logits + 0.7 * torch.randn(logits.shape, device="cuda", generator=gen), -1)
    tokens = torch.zeros(rows, dtype=torch.int64, device="cuda")
    for row in range(1, rows):                             # a row's token was drawn by the row before
        q = draft[row - 1].float()
        tokens[row] = (q / torch.empty_like(q).exponential_(generator=gen)).argmax()
    accept, pick = torch.rand(rows, device="cuda", generator=gen), torch.rand(requests, device="cuda", generator=gen)
    record = ft.VerifyCall(rows=rows, requests=requests, drafts=3, vocab=vocab, type=2 if dtype is FP32 else 0, draft=draft.data_ptr() if drawn else None,
                           target_stride=vocab, draft_stride=vocab)
    # (without a draft the workspace is that of a call with one, which is spread wherever the other is)
    assert (ft.verify_workspace(pool, record) > 0) == (spread if drawn else requests <= 85 or vocab * target.element_size() * 2 >= 1 << 20)
    got = ops().tree_verify(pool, tokens, ints(*starts), 3, target, accept, pick, draft=draft if drawn else None)
    want = defined(tokens, counts, target, accept, pick, draft if drawn else None)
    assert got[0].tolist() == want[0]
    assert got[1].tolist() == want[1]
    assert got[2].tolist() == want[2]
