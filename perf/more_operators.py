"""What a serving step does between its projections and its next tokens, operator by operator.

Beside the cache in the pool and its attention a step of a language model asks for
  linear   projections of few rows with weights of 4 bits, which transfers bring into the pool at a quarter of the bytes
  rotate   the norm of every head's query or key, and its rotation by the token's position, along one axis or several
  verify   which of a request's drafted tokens stand against the target's probabilities, and the token behind them
Each is a kind of case. Values come from the seed; trees, sections and the like from the case's `shape`.
"""
import random

import torch

own = False

SLAB = 64 << 10  # the pool's granule
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZES = {"bf16": 2, "fp16": 2, "fp32": 4}
EPS = 1e-6
LARGEST_PROBABILITIES = 1 << 26  # rows x vocabulary
LARGEST_WEIGHTS = 8192 * 32768


def listed():
    return [
        # the smallest calls: one request decodes one token, far into a long document
        {"name": "rotate_one", "kind": "rotate", "tokens": 1, "heads": 32, "kv_heads": 8, "dim": 128, "rot": 128, "axes": 1, "far": 131072,
         "neighbours": False, "norm": True, "type": "bf16", "shape": 1},
        # the rows of 64 trees of 16
        {"name": "rotate_step", "kind": "rotate", "tokens": 1024, "heads": 32, "kv_heads": 8, "dim": 128, "rot": 128, "axes": 1, "far": 32768,
         "neighbours": False, "norm": True, "type": "bf16", "shape": 2},
        # patches of an image or a video: time, height and width have pairs of their own, as many key heads as query heads
        {"name": "rotate_patches", "kind": "rotate", "tokens": 4111, "heads": 16, "kv_heads": 16, "dim": 80, "rot": 80, "axes": 3, "far": 512,
         "neighbours": True, "norm": True, "type": "bf16", "shape": 3},
        # the prompts of a batch, without norms
        {"name": "rotate_prompts", "kind": "rotate", "tokens": 32773, "heads": 32, "kv_heads": 8, "dim": 128, "rot": 128, "axes": 1, "far": 32768,
         "neighbours": False, "norm": False, "type": "fp16", "shape": 4},
        # a chain of four drafted tokens of one request
        {"name": "verify_one", "kind": "verify", "requests": 1, "new_lo": 5, "new_hi": 5, "tree": False, "drawn": True, "vocab": 32768,
         "type": "fp32", "shape": 5},
        # chains of three to seven of 64 requests, a large vocabulary
        {"name": "verify_chains", "kind": "verify", "requests": 64, "new_lo": 4, "new_hi": 8, "tree": False, "drawn": True, "vocab": 131072,
         "type": "fp32", "shape": 6},
        # trees whose siblings a small model has drawn
        {"name": "verify_trees", "kind": "verify", "requests": 32, "new_lo": 9, "new_hi": 16, "tree": True, "drawn": True, "vocab": 50001,
         "type": "bf16", "shape": 7},
        # trees of tokens that were looked up, not drawn: no probabilities of their own
        {"name": "verify_chosen", "kind": "verify", "requests": 17, "new_lo": 3, "new_hi": 25, "tree": True, "drawn": False, "vocab": 100003,
         "type": "fp16", "shape": 8},
        # one token's queries, keys and values
        {"name": "linear_token", "kind": "linear", "rows": 1, "width_in": 4096, "width_out": 6144, "group": 128, "zeros": False, "base": False,
         "type": "bf16", "shape": 9},
        # a token each of 16 requests, onto what they had before
        {"name": "linear_step", "kind": "linear", "rows": 16, "width_in": 4096, "width_out": 4096, "group": 64, "zeros": True, "base": True,
         "type": "fp16", "shape": 10},
        # a small model of odd widths and groups
        {"name": "linear_odd", "kind": "linear", "rows": 5, "width_in": 1000, "width_out": 777, "group": 40, "zeros": True, "base": False,
         "type": "bf16", "shape": 11},
        # the rows of four trees of 16 into the widest layer of a large model
        {"name": "linear_wide", "kind": "linear", "rows": 64, "width_in": 8192, "width_out": 32768, "group": 128, "zeros": True, "base": False,
         "type": "bf16", "shape": 12},
    ]


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    kind = rng.choice(["rotate", "rotate", "verify", "verify", "verify", "linear", "linear", "linear"])
    shape, dtype = rng.randrange(100, 1 << 20), rng.choice(["bf16", "fp16"])
    if kind == "rotate":
        kv_heads, dim = rng.choice([1, 2, 4, 8, 8, 16]), rng.choice([64, 64, 72, 80, 96, 128, 128, 256])
        heads = kv_heads * rng.choice([1, 2, 4, 4, 5])
        most = max(1, min(32773, 32773 * 40 * 128 // ((heads + kv_heads) * dim)))
        return {"kind": kind, "tokens": _log(rng, 1, most), "heads": heads, "kv_heads": kv_heads, "dim": dim,
                "rot": rng.choice([dim, dim, dim // 2, dim // 4 * 2 - 2]), "axes": rng.choice([1, 1, 2, 3]), "far": _log(rng, 64, 1 << 20),
                "neighbours": rng.random() < 0.4, "norm": rng.random() < 0.6, "type": dtype, "shape": shape}
    if kind == "verify":
        requests, vocab = _log(rng, 1, 128), _log(rng, 1000, 131072)
        new = max(1, min(_log(rng, 1, 64), LARGEST_PROBABILITIES // (requests * vocab)))
        return {"kind": kind, "requests": requests, "new_lo": max(1, new // rng.choice([1, 4])), "new_hi": new, "tree": rng.random() < 0.6,
                "drawn": rng.random() < 0.6, "vocab": vocab, "type": rng.choice(["bf16", "fp16", "fp32", "fp32"]), "shape": shape}
    widths = [_log(rng, 256, 16384), _log(rng, 256, 32768)]
    if rng.random() < 0.75:
        widths = [w // 128 * 128 for w in widths]
    while widths[0] * widths[1] > LARGEST_WEIGHTS:
        widths = [w // 2 for w in widths]
    return {"kind": kind, "rows": rng.choice([1, 1, _log(rng, 1, 64), _log(rng, 1, 64)]), "width_in": widths[0], "width_out": widths[1],
            "group": rng.choice([32, 64, 64, 128, 128, 40]), "zeros": rng.random() < 0.5, "base": rng.random() < 0.3, "type": dtype, "shape": shape}


# ---- shapes: functions of the case alone ------------------------------------------------------

def _starts(case):
    rng = random.Random(case["shape"])
    out = [0]
    for _ in range(case["requests"]):
        out.append(out[-1] + rng.randint(case["new_lo"], case["new_hi"]))
    return out


def _parents(case, starts):
    """Of every row the one that it hangs from, counted from its request's first row, which hangs from none."""
    rng = random.Random(case["shape"] + 1)
    out = []
    for a, b in zip(starts, starts[1:]):
        out += [-1] + [rng.randrange(max(0, i - 4), i) if case["tree"] else i - 1 for i in range(1, b - a)]
    return out


def _axes(case):
    """The axis of every pair: sections of about the same size, the first axis' the largest."""
    pairs, axes = case["rot"] // 2, case["axes"]
    return [i * axes // pairs for i in range(pairs)]


def _up(v, a):
    return -(-v // a) * a


# ---- state --------------------------------------------------------------------------------------

class State:
    """What a serving program has in hand: tensors, the pool over one of them, and handles of what lies in the pool."""

    def __init__(self, case, seed):
        self.case = case
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(seed)
        self.pool = None

    def randn(self, *shape, dtype=torch.float32, scale=1.0):
        return (torch.randn(shape, device="cuda", generator=self.gen) * scale).to(dtype)

    def rand(self, *shape):
        return torch.rand(shape, device="cuda", generator=self.gen)

    def randint(self, hi, shape, dtype):
        return torch.randint(hi, shape, device="cuda", generator=self.gen, dtype=dtype)

    def ints(self, values, dtype=torch.int32):
        return torch.tensor(values, dtype=dtype, device="cuda")

    def memory(self, sizes):
        """One device tensor with an allocation of every size; the allocations' offsets."""
        at = [0]
        for n in sizes:
            at.append(at[-1] + _up(n, SLAB))
        self.mem = torch.empty(at[-1], dtype=torch.uint8, device="cuda")
        if own:
            from paper_2411_01830_amd import binding as ft
            self.pool = ft.pool_create(self.mem.data_ptr(), at[-1], SLAB, self.mem.device.index or 0)
            if [ft.slab_alloc(self.pool, n) for n in sizes] != at[:-1]:
                raise RuntimeError("allocations lie elsewhere than expected")
        return at[:-1]

    def __del__(self):
        if self.pool is not None:
            from paper_2411_01830_amd import binding as ft
            ft.pool_destroy(self.pool)


def prepare(case, seed):
    st = State(case, seed)
    {"rotate": _prepare_rotate, "verify": _prepare_verify, "linear": _prepare_linear}[case["kind"]](st, case)
    return st


def _prepare_rotate(st, case):
    dtype, n, dim, rot = TYPES[case["type"]], case["tokens"], case["dim"], case["rot"]
    heads = case["heads"] + 2 * case["kv_heads"]
    # queries, keys and values as a projection gives them: beside each other in a row
    qkv = st.randn(n, heads, dim, dtype=dtype)
    st.q, st.k = qkv[:, :case["heads"]], qkv[:, case["heads"]:case["heads"] + case["kv_heads"]]
    st.positions = st.randint(case["far"], (n, case["axes"]), torch.int32)
    st.axes = _axes(case)
    st.axis = st.ints(st.axes, torch.int64)
    st.freqs = torch.tensor([10000.0 ** (-2 * i / rot) for i in range(rot // 2)], device="cuda")
    st.weights = [(1 + st.randn(dim, scale=0.2)).to(dtype) for _ in range(2)] if case["norm"] else [None, None]
    st.memory([SLAB])
    if own:
        from paper_2411_01830_amd import operators as ops
        st.rotation = ops.Rotation(st.pool, st.freqs, dim, axes=st.axes if case["axes"] > 1 else None, neighbours=case["neighbours"])


def _prepare_verify(st, case):
    dtype, vocab = TYPES[case["type"]], case["vocab"]
    starts = _starts(case)
    parents = _parents(case, starts)
    rows = starts[-1]
    st.starts_host, st.parents_host = starts, parents
    st.starts, st.most = st.ints(starts), max(b - a for a, b in zip(starts, starts[1:]))
    st.parent = st.ints(parents) if case["tree"] else None
    first = st.ints([a for a, b in zip(starts, starts[1:]) for _ in range(b - a)], torch.int64)
    hangs_from = first + st.ints([max(p, 0) for p in parents], torch.int64)
    st.target, st.draft = [torch.empty(rows, vocab, dtype=dtype, device="cuda") for _ in range(2)]
    for a in range(0, rows, 64):  # (of a large vocabulary all rows' logits at once are a lot)
        logits = st.randn(min(64, rows - a), vocab, scale=3.0)
        st.target[a:a + 64] = torch.softmax(logits, -1)
        st.draft[a:a + 64] = torch.softmax(logits + st.randn(*logits.shape, scale=0.7), -1)
    # a row's token was drawn from its parent's draft probabilities, or is one of the likeliest there, another one for each sibling
    rank, siblings = [], {}
    for t, p in enumerate(hangs_from.tolist()):
        rank.append(siblings.get(p, 0) if parents[t] >= 0 else 0)
        siblings[p] = rank[-1] + 1 if parents[t] >= 0 else 0
    tokens = []
    for a in range(0, rows, 64):
        q = st.draft[hangs_from[a:a + 64]].float()
        if case["drawn"]:
            tokens.append((q / torch.empty_like(q).exponential_(generator=st.gen)).argmax(-1))
        else:
            best = q.topk(min(64, vocab), -1).indices
            tokens.append(best.gather(1, st.ints(rank[a:a + 64], torch.int64)[:, None].clamp(max=best.shape[1] - 1))[:, 0])
    st.tokens = torch.cat(tokens)
    if not case["drawn"]:
        st.draft = None
    st.accept, st.pick = st.rand(rows), st.rand(case["requests"])
    st.memory([SLAB])


def _prepare_linear(st, case):
    dtype, ni, no, group = TYPES[case["type"]], case["width_in"], case["width_out"], case["group"]
    groups, row = -(-ni // group), -(-ni // 2)
    at = st.memory([no * row, 2 * no * groups, no * groups])
    st.weights = st.mem[at[0]:at[0] + no * row].view(no, row)
    st.weights.copy_(st.randint(256, (no, row), torch.uint8))
    st.scales = st.mem[at[1]:at[1] + 2 * no * groups].view(dtype).view(no, groups)
    st.scales.copy_((0.5 + st.rand(no, groups)) * (0.2 * ni ** -0.5))
    st.zeros = None
    if case["zeros"]:
        st.zeros = st.mem[at[2]:at[2] + no * groups].view(no, groups)
        st.zeros.copy_(4 + st.randint(9, (no, groups), torch.uint8))
    st.x = st.randn(case["rows"], ni, dtype=dtype)
    st.base = st.randn(case["rows"], no, dtype=dtype) if case["base"] else None
    if own:
        from paper_2411_01830_amd import operators as ops
        st.handle = ops.Linear4(st.pool, at[0], at[1], ni, no, group, dtype, zeros_off=at[2] if case["zeros"] else None)


# ---- one pass -----------------------------------------------------------------------------------

def run(st):
    return (_own if own else _plain)(st)


def _own(st):
    from paper_2411_01830_amd import operators as ops
    kind = st.case["kind"]
    if kind == "rotate":
        q, k = ops.rotate_heads(st.rotation, st.q, st.k, st.positions, q_weight=st.weights[0], k_weight=st.weights[1], eps=EPS if st.case["norm"] else None)
        return {"q": q, "k": k}
    if kind == "verify":
        keep, last, token = ops.tree_verify(st.pool, st.tokens, st.starts, st.most, st.target, st.accept, st.pick, draft=st.draft, parent=st.parent)
        return {"keep": keep, "last": last, "token": token}
    return {"out": ops.linear4_apply(st.handle, st.x, base=st.base)}


def _plain(st):
    return {"rotate": _plain_rotate, "verify": _plain_verify, "linear": _plain_linear}[st.case["kind"]](st)


def _plain_rotate(st):
    case, out = st.case, {}
    rot = case["rot"]
    angle = st.positions[:, st.axis].double() * st.freqs.double()
    c, s = angle.cos().float()[:, None], angle.sin().float()[:, None]
    for name, x, w in (("q", st.q, st.weights[0]), ("k", st.k, st.weights[1])):
        y = x.float()
        if case["norm"]:
            y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * w.float()
        if case["neighbours"]:
            a, b = y[..., 0:rot:2], y[..., 1:rot:2]
            turned = torch.stack([a * c - b * s, a * s + b * c], -1).flatten(-2)
        else:
            a, b = y[..., :rot // 2], y[..., rot // 2:rot]
            turned = torch.cat([a * c - b * s, a * s + b * c], -1)
        out[name] = torch.cat([turned, y[..., rot:]], -1).to(x.dtype)
    return out


def _plain_verify(st):
    """Rows in ascending order, all requests at once. Sums over the vocabulary and what is compared are 64 bits: in 32 a sum of 10^5 numbers
    is off by more than a step from one token to the next."""
    rows, vocab = st.target.shape
    starts = st.starts.long()
    lo, n = starts[:-1], starts[1:] - starts[:-1]
    r = torch.arange(len(lo), device="cuda")
    node = torch.zeros_like(lo)                       # the last row that stands, counted from the first
    keep = torch.zeros(rows, dtype=torch.uint8, device="cuda")
    keep[lo] = 1
    p = st.target[lo].double()                        # what is left of the node's probabilities is max(p - taken q, 0)
    q = torch.zeros_like(p) if st.draft is None else st.draft[lo].double()
    taken, mass = torch.zeros(len(lo), dtype=torch.float64, device="cuda"), torch.ones(len(lo), dtype=torch.float64, device="cuda")
    for j in range(1, st.most):
        t = (lo + j).clamp(max=rows - 1)
        there = j < n
        hangs = there & ((st.parent[t] == node) if st.parent is not None else (node == j - 1))
        token = st.tokens[t]
        left = (p[r, token] - taken * q[r, token]).clamp(min=0)
        u = st.accept[t].double()
        stands = hangs & (u * mass * (q[r, token] if st.draft is not None else 1) < left)
        falls = hangs & ~stands
        if st.draft is None:
            # the token's probability is taken out (a second one of its kind finds nothing)
            mass = torch.where(falls, (mass - left).clamp(min=0), mass)
            p[r, token] = torch.where(falls, 0, p[r, token])
        else:
            taken = torch.where(falls, taken + mass, taken)
            mass = torch.where(falls, (p - taken[:, None] * q).clamp_(min=0).sum(-1), mass)
        keep[t] = torch.where(stands, 1, keep[t])
        node = torch.where(stands, j, node)
        p = torch.where(stands[:, None], st.target[t].double(), p)
        if st.draft is not None:
            q = torch.where(stands[:, None], st.draft[t].double(), q)
        taken, mass = torch.where(stands, 0, taken), torch.where(stands, 1, mass)
    left = (p - taken[:, None] * q).clamp_(min=0)
    left = torch.where(left.sum(-1, keepdim=True) > 0, left, st.target[lo + node].double())
    sums = left.cumsum(-1)
    over = sums > st.pick.double()[:, None] * sums[:, -1:]
    most = torch.where(left > 0, torch.arange(vocab, device="cuda"), -1).amax(-1)
    token = torch.where(over.any(-1), over.to(torch.uint8).argmax(-1), most)
    return {"keep": keep, "last": (lo + node).int(), "token": token}


def _plain_linear(st):
    case = st.case
    w = torch.stack([st.weights & 15, st.weights >> 4], -1).flatten(1)[:, :case["width_in"]].float()
    spread = lambda t: t.float().repeat_interleave(case["group"], 1)[:, :case["width_in"]]  # noqa: E731
    w = (w - (8 if st.zeros is None else spread(st.zeros))) * spread(st.scales)
    y = torch.matmul(st.x.float(), w.t())
    return {"out": (y if st.base is None else y + st.base.float()).to(st.x.dtype)}


# ---- the definitions, in 64 bits ------------------------------------------------------------------

def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "rotate":
        dim, rot, out = case["dim"], case["rot"], {}
        angle = torch.empty(case["tokens"], rot // 2, dtype=torch.float64, device="cuda")
        for i, a in enumerate(st.axes):
            angle[:, i] = st.positions[:, a].double() * float(st.freqs[i])
        turn = torch.polar(torch.ones_like(angle), angle)[:, None]
        for name, x, w in (("q", st.q, st.weights[0]), ("k", st.k, st.weights[1])):
            y = x.double()
            if case["norm"]:
                y = y / (y.square().sum(-1, keepdim=True) / dim + EPS).sqrt() * w.double()
            first = [2 * i if case["neighbours"] else i for i in range(rot // 2)]
            second = [2 * i + 1 if case["neighbours"] else i + rot // 2 for i in range(rot // 2)]
            z = torch.complex(y[..., first], y[..., second]) * turn
            y[..., first], y[..., second] = z.real, z.imag
            out[name] = y
        return out
    if case["kind"] == "verify":
        tokens, accept, pick = st.tokens.tolist(), st.accept.tolist(), st.pick.tolist()
        keep, last, after = [0] * len(tokens), [], []
        for r, (a, b) in enumerate(zip(st.starts_host, st.starts_host[1:])):
            row, keep[a] = a, 1
            while True:
                p = st.target[row].double()
                left, mass = p.clone(), 1.0
                q = st.draft[row].double() if st.draft is not None else None
                found = None
                for t in (t for t in range(row + 1, b) if a + st.parents_host[t] == row):
                    here = float(left[tokens[t]])
                    if accept[t] * mass * (1.0 if q is None else float(q[tokens[t]])) < here:
                        found = t
                        break
                    if q is None:
                        left[tokens[t]] = 0
                        mass = max(mass - here, 0.0)
                    else:
                        # max(max(a - b, 0) - c, 0) = max(a - b - c, 0), so what is left may be cut down again and again
                        left = (left - mass * q).clamp(min=0)
                        mass = float(left.sum())
                if found is None:
                    break
                row, keep[found] = found, 1
            if float(left.sum()) == 0:
                left = p
            sums = left.cumsum(0)
            over = torch.nonzero(sums > pick[r] * float(sums[-1]))[:, 0]
            after.append(int(over[0]) if len(over) else int(torch.nonzero(left > 0)[-1]))
            last.append(row)
        return {"keep": torch.tensor(keep, dtype=torch.uint8), "last": torch.tensor(last, dtype=torch.int32), "token": torch.tensor(after)}
    ni, group = case["width_in"], case["group"]
    want = torch.zeros(case["rows"], case["width_out"], dtype=torch.float64, device="cuda") if st.base is None else st.base.double()
    for g, k in enumerate(range(0, ni, group)):
        at = torch.arange(k, min(k + group, ni), device="cuda")
        codes = ((st.weights[:, at // 2] >> (4 * (at % 2)).to(torch.uint8)) & 15).double()
        zero = 8.0 if st.zeros is None else st.zeros[:, g:g + 1].double()
        want += (st.x[:, at].double() @ (codes - zero).t().contiguous()) * st.scales[:, g].double()
    return {"out": want}


# ---- what a pass cannot do without -----------------------------------------------------------------

def work(case):
    if case["kind"] == "rotate":
        elements = case["tokens"] * (case["heads"] + case["kv_heads"]) * case["dim"]
        return {"bytes": 4 * elements + 4 * case["tokens"] * case["axes"] + 4 * case["dim"] * case["norm"] + 2 * case["rot"],
                "flops": elements * (3 + 4 * case["norm"])}
    if case["kind"] == "verify":
        starts, size = _starts(case), SIZES[case["type"]]
        rows, requests = starts[-1], case["requests"]
        sides = 2 if case["drawn"] else 1
        # one row of probabilities (of either kind) for every request's next token; tokens, flags, random numbers and what they are tested against
        return {"bytes": requests * (case["vocab"] * size * sides + 20) + rows * (13 + (4 if case["tree"] else 0) + size * sides),
                "flops": requests * case["vocab"] * (3 if case["drawn"] else 1)}
    rows, ni, no = case["rows"], case["width_in"], case["width_out"]
    groups = -(-ni // case["group"])
    return {"bytes": no * -(-ni // 2) + no * groups * (3 if case["zeros"] else 2) + 2 * rows * (ni + no * (2 if case["base"] else 1)),
            "flops": 2 * rows * no * ni}
