"""The operators on memory of the pool, on PyTorch tensors.

A key/value cache, low-rank adapters and weights of 4 bits lie in allocations of a pool (`binding.pool_create`, `binding.slab_alloc`), where
transfers bring and move them; everything else is the caller's tensors. Each call checks what it is given, allocates
its results and its workspace through PyTorch, and queues its kernels on the current stream of the pool's GPU, where all tensors have to lie. What is wrong with the
arguments raises `binding.FtError` with the library's code, before anything is launched. The operators serve and do not train: inputs
that ask for a gradient are refused, as results would not lead back to them.

One step of a server:

    groups = adapter_groups(adapters, ids)                            # once a step
    qkv = adapters_apply(adapters, groups, x, linear4_apply(w, x))    # beside every projection
    q, k = rotate_heads(rotation, q, k, positions, q_weight, k_weight, eps)
    out = tree_attention(cache, q, k, v, starts, lens, table, drafts, mask)
    keep, last, token = tree_verify(pool, drafted, starts, drafts, target, accept, pick, draft)       # behind the last layer
    slots, lens, state = kv_grow(pool, lens, starts, tokens, table, free, state, page_tokens, keep)   # keep: what was accepted
    kv_append(cache, k, v, slots)                                     # in every layer
"""
import ctypes as C

import torch

from . import binding as ft

FT_EINVAL = -1
TYPES = {torch.bfloat16: 0, torch.float16: 1}
PROBABILITIES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}


def _refuse(what):
    raise ft.FtError(FT_EINVAL, what)


def _ints(name, t, dtype, dims, device):
    """A contiguous tensor of whole numbers on the GPU. (What is wrong is put into words only when something is: these calls are made in
    loops that wait for them.)"""
    if isinstance(t, torch.Tensor) and t.dtype is dtype and t.device == device and t.dim() == dims and t.is_contiguous():
        return
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype is dtype and t.dim() == dims and t.is_contiguous()):
        _refuse(f"{name}: a contiguous {dtype} tensor of {dims} dimensions on the GPU is needed")
    if t.device != device:
        _refuse(f"{name} lies on another GPU")


def _rows(name, t, dtype, shape, device):
    """A tensor of elements whose rows are contiguous."""
    if isinstance(t, torch.Tensor) and t.dtype is dtype and t.device == device and t.shape == shape and t.stride(-1) == 1 and not t.requires_grad:
        return
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype is dtype and t.device == device):
        _refuse(f"{name}: a {dtype} tensor on {device} is needed")
    if t.shape != shape:
        _refuse(f"{name}: the shape is {tuple(t.shape)}, not {tuple(shape)}")
    if t.stride(-1) != 1 and t.shape[-1] != 1 and t.numel() != 0:
        _refuse(f"{name}: rows are not contiguous")
    if t.requires_grad and torch.is_grad_enabled():
        _refuse(f"{name} asks for a gradient, and there is none (under torch.no_grad it is not asked for)")


def _device(name, t, pool):
    """The GPU that a call's tensors have to lie on, which is the pool's."""
    if not (isinstance(t, torch.Tensor) and t.is_cuda):
        _refuse(f"{name}: a tensor on the GPU is needed")
    dev = t.device
    if dev.index != getattr(pool, "device", dev.index):  # (a handle from elsewhere than pool_create does not know)
        _refuse(f"{name} lies on {dev}, the pool on GPU {pool.device}")
    return dev


def _tensor(name, t):
    """Ahead of looking at what a tensor is like."""
    if not isinstance(t, torch.Tensor):
        _refuse(f"{name}: a tensor on the GPU is needed")


def _flags(name, t, device, n):
    _tensor(name, t)
    if t.dtype is not torch.uint8 and t.dtype is not torch.bool:
        _refuse(f"{name} is uint8 or bool")
    _ints(name, t, t.dtype, 1, device)
    if t.shape[0] != n:
        _refuse(f"{name} has {n} entries")


_linear4, _rotate, _verify = ft.LINEAR4_CALL.pack, ft.ROTATE_CALL.pack, ft.VERIFY_CALL.pack
_stream = torch._C._cuda_getCurrentRawStream  # of a device's index: torch.cuda.current_stream without the object that holds it


class KvCache:
    """A key/value cache in two allocations of the pool. strides: elements from page to page, token to token, head to head
    (None: pages of tokens of heads, without gaps)."""

    def __init__(self, pool, k_off, v_off, pages, page_tokens, heads, dim, dtype, strides=None):
        if dtype not in TYPES:
            _refuse(f"a cache holds bfloat16 or float16, not {dtype}")
        page, token, head = strides if strides is not None else (page_tokens * heads * dim, heads * dim, dim)
        self.pool, self.dtype, self.heads, self.dim, self.page_tokens = pool, dtype, heads, dim, page_tokens
        self.record = ft.KvCacheRecord(k_off, v_off, TYPES[dtype], pages, page_tokens, heads, dim, 0, page, token, head)


def _tables(pool, lens, table, free, state, page_tokens):
    dev = _device("lens", lens, pool)
    _ints("lens", lens, torch.int32, 1, dev)
    _ints("table", table, torch.int32, 2, dev)
    _ints("free", free, torch.int32, 1, dev)
    _ints("state", state, torch.int32, 1, dev)
    requests, (rows, blocks) = lens.shape[0], table.shape
    if rows != requests or state.shape[0] != 4:
        _refuse("table has a row and state four entries for the requests of lens")
    return dev, ft.KvTables(lens.data_ptr(), table.data_ptr(), free.data_ptr(), state.data_ptr(), requests, blocks, free.shape[0], page_tokens)


def kv_grow(pool, lens, starts, tokens, table, free, state, page_tokens, keep=None):
    """Pages and slots of a step's `tokens` rows: (slots, lengths and state after the step); table gets its new entries in place."""
    dev, tables = _tables(pool, lens, table, free, state, page_tokens)
    _ints("starts", starts, torch.int32, 1, dev)
    if starts.shape[0] != tables.requests + 1:
        _refuse("starts has one entry more than lens")
    if keep is not None:
        _flags("keep", keep, dev, tokens)
    slots = torch.empty(tokens, dtype=torch.int64, device=dev)
    lens_out, state_out = torch.empty_like(lens), torch.empty_like(state)
    ft.kv_grow(pool, tables, starts.data_ptr(), None if keep is None else keep.data_ptr(), tokens, slots.data_ptr(), lens_out.data_ptr(),
               state_out.data_ptr(), _stream(dev.index))
    return slots, lens_out, state_out


def kv_release(pool, done, lens, table, free, state, page_tokens):
    """The pages of the requests with done != 0 go back on the stack, in place: (lengths, state) after it."""
    dev, tables = _tables(pool, lens, table, free, state, page_tokens)
    _flags("done", done, dev, tables.requests)
    lens_out, state_out = torch.empty_like(lens), torch.empty_like(state)
    ft.kv_release(pool, tables, done.data_ptr(), lens_out.data_ptr(), state_out.data_ptr(), _stream(dev.index))
    return lens_out, state_out


def kv_append(cache, k, v, slots):
    """cache[slots[t]] = k[t], v[t]; rows with slot -1 are skipped."""
    dev = _device("slots", slots, cache.pool)
    _ints("slots", slots, torch.int64, 1, dev)
    shape = (slots.shape[0], cache.heads, cache.dim)
    _rows("k", k, cache.dtype, shape, dev)
    _rows("v", v, cache.dtype, shape, dev)
    ft.kv_append(cache.pool, cache.record, k.data_ptr(), v.data_ptr(), k.stride()[:2], v.stride()[:2], slots.data_ptr(), shape[0], _stream(dev.index))


def tree_attention(cache, q, k, v, starts, lens, table, drafts, mask=None, scale=None, lse=False, out=None):
    """Attention of every request's drafted tokens over its cached ones and, as the mask's bits say (None: up to itself), over each other.

    q: tokens x heads x dim; k, v: tokens x the cache's heads x dim. drafts: the most drafted tokens of one request. mask: int64 or
    uint64, a word of 64 bits a token, or several as a second dimension. scale: dim ** -0.5 by default. With lse also
    log(sum(exp)) of every row, in 32 bits. Rows of no request (a padded step has them) and those beyond `drafts` are not written: in `out` they
    stay as they were, in results that are made here they hold anything."""
    dev = _device("q", q, cache.pool)
    if q.dim() != 3:
        _refuse("q has three dimensions")
    shape, dtype, dim = q.shape, cache.dtype, cache.dim
    tokens, heads, _ = shape
    _rows("q", q, dtype, (tokens, heads, dim), dev)
    _rows("k", k, dtype, (tokens, cache.heads, dim), dev)
    _rows("v", v, dtype, (tokens, cache.heads, dim), dev)
    _ints("starts", starts, torch.int32, 1, dev)
    _ints("lens", lens, torch.int32, 1, dev)
    _ints("table", table, torch.int32, 2, dev)
    requests, (rows, blocks) = lens.shape[0], table.shape
    if starts.shape[0] != requests + 1 or rows != requests:
        _refuse("starts has one entry more than lens, table a row for each")
    words, mask_at = 0, None
    if mask is not None:
        _tensor("mask", mask)
        if mask.dtype is not torch.int64 and mask.dtype is not torch.uint64:
            _refuse("mask has words of 64 bits")
        dims = mask.dim()
        _ints("mask", mask, mask.dtype, dims, dev)
        if dims not in (1, 2) or mask.shape[0] != tokens:
            _refuse("mask has a row for every token")
        words, mask_at = mask.shape[1] if dims == 2 else 1, mask.data_ptr()
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
    else:
        _rows("out", out, dtype, shape, dev)
    z = torch.empty(tokens, heads, dtype=torch.float32, device=dev) if lse else None
    qs, ks, vs, os = q.stride(), k.stride(), v.stride(), out.stride()
    call = ft.TreeCall(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), z.data_ptr() if lse else None, starts.data_ptr(), lens.data_ptr(),
                       table.data_ptr(), mask_at, qs[0], qs[1], ks[0], ks[1], vs[0], vs[1], os[0], os[1],
                       requests, tokens, drafts, heads, blocks, words, dim ** -0.5 if scale is None else scale, 0, None, 0)
    need = ft.tree_workspace(cache.pool, cache.record, call)
    if need:
        work = torch.empty(need, dtype=torch.uint8, device=dev)
        call.workspace, call.workspace_bytes = work.data_ptr(), need
    ft.tree_attention(cache.pool, cache.record, call, _stream(dev.index))
    return (out, z) if lse else out


class Adapters:
    """Low-rank adapters of one projection, in the pool: (offset of A, offset of B, rank, scale) of each. A is rank x width_in,
    B width_out x rank. Holds as long as their allocations do."""

    def __init__(self, pool, adapters, width_in, width_out, dtype, device=None):
        if dtype not in TYPES:
            _refuse(f"adapters hold bfloat16 or float16, not {dtype}")
        if len(adapters) == 0:
            _refuse("there are no adapters")
        on = torch.device("cuda", getattr(pool, "device", 0)) if device is None else torch.device(device)
        if on.index not in (None, getattr(pool, "device", on.index)):
            _refuse(f"the pool lies on GPU {pool.device}, not on {on}")
        records = ft.adapters_resolve(pool, [tuple(a) for a in adapters], width_in, width_out)
        self.pool, self.dtype, self.count, self.width_in, self.width_out = pool, dtype, len(adapters), width_in, width_out
        self.max_rank = max(a[2] for a in adapters)
        self.records = torch.frombuffer(bytearray(records), dtype=torch.uint8).to(on)


class AdapterGroups:
    """The rows of a step in the order of their adapters; for any projection of the same adapters. `memory` is of the stream that they were
    made on: another stream's calls wait for it, and memory.record_stream says so, as for any tensor."""

    def __init__(self, rows, count, memory):
        self.rows, self.count, self.memory = rows, count, memory


def adapter_groups(adapters, ids):
    """ids: int32, a row's adapter, or anything outside [0, count) for none."""
    dev = _device("ids", ids, adapters.pool)
    _ints("ids", ids, torch.int32, 1, dev)
    rows = ids.shape[0]
    need = ft.adapters_group_bytes(rows, adapters.count)
    memory = torch.empty(need, dtype=torch.uint8, device=dev)
    ft.adapters_group(adapters.pool, ids.data_ptr(), rows, adapters.count, memory.data_ptr(), need, _stream(dev.index))
    return AdapterGroups(rows, adapters.count, memory)


def adapters_apply(adapters, groups, x, base=None, out=None):
    """base (None: 0) and every row's scale * B (A x) on top; out may be base."""
    dev = _device("x", x, adapters.pool)
    rows, dtype, records, memory = groups.rows, adapters.dtype, adapters.records, groups.memory
    if x.dim() != 2 or x.shape[0] != rows or groups.count != adapters.count:
        _refuse("the groups are of other rows or adapters")
    if records.device != dev or memory.device != dev:
        _refuse("x lies on another GPU than adapters and groups")
    shape = (rows, adapters.width_out)
    _rows("x", x, dtype, (rows, adapters.width_in), dev)
    if base is not None:
        _rows("base", base, dtype, shape, dev)
    if out is None:
        out = torch.empty(shape, dtype=dtype, device=dev)
    else:
        _rows("out", out, dtype, shape, dev)
    one = rows <= 1  # a single row's stride means nothing
    call = ft.AdaptersCall(records.data_ptr(), memory.data_ptr(), x.data_ptr(), None if base is None else base.data_ptr(), out.data_ptr(),
                           adapters.width_in if one else x.stride(0), adapters.width_out if one or base is None else base.stride(0),
                           adapters.width_out if one else out.stride(0), rows, adapters.count, TYPES[dtype], adapters.width_in, adapters.width_out,
                           adapters.max_rank, None, 0)
    need = ft.adapters_workspace(adapters.pool, call)
    if need:
        work = torch.empty(need, dtype=torch.uint8, device=dev)
        call.workspace, call.workspace_bytes = work.data_ptr(), need
    ft.adapters_apply(adapters.pool, call, _stream(dev.index))
    return out



class Linear4:
    """A projection's weights in the pool, in 4 bits: codes two to a byte (an even element's in the low half), width_out rows of
    (width_in + 1) // 2 bytes; a scale of `dtype` for each group of neighbouring elements of a row, width_out x ceil(width_in / group);
    zeros likewise, a byte each (None: 8 everywhere). A weight is scale * (code - zero). Holds as long as the allocations do."""

    def __init__(self, pool, weights_off, scales_off, width_in, width_out, group, dtype, zeros_off=None):
        if dtype not in TYPES:
            _refuse(f"scales are bfloat16 or float16, not {dtype}")
        self.pool, self.dtype, self.width_in, self.width_out = pool, dtype, width_in, width_out
        self.record = ft.Linear4Record(weights_off, scales_off, ft.NO_ZEROS if zeros_off is None else zeros_off, TYPES[dtype], width_in, width_out, group)


def linear4_apply(weights, x, base=None, out=None):
    """base (None: 0) and x's rows times the weights on top; out may be base. For the few rows of a step: weights are read once for 16 to 64 of them
    (for 8 in groups below 32 elements, or more than 1024 of them to a row)."""
    pool, dtype, ni, no = weights.pool, weights.dtype, weights.width_in, weights.width_out
    dev = _device("x", x, pool)
    given = x.shape
    if len(given) != 2:
        _refuse("x has two dimensions")
    rows = given[0]
    _rows("x", x, dtype, (rows, ni), dev)
    shape = (rows, no)
    if out is None:
        out = x.new_empty(shape)
    else:
        _rows("out", out, dtype, shape, dev)
    base_at, base_stride, x_stride, out_stride = 0, no, ni, no
    if base is not None:
        _rows("base", base, dtype, shape, dev)
        base_at = base.data_ptr()
    if rows > 1:  # (a single row's stride means nothing)
        x_stride, out_stride = x.stride()[0], out.stride()[0]
        if base is not None:
            base_stride = base.stride()[0]
    x_at, out_at = x.data_ptr(), out.data_ptr()
    call = _linear4(x_at, base_at, out_at, x_stride, base_stride, out_stride, rows, 0, 0, 0)
    need = ft.linear4_workspace(pool, weights.record, call)
    if need:
        work = torch.empty(need, dtype=torch.uint8, device=dev)
        call = _linear4(x_at, base_at, out_at, x_stride, base_stride, out_stride, rows, 0, work.data_ptr(), need)
    ft.linear4_apply(pool, weights.record, call, _stream(dev.index))
    return out


class Rotation:
    """How positions turn the pairs of heads of `dim` elements: freqs are radians a position, one for each of the pairs (elements behind the first
    2 * len(freqs) are not turned); axes names the axis of each pair (None: there is one axis); neighbours: pairs are elements 2i and 2i + 1,
    without it i and i + len(freqs). It keeps copies of both, of the stream that it was made on: another stream's calls wait for it."""

    def __init__(self, pool, freqs, dim, axes=None, neighbours=False):
        on = torch.device("cuda", getattr(pool, "device", 0))
        self.pool, self.dim, self.neighbours = pool, dim, neighbours
        pairs = len(freqs)
        if 2 * pairs > dim:
            _refuse(f"{pairs} pairs are more than a head of {dim} elements has")
        if isinstance(freqs, torch.Tensor) and freqs.requires_grad:
            _refuse("freqs asks for a gradient, which a rotation does not give")
        self.axis, self.axes = None, 1
        if axes is not None:
            axes = [int(a) for a in axes]
            if len(axes) != pairs or any(a < 0 or a > 255 for a in axes):
                _refuse("axes has a number from 0 to 255 for every pair")
            self.axes = max(axes, default=0) + 1
            self.axis = torch.tensor(axes, dtype=torch.uint8).to(on)
        self.freqs = torch.as_tensor(freqs, dtype=torch.float32).to(on, copy=True).contiguous()  # (its own, whatever becomes of the caller's)
        if self.freqs.dim() != 1:
            _refuse("freqs has one dimension")
        self.rot, self.axis_at = 2 * pairs, 0 if self.axis is None else self.axis.data_ptr()


def rotate_heads(rotation, q, k, positions, q_weight=None, k_weight=None, eps=None, q_out=None, k_out=None):
    """Queries and keys (None: queries alone) with their heads turned by the tokens' positions: (queries, keys). With eps every head is divided by
    the root of the mean of its squares before, and multiplied by the weights (None: ones).

    q: tokens x heads x dim; k: tokens x its heads x dim. positions: int32, tokens, or tokens x axes where there are several. q_out and k_out may
    be q and k."""
    pool, dim, freqs = rotation.pool, rotation.dim, rotation.freqs
    dev = _device("q", q, pool)
    dtype, shape = q.dtype, q.shape
    if len(shape) != 3 or dtype not in TYPES:
        _refuse("q has three dimensions of bfloat16 or float16")
    tokens, heads, _ = shape
    _rows("q", q, dtype, (tokens, heads, dim), dev)
    _tensor("positions", positions)
    at = positions.shape
    _ints("positions", positions, torch.int32, len(at), dev)
    axes = at[1] if len(at) == 2 else 1
    if len(at) not in (1, 2) or at[0] != tokens or axes < rotation.axes:
        _refuse("positions has a row for every token, and a column for every axis")
    if freqs.device != dev:
        _refuse("q lies on another GPU than the rotation")
    flags = ft.ROTATE_NEIGHBOURS if rotation.neighbours else 0
    q_by = k_by = 0
    if eps is not None:
        if not 0 <= eps < 3e38:
            _refuse("eps is a number of 32 bits, not below 0")
        flags |= ft.ROTATE_NORM
        if q_weight is not None:
            _rows("q_weight", q_weight, dtype, (dim,), dev)
            q_by = q_weight.data_ptr()
        if k_weight is not None:
            _rows("k_weight", k_weight, dtype, (dim,), dev)
            k_by = k_weight.data_ptr()
    elif q_weight is not None or k_weight is not None:
        _refuse("weights belong to a norm, which asks for eps")
    else:
        eps = 0.0
    if q_out is None:
        q_out = torch.empty_like(q, memory_format=torch.contiguous_format)
    else:
        _rows("q_out", q_out, dtype, shape, dev)
    qs, os = q.stride(), q_out.stride()
    k_at, k_to, kv_heads, ks, kos = 0, 0, 0, (0, 0), (0, 0)
    if k is not None:
        _tensor("k", k)
        given = k.shape
        if len(given) != 3:
            _refuse("k has three dimensions")
        kv_heads = given[1]
        _rows("k", k, dtype, (tokens, kv_heads, dim), dev)
        if k_out is None:
            k_out = torch.empty_like(k, memory_format=torch.contiguous_format)
        else:
            _rows("k_out", k_out, dtype, k.shape, dev)
        k_at, k_to, ks, kos = k.data_ptr(), k_out.data_ptr(), k.stride(), k_out.stride()
    elif k_out is not None:
        _refuse("there are no keys for k_out")
    call = _rotate(q.data_ptr(), k_at, q_out.data_ptr(), k_to, q_by, k_by, positions.data_ptr(), freqs.data_ptr(), rotation.axis_at, qs[0], qs[1], ks[0],
                   ks[1], os[0], os[1], kos[0], kos[1], tokens, heads, kv_heads, dim, rotation.rot, axes, TYPES[dtype], flags, eps, 0)
    ft.rotate_heads(pool, call, _stream(dev.index))
    return q_out, k_out


def tree_verify(pool, tokens, starts, drafts, target, accept, pick, draft=None, parent=None):
    """Judges every request's drafted tokens: (keep, last, token) - flags of the rows that stand, as kv_grow takes them, and of every request
    the last of these and the token behind it, -1 where there is none.

    tokens: int64, a row's token. Rows [starts[r], starts[r + 1]) are request r's, the first of them known, `drafts` the most of one. parent: int32,
    the row that a row hangs from, counted from its request's first (None: the row before). target: rows x vocabulary, the model's probabilities behind
    each row; draft: those that the rows which hang from a row were drawn by (None: they were not drawn, but chosen otherwise). accept and
    pick: float32 random numbers from [0, 1), one a row and one a request."""
    dev = _device("tokens", tokens, pool)
    _ints("tokens", tokens, torch.int64, 1, dev)
    _ints("starts", starts, torch.int32, 1, dev)
    rows, requests = tokens.shape[0], starts.shape[0] - 1
    if requests < 0:
        _refuse("starts has one entry more than there are requests")
    if not 0 < drafts < 1 << 32:
        _refuse("drafts is the most rows of a request")
    _ints("accept", accept, torch.float32, 1, dev)
    _ints("pick", pick, torch.float32, 1, dev)
    if accept.shape[0] != rows or pick.shape[0] != requests:
        _refuse("accept has an entry for every row, pick for every request")
    _tensor("target", target)
    shape, dtype = target.shape, target.dtype
    if len(shape) != 2 or dtype not in PROBABILITIES:
        _refuse("target has two dimensions of bfloat16, float16 or float32")
    vocab = shape[1]
    _rows("target", target, dtype, (rows, vocab), dev)
    if draft is not None:
        _rows("draft", draft, dtype, (rows, vocab), dev)
    if parent is not None:
        _ints("parent", parent, torch.int32, 1, dev)
        if parent.shape[0] != rows:
            _refuse("parent has an entry for every row")
    keep, last, token = torch.empty(rows, dtype=torch.uint8, device=dev), starts.new_empty(requests), tokens.new_empty(requests)
    one = rows <= 1
    at = (tokens.data_ptr(), starts.data_ptr(), 0 if parent is None else parent.data_ptr(), target.data_ptr(), 0 if draft is None else draft.data_ptr(),
          accept.data_ptr(), pick.data_ptr(), keep.data_ptr(), last.data_ptr(), token.data_ptr(), vocab if one else target.stride()[0],
          vocab if one or draft is None else draft.stride()[0], rows, requests, drafts, vocab, PROBABILITIES[dtype], 0)
    call = _verify(*at, 0, 0)
    need = ft.verify_workspace(pool, call)
    if need:
        work = torch.empty(need, dtype=torch.uint8, device=dev)
        call = _verify(*at, work.data_ptr(), need)
    ft.tree_verify(pool, call, _stream(dev.index))
    return keep, last, token


assert C.sizeof(ft.KvCacheRecord) == 64 and C.sizeof(ft.KvTables) == 48 and C.sizeof(ft.TreeCall) == 184 and C.sizeof(ft.AdaptersCall) == 104
assert C.sizeof(ft.Linear4Record) == 40 and C.sizeof(ft.Linear4Call) == 72 and C.sizeof(ft.RotateCall) == 176 and C.sizeof(ft.VerifyCall) == 136
