"""The operators on memory of the pool, on PyTorch tensors.

A key/value cache and low-rank adapters lie in allocations of a pool (`binding.pool_create`, `binding.slab_alloc`), where
transfers bring and move them; everything else is the caller's tensors. Each call checks what it is given, allocates
its results and its workspace through PyTorch, and queues its kernels on the current stream of the pool's GPU, where all tensors have to lie. What is wrong with the
arguments raises `binding.FtError` with the library's code, before anything is launched. The operators serve and do not train: inputs
that ask for a gradient are refused, as results would not lead back to them.

One step of a server:

    groups = adapter_groups(adapters, ids)                            # once a step
    qkv = adapters_apply(adapters, groups, x, x @ w.t())              # beside every projection
    out = tree_attention(cache, q, k, v, starts, lens, table, drafts, mask)
    slots, lens, state = kv_grow(pool, lens, starts, tokens, table, free, state, page_tokens, keep)   # keep: what was accepted
    kv_append(cache, k, v, slots)                                     # in every layer
"""
import ctypes as C

import torch

from . import binding as ft

FT_EINVAL = -1
TYPES = {torch.bfloat16: 0, torch.float16: 1}


def _refuse(what):
    raise ft.FtError(FT_EINVAL, what)


def _ints(name, t, dtype, dims, device):
    """A contiguous tensor of whole numbers on the GPU. (What is wrong is put into words only when something is: these calls are made in
    loops that wait for them.)"""
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype is dtype and t.dim() == dims and t.is_contiguous()):
        _refuse(f"{name}: a contiguous {dtype} tensor of {dims} dimensions on the GPU is needed")
    if t.device != device:
        _refuse(f"{name} lies on another GPU")


def _rows(name, t, dtype, shape, device):
    """A tensor of elements whose rows are contiguous."""
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


def _flags(name, t, device, n):
    if t.dtype is not torch.uint8 and t.dtype is not torch.bool:
        _refuse(f"{name} is uint8 or bool")
    _ints(name, t, t.dtype, 1, device)
    if t.shape[0] != n:
        _refuse(f"{name} has {n} entries")


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


assert C.sizeof(ft.KvCacheRecord) == 64 and C.sizeof(ft.KvTables) == 48 and C.sizeof(ft.TreeCall) == 184 and C.sizeof(ft.AdaptersCall) == 104
