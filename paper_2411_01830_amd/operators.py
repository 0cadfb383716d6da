"""The operators on memory of the pool, on PyTorch tensors.

A key/value cache and low-rank adapters lie in allocations of a pool (`binding.pool_create`, `binding.slab_alloc`), where
transfers bring and move them; everything else is the caller's tensors. Each call checks what it is given, allocates
its results and its workspace through PyTorch, and queues its kernels on the current stream. What is wrong with the
arguments raises `binding.FtError` with the library's code, before anything is launched.

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


def _need(good, what):
    if not good:
        raise ft.FtError(FT_EINVAL, what)


def _ints(name, t, dtype, dims, device=None):
    """A contiguous tensor of whole numbers on the GPU."""
    _need(isinstance(t, torch.Tensor) and t.is_cuda and t.dtype == dtype and t.dim() == dims and t.is_contiguous(),
          f"{name}: a contiguous {dtype} tensor of {dims} dimensions on the GPU is needed")
    _need(device is None or t.device == device, f"{name} lies on another GPU")


def _rows(name, t, dtype, shape, device):
    """A tensor of elements whose rows are contiguous."""
    _need(isinstance(t, torch.Tensor) and t.is_cuda and t.device == device and t.dtype == dtype, f"{name}: a {dtype} tensor on {device} is needed")
    _need(tuple(t.shape) == tuple(shape), f"{name}: the shape is {tuple(t.shape)}, not {tuple(shape)}")
    _need(t.stride(-1) == 1 or t.shape[-1] == 1 or t.numel() == 0, f"{name}: rows are not contiguous")


def _stream(device):
    return torch.cuda.current_stream(device).cuda_stream


class KvCache:
    """A key/value cache in two allocations of the pool. strides: elements from page to page, token to token, head to head
    (None: pages of tokens of heads, without gaps)."""

    def __init__(self, pool, k_off, v_off, pages, page_tokens, heads, dim, dtype, strides=None):
        _need(dtype in TYPES, f"a cache holds bfloat16 or float16, not {dtype}")
        page, token, head = strides if strides is not None else (page_tokens * heads * dim, heads * dim, dim)
        self.pool, self.dtype, self.heads, self.dim, self.page_tokens = pool, dtype, heads, dim, page_tokens
        self.record = ft.KvCacheRecord(k_off, v_off, TYPES[dtype], pages, page_tokens, heads, dim, 0, page, token, head)


def _tables(lens, table, free, state, page_tokens):
    _ints("lens", lens, torch.int32, 1)
    _ints("table", table, torch.int32, 2, lens.device)
    _ints("free", free, torch.int32, 1, lens.device)
    _ints("state", state, torch.int32, 1, lens.device)
    _need(table.shape[0] == lens.shape[0] and state.shape[0] == 4, "table has a row and state four entries for the requests of lens")
    return ft.KvTables(lens.data_ptr(), table.data_ptr(), free.data_ptr(), state.data_ptr(), lens.shape[0], table.shape[1], free.shape[0], page_tokens)


def kv_grow(pool, lens, starts, tokens, table, free, state, page_tokens, keep=None):
    """Pages and slots of a step's `tokens` rows: (slots, lengths and state after the step); table gets its new entries in place."""
    tables = _tables(lens, table, free, state, page_tokens)
    dev = lens.device
    _ints("starts", starts, torch.int32, 1, dev)
    _need(starts.shape[0] == lens.shape[0] + 1, "starts has one entry more than lens")
    if keep is not None:
        _need(keep.dtype in (torch.uint8, torch.bool), "keep is uint8 or bool")
        _ints("keep", keep, keep.dtype, 1, dev)
        _need(keep.shape[0] == tokens, "keep has an entry for every row")
    slots = torch.empty(tokens, dtype=torch.int64, device=dev)
    lens_out, state_out = torch.empty_like(lens), torch.empty_like(state)
    ft.kv_grow(pool, tables, starts.data_ptr(), keep.data_ptr() if keep is not None else None, tokens, slots.data_ptr(), lens_out.data_ptr(),
               state_out.data_ptr(), _stream(dev))
    return slots, lens_out, state_out


def kv_release(pool, done, lens, table, free, state, page_tokens):
    """The pages of the requests with done != 0 go back on the stack, in place: (lengths, state) after it."""
    tables = _tables(lens, table, free, state, page_tokens)
    _need(done.dtype in (torch.uint8, torch.bool), "done is uint8 or bool")
    _ints("done", done, done.dtype, 1, lens.device)
    _need(done.shape == lens.shape, "done has an entry for every request")
    lens_out, state_out = torch.empty_like(lens), torch.empty_like(state)
    ft.kv_release(pool, tables, done.data_ptr(), lens_out.data_ptr(), state_out.data_ptr(), _stream(lens.device))
    return lens_out, state_out


def kv_append(cache, k, v, slots):
    """cache[slots[t]] = k[t], v[t]; rows with slot -1 are skipped."""
    _ints("slots", slots, torch.int64, 1)
    shape = (slots.shape[0], cache.heads, cache.dim)
    _rows("k", k, cache.dtype, shape, slots.device)
    _rows("v", v, cache.dtype, shape, slots.device)
    ft.kv_append(cache.pool, cache.record, k.data_ptr(), v.data_ptr(), k.stride()[:2], v.stride()[:2], slots.data_ptr(), shape[0], _stream(slots.device))


def tree_attention(cache, q, k, v, starts, lens, table, drafts, mask=None, scale=None, lse=False, out=None):
    """Attention of every request's drafted tokens over its cached ones and, as the mask's bits say (None: up to itself), over each other.

    q: tokens x heads x dim; k, v: tokens x the cache's heads x dim. drafts: the most drafted tokens of one request. mask: int64 or
    uint64, a word of 64 bits a token, or several as a second dimension. scale: dim ** -0.5 by default. With lse also
    log(sum(exp)) of every row, in 32 bits."""
    _need(isinstance(q, torch.Tensor) and q.dim() == 3, "q has three dimensions")
    dev, (tokens, heads, _) = q.device, q.shape
    _rows("q", q, cache.dtype, (tokens, heads, cache.dim), dev)
    _rows("k", k, cache.dtype, (tokens, cache.heads, cache.dim), dev)
    _rows("v", v, cache.dtype, (tokens, cache.heads, cache.dim), dev)
    _ints("starts", starts, torch.int32, 1, dev)
    _ints("lens", lens, torch.int32, 1, dev)
    _ints("table", table, torch.int32, 2, dev)
    requests = lens.shape[0]
    _need(starts.shape[0] == requests + 1 and table.shape[0] == requests, "starts has one entry more than lens, table a row for each")
    words = 0
    if mask is not None:
        _need(mask.dtype in (torch.int64, torch.uint64), "mask has words of 64 bits")
        _ints("mask", mask, mask.dtype, mask.dim(), dev)
        _need(mask.dim() in (1, 2) and mask.shape[0] == tokens, "mask has a row for every token")
        words = mask.shape[1] if mask.dim() == 2 else 1
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
    else:
        _rows("out", out, cache.dtype, q.shape, dev)
    z = torch.empty(tokens, heads, dtype=torch.float32, device=dev) if lse else None
    qs, ks, vs, os = q.stride(), k.stride(), v.stride(), out.stride()
    call = ft.TreeCall(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), z.data_ptr() if lse else None, starts.data_ptr(), lens.data_ptr(),
                       table.data_ptr(), mask.data_ptr() if mask is not None else None, qs[0], qs[1], ks[0], ks[1], vs[0], vs[1], os[0], os[1],
                       requests, tokens, drafts, heads, table.shape[1], words, cache.dim ** -0.5 if scale is None else scale, 0, None, 0)
    need = ft.tree_workspace(cache.pool, cache.record, call)
    if need:
        work = torch.empty(need, dtype=torch.uint8, device=dev)
        call.workspace, call.workspace_bytes = work.data_ptr(), need
    ft.tree_attention(cache.pool, cache.record, call, _stream(dev))
    return (out, z) if lse else out


class Adapters:
    """Low-rank adapters of one projection, in the pool: (offset of A, offset of B, rank, scale) of each. A is rank x width_in,
    B width_out x rank. Holds as long as their allocations do."""

    def __init__(self, pool, adapters, width_in, width_out, dtype, device=None):
        _need(dtype in TYPES, f"adapters hold bfloat16 or float16, not {dtype}")
        _need(len(adapters) > 0, "there are no adapters")
        records = ft.adapters_resolve(pool, [tuple(a) for a in adapters], width_in, width_out)
        self.pool, self.dtype, self.count, self.width_in, self.width_out = pool, dtype, len(adapters), width_in, width_out
        self.max_rank = max(a[2] for a in adapters)
        self.records = torch.frombuffer(bytearray(records), dtype=torch.uint8).to("cuda" if device is None else device)


class AdapterGroups:
    """The rows of a step in the order of their adapters; for any projection of the same adapters."""

    def __init__(self, rows, count, memory):
        self.rows, self.count, self.memory = rows, count, memory


def adapter_groups(adapters, ids):
    """ids: int32, a row's adapter, or anything outside [0, count) for none."""
    _ints("ids", ids, torch.int32, 1)
    need = ft.adapters_group_bytes(ids.shape[0], adapters.count)
    memory = torch.empty(max(need, 16), dtype=torch.uint8, device=ids.device)
    ft.adapters_group(adapters.pool, ids.data_ptr(), ids.shape[0], adapters.count, memory.data_ptr(), need, _stream(ids.device))
    return AdapterGroups(ids.shape[0], adapters.count, memory)


def adapters_apply(adapters, groups, x, base=None, out=None):
    """base (None: 0) and every row's scale * B (A x) on top; out may be base."""
    _need(isinstance(x, torch.Tensor) and x.dim() == 2, "x has two dimensions")
    dev = x.device
    _need(groups.rows == x.shape[0] and groups.count == adapters.count, "the groups are of other rows or adapters")
    _need(adapters.records.device == dev and groups.memory.device == dev, "x lies on another GPU than adapters and groups")
    shape = (groups.rows, adapters.width_out)
    _rows("x", x, adapters.dtype, (groups.rows, adapters.width_in), dev)
    if base is not None:
        _rows("base", base, adapters.dtype, shape, dev)
    if out is None:
        out = torch.empty(shape, dtype=adapters.dtype, device=dev)
    else:
        _rows("out", out, adapters.dtype, shape, dev)
    stride = lambda t: t.stride(0) if t.shape[0] > 1 else t.shape[1]  # noqa: E731  (of one row it means nothing)
    call = ft.AdaptersCall(adapters.records.data_ptr(), groups.memory.data_ptr(), x.data_ptr(), base.data_ptr() if base is not None else None,
                           out.data_ptr(), stride(x), stride(base) if base is not None else 0, stride(out), groups.rows, adapters.count,
                           TYPES[adapters.dtype], adapters.width_in, adapters.width_out, adapters.max_rank, None, 0)
    need = ft.adapters_workspace(adapters.pool, call)
    if need:
        work = torch.empty(need, dtype=torch.uint8, device=dev)
        call.workspace, call.workspace_bytes = work.data_ptr(), need
    ft.adapters_apply(adapters.pool, call, _stream(dev))
    return out


assert C.sizeof(ft.KvCacheRecord) == 64 and C.sizeof(ft.KvTables) == 48 and C.sizeof(ft.TreeCall) == 184 and C.sizeof(ft.AdaptersCall) == 104
