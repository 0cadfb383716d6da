"""What the operators on pool memory refuse: checked before anything reaches a device, so without one."""
import ctypes as C
import math
import os

import pytest

from paper_2411_01830_amd import binding as ft

BASE = 0x7F0000000000          # never dereferenced
MiB = 1 << 20
EINVAL, ERANGE = -1, -3


@pytest.fixture()
def pool():
    p = ft.pool_create(BASE, 64 * MiB, 4096, 0)
    yield p
    ft.pool_destroy(p)


def code(call, *args):
    try:
        call(*args)
    except ft.FtError as e:
        return e.code
    return 0


def cache(pool, **other):
    given = dict(k=ft.slab_alloc(pool, MiB), v=ft.slab_alloc(pool, MiB), type=0, pages=32, page_tokens=16, heads=8, dim=128, _pad=0,
                 page_stride=16 * 8 * 128, token_stride=8 * 128, head_stride=128)
    given.update(other)
    return ft.KvCacheRecord(*[given[n] for n, _ in ft.KvCacheRecord._fields_])


def call(**other):
    given = {n: BASE for n in ("q", "k", "v", "out", "lse", "starts", "lens", "table", "mask")}
    given.update({n: 128 for n, _ in ft.TreeCall._fields_ if n.endswith("stride")})
    given.update(requests=2, tokens=8, drafts=4, heads=32, blocks=4, mask_words=1, scale=0.1, _pad=0, workspace=BASE, workspace_bytes=0)
    given.update(other)
    return ft.TreeCall(*[given[n] for n, _ in ft.TreeCall._fields_])


def test_records_have_the_headers_layout(tmp_path):
    import shutil
    import subprocess
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("no C compiler")
    both = [("ft_kv_cache", ft.KvCacheRecord), ("ft_kv_tables", ft.KvTables), ("ft_tree_call", ft.TreeCall), ("ft_adapter", ft.AdapterRecord),
            ("ft_adapter_record", ft.AdapterRecord), ("ft_adapters_call", ft.AdaptersCall)]
    src = ["#include <stddef.h>", "#include <stdio.h>", '#include "faastube.h"', "int main(void) {"]
    want = []
    for name, rec in both:
        src.append(f'  printf("{name} %zu\\n", sizeof({name}));')
        want.append(f"{name} {C.sizeof(rec)}")
        for field, _ in rec._fields_:
            src.append(f'  printf("{name}.{field} %zu\\n", offsetof({name}, {field}));')
            want.append(f"{name}.{field} {getattr(rec, field).offset}")
    (tmp_path / "t.c").write_text("\n".join(src + ["  return 0;", "}"]))
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    subprocess.run([gcc, "-std=c99", "-Wall", "-Werror", "-I", os.path.join(root, "include"), str(tmp_path / "t.c"), "-o", str(tmp_path / "t")], check=True)
    assert subprocess.run([str(tmp_path / "t")], capture_output=True, text=True, check=True).stdout.split("\n")[:-1] == want


BAD_CACHES = [dict(type=2), dict(pages=0), dict(page_tokens=0), dict(heads=0), dict(dim=0), dict(dim=4), dict(dim=130), dict(dim=264), dict(k=1), dict(v=4097),
              dict(pages=1 << 16, page_tokens=1 << 15), dict(page_stride=127), dict(token_stride=0), dict(head_stride=120), dict(page_stride=1 << 40)]
FAR_CACHES = [dict(pages=33), dict(page_stride=16 * 8 * 128 + 1), dict(k=64 * MiB), dict(v=1 << 62), dict(page_stride=(1 << 40) - 1)]


@pytest.mark.parametrize("other", BAD_CACHES + FAR_CACHES, ids=str)
def test_caches_that_are_refused(pool, other):
    c = cache(pool, **other)
    want = EINVAL if other in BAD_CACHES else ERANGE
    assert code(ft.kv_append, pool, c, BASE, BASE, (128, 128), (128, 128), BASE, 4) == want
    assert code(ft.kv_append, pool, c, None, None, (128, 128), (128, 128), None, 0) == want
    assert code(ft.tree_attention, pool, c, call(tokens=0)) == want
    if want == EINVAL:
        assert code(ft.tree_attention, pool, c, call()) == want
        assert code(ft.tree_workspace, pool, c, call()) == want


def test_a_cache_whose_allocation_is_gone_is_refused(pool):
    c = cache(pool)
    assert code(ft.kv_append, pool, c, None, None, (0, 0), (0, 0), None, 0) == 0
    ft.slab_free(pool, c.v)
    assert code(ft.kv_append, pool, c, None, None, (0, 0), (0, 0), None, 0) == ERANGE


@pytest.mark.parametrize("args", [(None, BASE, BASE), (BASE, None, BASE), (BASE, BASE, None), (BASE + 1, BASE, BASE), (BASE, BASE, BASE + 4)], ids=str)
def test_appends_that_are_refused(pool, args):
    k, v, slots = args
    assert code(ft.kv_append, pool, cache(pool), k, v, (128, 128), (128, 128), slots, 4) == EINVAL


def test_appends_of_strides_and_counts_that_are_refused(pool):
    c = cache(pool)
    assert code(ft.kv_append, pool, c, BASE, BASE, (1 << 40, 128), (128, 128), BASE, 4) == EINVAL
    assert code(ft.kv_append, pool, c, BASE, BASE, (128, 128), (128, 128), BASE, 1 << 31) == EINVAL


@pytest.mark.parametrize("other", [
    dict(q=None), dict(k=None), dict(v=None), dict(out=None), dict(starts=None), dict(lens=None), dict(table=None), dict(q=BASE + 1), dict(out=BASE + 1),
    dict(lse=BASE + 2), dict(mask=BASE + 4), dict(starts=BASE + 1), dict(lens=BASE + 2), dict(table=BASE + 1), dict(drafts=0), dict(drafts=65),
    dict(mask_words=0), dict(heads=0), dict(heads=12), dict(heads=1 << 17), dict(scale=math.inf), dict(scale=math.nan), dict(tokens=1 << 31),
    dict(requests=(1 << 24) + 1), dict(q_token_stride=1 << 40), dict(v_head_stride=1 << 50)], ids=str)
def test_attention_calls_that_are_refused(pool, other):
    assert code(ft.tree_attention, pool, cache(pool), call(**other)) == EINVAL


def test_scales_that_powers_of_two_do_not_hold_are_refused(pool):
    c = cache(pool)
    for scale in (2.4e38, -3e38):
        assert code(ft.tree_attention, pool, c, call(scale=scale)) == EINVAL
        assert code(ft.tree_workspace, pool, c, call(scale=scale)) == EINVAL
    assert code(ft.tree_workspace, pool, c, call(scale=-2.3e38)) != EINVAL


def test_calls_of_more_workgroups_than_a_grid_holds_are_refused(pool):
    """The second launch has 256 threads for every request's key head, and a grid less than 2^32: refused before the first launch."""
    c = cache(pool)
    assert code(ft.tree_attention, pool, c, call(requests=1 << 21)) == EINVAL
    assert code(ft.tree_workspace, pool, c, call(requests=1 << 21)) == EINVAL
    assert code(ft.tree_workspace, pool, c, call(requests=(1 << 21) - 1)) != EINVAL
    assert code(ft.tree_workspace, pool, c, call(heads=8, tokens=1 << 20, drafts=1 << 20)) == EINVAL
    assert code(ft.tree_workspace, pool, c, call(heads=8, tokens=1 << 20, drafts=(1 << 20) - 1)) != EINVAL
    for rows, want in (((1 << 30) - 384, 0), ((1 << 30) - 320, EINVAL), (1 << 30, EINVAL)):      # 64 rows of one adapter a workgroup
        assert code(ft.adapters_workspace, pool, adapters_call(rows=rows)) == want, rows
        if want != 0:
            assert code(ft.adapters_apply, pool, adapters_call(rows=rows, workspace_bytes=1 << 62)) == want, rows


def test_nothing_to_attend_is_nothing_wrong(pool):
    c = cache(pool)
    for other in (dict(tokens=0), dict(requests=0)):
        empty = {n: None for n in ("q", "k", "v", "out", "lse", "starts", "lens", "table", "mask")}
        assert code(ft.tree_attention, pool, c, call(**empty, **other)) == 0
        assert ft.tree_workspace(pool, c, call(**other)) == 0


def tables(**other):
    given = dict(lens=BASE, table=BASE, free_pages=BASE, state=BASE, requests=4, blocks=8, pages=100, page_tokens=16)
    given.update(other)
    return ft.KvTables(*[given[n] for n, _ in ft.KvTables._fields_])


@pytest.mark.parametrize("other", [dict(lens=None), dict(table=None), dict(free_pages=None), dict(state=None), dict(lens=BASE + 2), dict(blocks=0),
                                   dict(pages=0), dict(page_tokens=0), dict(pages=1 << 27, page_tokens=16), dict(requests=1 << 24)], ids=str)
def test_tables_that_are_refused(pool, other):
    t = tables(**other)
    assert code(ft.kv_grow, pool, t, BASE, None, 4, BASE, BASE + 64, BASE + 64) == EINVAL
    assert code(ft.kv_release, pool, t, BASE, BASE + 64, BASE + 64) == EINVAL


def test_steps_that_are_refused(pool):
    t = tables()
    good = [pool, t, BASE, None, 4, BASE, BASE + 64, BASE + 64]
    for at, value in ((2, None), (2, BASE + 1), (4, 1 << 31), (5, None), (5, BASE + 4), (6, None), (6, BASE), (7, None), (7, BASE)):
        args = list(good)
        args[at] = value
        assert code(ft.kv_grow, *args) == EINVAL, (at, value)
    good = [pool, t, BASE, BASE + 64, BASE + 64]
    for at, value in ((2, None), (3, None), (3, BASE), (4, None), (4, BASE), (4, BASE + 2)):
        args = list(good)
        args[at] = value
        assert code(ft.kv_release, *args) == EINVAL, (at, value)
    assert code(ft.kv_grow, pool, tables(requests=0), None, None, 0, None, None, None) == 0
    assert code(ft.kv_grow, pool, tables(requests=0), BASE, None, 3, BASE, BASE, BASE) == EINVAL
    assert code(ft.kv_release, pool, tables(requests=0), None, None, None) == 0


def test_steps_of_no_requests_that_are_refused(pool):
    """Their state is written all the same, so what it is read from and written to is looked at."""
    none = tables(requests=0, lens=None, table=None, free_pages=None)
    for other in (dict(state=None), dict(state=BASE + 2), dict(page_tokens=0), dict(pages=1 << 31), dict(pages=1 << 27)):
        bad = tables(**{"requests": 0, "lens": None, "table": None, "free_pages": None, **other})
        assert code(ft.kv_grow, pool, bad, None, None, 0, None, None, BASE + 64) == EINVAL, other
        assert code(ft.kv_release, pool, bad, None, None, BASE + 64) == EINVAL, other
    assert code(ft.kv_grow, pool, none, None, None, 3, None, None, BASE + 64) == EINVAL
    assert code(ft.kv_grow, pool, none, None, None, 3, BASE, None, None) == EINVAL
    for state_out in (BASE, BASE + 66):
        assert code(ft.kv_grow, pool, none, None, None, 0, None, None, state_out) == EINVAL
        assert code(ft.kv_release, pool, none, None, None, state_out) == EINVAL


def test_adapters_that_are_refused(pool):
    a, b = ft.slab_alloc(pool, 2 * 16 * 512), ft.slab_alloc(pool, 2 * 16 * 256)
    good = (a, b, 16, 1.0)
    records = ft.adapters_resolve(pool, [good, (a + 2 * 512, b, 15, 2.0)], 512, 256)
    assert len(records) == 48
    got = (ft.AdapterRecord * 2).from_buffer_copy(records)
    assert [(r.a, r.b, r.rank, r.scale) for r in got] == [(BASE + a, BASE + b, 16, 1.0), (BASE + a + 1024, BASE + b, 15, 2.0)]
    for bad in ((a, b, 0, 1.0), (a, b, 257, 1.0), (a, b, 16, math.nan), (a, b, 16, math.inf), (a + 1, b, 8, 1.0), (a, b + 1, 8, 1.0)):
        assert code(ft.adapters_resolve, pool, [good, bad], 512, 256) == EINVAL
    for bad in ((a, b, 17, 1.0), (a + 2, b, 16, 1.0), (b, a, 16, 1.0), (1 << 60, b, 16, 1.0)):
        assert code(ft.adapters_resolve, pool, [good, bad], 512, 256) == ERANGE
    assert code(ft.adapters_resolve, pool, [good], 0, 256) == EINVAL
    assert code(ft.adapters_resolve, pool, [good], 512, 1 << 24) == EINVAL
    assert ft.adapters_resolve(pool, [], 512, 256) == b""


def adapters_call(**other):
    given = dict(records=BASE, groups=BASE, x=BASE, base=BASE, out=BASE, x_stride=512, base_stride=256, out_stride=256, rows=8, count=4, type=0,
                 width_in=512, width_out=256, max_rank=16, workspace=BASE, workspace_bytes=0)
    given.update(other)
    return ft.AdaptersCall(*[given[n] for n, _ in ft.AdaptersCall._fields_])


@pytest.mark.parametrize("other", [
    dict(records=None), dict(groups=None), dict(groups=BASE + 8), dict(x=None), dict(out=None), dict(x=BASE + 1), dict(base=BASE + 1), dict(out=BASE + 1),
    dict(records=BASE + 4), dict(x_stride=511), dict(base_stride=255), dict(out_stride=255), dict(out_stride=1 << 40), dict(count=0), dict(type=2),
    dict(width_in=0), dict(width_out=0), dict(max_rank=0), dict(max_rank=257), dict(rows=1 << 31), dict(workspace_bytes=15)], ids=str)
def test_adapter_calls_that_are_refused(pool, other):
    assert code(ft.adapters_apply, pool, adapters_call(**{"workspace_bytes": 1 << 40, **other})) == EINVAL


def test_adapters_in_place_with_another_stride_are_refused(pool):
    """A row's result would lie where another row's base is still to be read."""
    for other in (dict(out_stride=264), dict(base_stride=300)):
        assert code(ft.adapters_apply, pool, adapters_call(workspace_bytes=1 << 40, **other)) == EINVAL, other


def test_groups_that_are_refused(pool):
    need = ft.adapters_group_bytes(100, 4)
    assert need >= 400
    for args in ((None, 100, 4, BASE, need), (BASE + 2, 100, 4, BASE, need), (BASE, 100, 0, BASE, need), (BASE, 100, 4, None, need),
                 (BASE, 100, 4, BASE + 8, need), (BASE, 100, 4, BASE, need - 1), (BASE, 1 << 31, 4, BASE, 1 << 40), (BASE, 100, (1 << 20) + 1, BASE, need)):
        assert code(ft.adapters_group, pool, *args) == EINVAL, args
    assert code(ft.adapters_group_bytes, 100, 0) == EINVAL
    assert code(ft.adapters_apply, pool, adapters_call(rows=0)) == 0


def test_tensors_that_are_refused(pool):
    """What the PyTorch side looks at before it hands pointers on: no tensor here lies on a GPU."""
    import torch
    from paper_2411_01830_amd import operators as ops
    i = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    x = torch.zeros(4, 8, 128, dtype=torch.bfloat16)
    c = ops.KvCache(pool, 0, 0, 32, 16, 8, 128, torch.bfloat16)
    assert code(ops.kv_append, c, x, x, torch.zeros(4, dtype=torch.int64)) == EINVAL
    assert code(ops.kv_grow, pool, i(4), i(5), 4, i(4, 8), i(9), i(4), 16) == EINVAL
    assert code(ops.kv_release, pool, torch.zeros(4, dtype=torch.bool), i(4), i(4, 8), i(9), i(4), 16) == EINVAL
    assert code(ops.tree_attention, c, x, x, x, i(2), i(1), i(1, 4), 4) == EINVAL
    assert code(ops.KvCache, pool, 0, 0, 32, 16, 8, 128, torch.float32) == EINVAL
    assert code(ops.Adapters, pool, [], 64, 64, torch.bfloat16) == EINVAL
    assert code(ops.Adapters, pool, [(0, 0, 8, 1.0)], 64, 64, torch.float32) == EINVAL
