"""What the operators between projections and next tokens refuse: checked before anything reaches a device, so without one."""
import ctypes as C
import math
import os
import shutil
import subprocess

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


def make(record, given, other):
    given = {**{n: 0 for n, _ in record._fields_}, **given, **other}
    return record(*[given[n] for n, _ in record._fields_])


def test_records_have_the_headers_layout(tmp_path):
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("no C compiler")
    both = [("ft_linear4", ft.Linear4Record), ("ft_linear4_call", ft.Linear4Call), ("ft_rotate_call", ft.RotateCall), ("ft_verify_call", ft.VerifyCall)]
    src = ["#include <stddef.h>", "#include <stdio.h>", '#include "faastube.h"', "int main(void) {"]
    want = []
    for name, rec in both:
        src.append(f'  printf("{name} %zu\\n", sizeof({name}));')
        want.append(f"{name} {C.sizeof(rec)}")
        for field, _ in rec._fields_:
            src.append(f'  printf("{name}.{field} %zu\\n", offsetof({name}, {field}));')
            want.append(f"{name}.{field} {getattr(rec, field).offset}")
    src.append('  printf("%d %d %d %d %d\\n", FT_FP32, FT_ROTATE_NORM, FT_ROTATE_NEIGHBOURS, FT_NO_ZEROS == ~(ft_off_t)0, (int)sizeof(ft_off_t));')
    want.append(f"2 {ft.ROTATE_NORM} {ft.ROTATE_NEIGHBOURS} 1 8")
    (tmp_path / "t.c").write_text("\n".join(src + ["  return 0;", "}"]))
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    subprocess.run([gcc, "-std=c99", "-Wall", "-Werror", "-I", os.path.join(root, "include"), str(tmp_path / "t.c"), "-o", str(tmp_path / "t")], check=True)
    assert subprocess.run([str(tmp_path / "t")], capture_output=True, text=True, check=True).stdout.split("\n")[:-1] == want


# ---- weights of 4 bits ------------------------------------------------------------------------------

def linear(pool, **other):
    given = dict(weights=ft.slab_alloc(pool, 256 * 500), scales=ft.slab_alloc(pool, 2 * 500 * 8), zeros=ft.slab_alloc(pool, 500 * 8), type=0, width_in=512,
                 width_out=500, group=64)
    return make(ft.Linear4Record, given, other)


def linear_call(**other):
    return make(ft.Linear4Call, dict(x=BASE, base=BASE, out=BASE + MiB, x_stride=512, base_stride=500, out_stride=500, rows=8, workspace=BASE,
                                     workspace_bytes=1 << 40), other)


@pytest.mark.parametrize("other", [dict(type=2), dict(width_in=0), dict(width_out=0), dict(width_in=1 << 24), dict(width_out=1 << 24), dict(group=0), dict(group=4),
                                   dict(group=60), dict(group=1 << 31), dict(scales=4097)], ids=str)
def test_weights_that_are_refused(pool, other):
    w = linear(pool, **other)
    assert code(ft.linear4_apply, pool, w, linear_call(x_stride=1 << 30, base_stride=1 << 30, out_stride=1 << 30)) == EINVAL
    assert code(ft.linear4_apply, pool, w, linear_call(rows=0)) == EINVAL
    assert code(ft.linear4_workspace, pool, w, linear_call()) == EINVAL


@pytest.mark.parametrize("other", [dict(width_out=513), dict(width_in=530), dict(group=8), dict(weights=64 * MiB), dict(scales=1 << 62), dict(zeros=1 << 40)], ids=str)
def test_weights_outside_their_allocations_are_refused(pool, other):
    assert code(ft.linear4_apply, pool, linear(pool, **other), linear_call(rows=0)) == ERANGE
    assert code(ft.linear4_apply, pool, linear(pool, **other), linear_call(x_stride=1024, base_stride=1024, out_stride=1024)) == ERANGE


def test_weights_without_zeros_need_none(pool):
    assert code(ft.linear4_apply, pool, linear(pool, zeros=ft.NO_ZEROS), linear_call(rows=0)) == 0
    w = linear(pool)
    assert code(ft.linear4_apply, pool, w, linear_call(rows=0)) == 0
    ft.slab_free(pool, w.zeros)
    assert code(ft.linear4_apply, pool, w, linear_call(rows=0)) == ERANGE


@pytest.mark.parametrize("other", [dict(x=None), dict(out=None), dict(x=BASE + 1), dict(base=BASE + 1), dict(out=BASE + 1), dict(x_stride=511), dict(base_stride=499),
                                   dict(out_stride=499), dict(x_stride=1 << 40), dict(rows=1 << 20), dict(out=BASE, base=BASE, out_stride=501),
                                   dict(out=BASE), dict(out=BASE, base=None, rows=1)], ids=str)
def test_products_that_are_refused(pool, other):
    assert code(ft.linear4_apply, pool, linear(pool), linear_call(**other)) == EINVAL


# ---- norms and rotations --------------------------------------------------------------------------------

def rotate_call(**other):
    given = {n: BASE for n in ("q", "k", "q_weight", "k_weight", "positions", "freqs", "axis")}
    given.update({n: 128 for n, _ in ft.RotateCall._fields_ if n.endswith("stride")})
    given.update(q_out=BASE + MiB, k_out=BASE + MiB, tokens=8, heads=4, kv_heads=2, dim=128, rot=128, axes=1, type=0, flags=3, eps=1e-6)
    return make(ft.RotateCall, given, other)


@pytest.mark.parametrize("other", [
    dict(q=None), dict(k=None), dict(q_out=None), dict(k_out=None), dict(q=BASE + 1), dict(k_out=BASE + 1), dict(positions=None), dict(positions=BASE + 2),
    dict(freqs=None), dict(freqs=BASE + 2), dict(q_weight=BASE + 1), dict(k_weight=BASE + 1), dict(eps=math.nan), dict(eps=math.inf), dict(eps=-1e-6),
    dict(type=2), dict(flags=4), dict(dim=0), dict(dim=12), dict(dim=264), dict(rot=129), dict(rot=127), dict(rot=136), dict(axes=0), dict(axes=257),
    dict(tokens=1 << 31), dict(heads=(1 << 16) + 1), dict(tokens=1 << 30, kv_heads=0), dict(q_token_stride=1 << 40), dict(k_head_stride=1 << 41),
    dict(q_out_token_stride=127), dict(k_out_head_stride=0), dict(q_out=BASE, q_out_token_stride=256), dict(k_out=BASE, k_out_head_stride=136)], ids=str)
def test_rotations_that_are_refused(pool, other):
    assert code(ft.rotate_heads, pool, rotate_call(**other)) == EINVAL


def test_nothing_to_rotate_is_nothing_wrong(pool):
    nothing = {n: None for n, t in ft.RotateCall._fields_ if t is C.c_void_p}
    assert code(ft.rotate_heads, pool, rotate_call(tokens=0, **nothing)) == 0
    assert code(ft.rotate_heads, pool, rotate_call(heads=0, kv_heads=0, **{**nothing, "positions": BASE, "freqs": BASE})) == 0


# ---- drafted tokens -------------------------------------------------------------------------------------

def verify_call(**other):
    given = {n: BASE for n, t in ft.VerifyCall._fields_ if t is C.c_void_p}
    given.update(target_stride=1000, draft_stride=1000, rows=20, requests=3, drafts=8, vocab=1000, type=2, workspace_bytes=1 << 40)
    return make(ft.VerifyCall, given, other)


@pytest.mark.parametrize("other", [
    dict(tokens=None), dict(tokens=BASE + 4), dict(starts=None), dict(starts=BASE + 2), dict(parent=BASE + 2), dict(target=None), dict(target=BASE + 2),
    dict(draft=BASE + 2), dict(accept=None), dict(accept=BASE + 2), dict(pick=None), dict(pick=BASE + 1), dict(keep=None), dict(last=None), dict(last=BASE + 2),
    dict(token=None), dict(token=BASE + 4), dict(target_stride=999), dict(draft_stride=999), dict(target_stride=1 << 40), dict(rows=1 << 31),
    dict(requests=(1 << 22) - 1), dict(drafts=0), dict(drafts=1025, rows=1025), dict(vocab=0), dict(vocab=(1 << 22) + 1, target_stride=1 << 23, draft_stride=1 << 23),
    dict(type=3), dict(type=0, target=BASE + 1)], ids=str)
def test_drafts_that_are_refused(pool, other):
    assert code(ft.tree_verify, pool, verify_call(**other)) == EINVAL


def test_no_drafts_are_nothing_wrong(pool):
    nothing = {n: None for n, t in ft.VerifyCall._fields_ if t is C.c_void_p}
    assert code(ft.tree_verify, pool, verify_call(rows=0, requests=0, **nothing)) == 0
    assert ft.verify_workspace(pool, verify_call(rows=0, requests=0)) == 0


def test_tensors_that_are_refused(pool):
    """What the PyTorch side looks at before it hands pointers on: no tensor here lies on a GPU."""
    import torch
    from paper_2411_01830_amd import operators as ops
    x = torch.zeros(4, 512, dtype=torch.bfloat16)
    w = ops.Linear4(pool, 0, 0, 512, 500, 64, torch.bfloat16)
    assert code(ops.linear4_apply, w, x) == EINVAL
    assert code(ops.Linear4, pool, 0, 0, 512, 500, 64, torch.float32) == EINVAL
    assert code(ops.Rotation, pool, [1.0] * 65, 128) == EINVAL
    assert code(ops.Rotation, pool, [1.0] * 4, 128, [0, 1, 2]) == EINVAL
    assert code(ops.Rotation, pool, [1.0] * 4, 128, [0, 1, 2, 256]) == EINVAL
    assert code(ops.Rotation, pool, [1.0] * 4, 128, [0, 1, 2, -1]) == EINVAL
    assert code(ops.Rotation, pool, torch.ones(4, requires_grad=True), 128) == EINVAL
    i = torch.zeros(4, dtype=torch.int32)
    p = torch.zeros(4, 10)
    assert code(ops.tree_verify, pool, i.long(), i[:2], 4, p, p[:, 0], p[:1, 0]) == EINVAL
