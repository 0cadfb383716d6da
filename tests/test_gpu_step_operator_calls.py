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
