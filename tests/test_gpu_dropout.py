"""Dropout on the GPU against the generator in whole numbers.

Tolerances: a kept value is one fp32 product with a factor that is rounded to fp32, a residual one addition: three roundings
of 2^-24, the last on the sum, then rounded to the type (bf16 2^-8, half a step)."""

import numpy as np
import pytest
import torch

from paper_2609_33645_b200 import binding
from tests.philox import kept

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 2.0 ** -24
HALF = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8}
BF, FP = torch.bfloat16, torch.float32


def values(shape, dtype, seed):
    return torch.randn(shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV).to(dtype)


def check(got, x, p, seed, offset, residual=None):
    keep, scale = kept(0, x.numel(), p, seed, offset)
    keep = torch.from_numpy(keep).to(DEV).reshape(x.shape)
    part = torch.where(keep, x.double() * scale, 0.0)
    want = part if residual is None else part + residual.double()
    near = 2 * EPS * part.abs() + (0 if residual is None else EPS * want.abs())
    assert bool(((got.double() - want).abs() <= near + HALF[got.dtype] * (want.abs() + near)).all())
    if residual is None:
        assert torch.equal(got == 0, ~keep | (x == 0))


@pytest.mark.parametrize("shape", [(1,), (7,), (8,), (9,), (3, 5), (5, 64), (2, 3, 40), (33, 250), (1, 4099), (4, 2048)])
@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("p,seed,offset", [(0.1, 0, 0), (0.5, 2 ** 63 + 12345, 7), (0.3, -1, 2 ** 40 + 3), (0.97, 99, 2 ** 64 - 1)])
def test_values(shape, dtype, p, seed, offset):
    x, r = values(shape, dtype, 1), values(shape, dtype, 2)
    check(binding.dropout(x, p, seed, offset=offset), x, p, seed, offset)
    check(binding.dropout(x, p, seed, offset=offset, residual=r), x, p, seed, offset, r)
    place = x.clone()
    version = place._version
    assert binding.dropout(place, p, seed, offset=offset, out=place) is place and place._version > version
    check(place, x, p, seed, offset)
    onto = r.clone()
    binding.dropout(x, p, seed, offset=offset, residual=onto, out=onto)
    check(onto, x, p, seed, offset, r)


def test_many_values_take_the_form_with_four_groups_a_thread():
    for dtype in (BF, FP):
        for shape in ((6000, 1024), (48_001, 128), (6_300_013,)):
            x = values(shape, dtype, 3)
            y = binding.dropout(x, 0.25, 5, offset=6)
            n = x.numel()
            flat, out = x.view(-1), y.view(-1)
            for first in (0, n // 2 // 8 * 8, (n - 2000) // 8 * 8):
                part = slice(first, min(n, first + 2000))
                keep, scale = kept(first, flat[part].numel(), 0.25, 5, 6)
                want = torch.where(torch.from_numpy(keep).to(DEV), flat[part].double() * scale, 0.0)
                assert bool(((out[part].double() - want).abs() <= want.abs() * (2 * EPS + HALF[dtype] * (1 + 2 * EPS))).all())
            # 16-bit words of a counter are as good as independent: the share of zeros within six deviations
            assert abs(float((y == 0).double().mean()) - 0.25) < 6 * (0.25 * 0.75 / n) ** 0.5


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("rows,cols,pad,shift", [(5, 64, 8, 0), (7, 24, 3, 0), (3, 40, 0, 1), (6, 33, 7, 8), (2, 8, 120, 16)])
def test_strides_do_not_change_the_mask(dtype, rows, cols, pad, shift):
    dense = values((rows, cols), dtype, 4)
    res = values((rows, cols), dtype, 5)

    def spread(v):
        buf = torch.full((rows * (cols + pad) + shift + 16,), 7.0, device=DEV, dtype=dtype)
        view = buf[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
        view.copy_(v)
        return buf, view
    want, want_res = binding.dropout(dense, 0.4, 8), binding.dropout(dense, 0.4, 8, residual=res)
    (_, x), (_, r), (buf, out) = spread(dense), spread(res), spread(dense)
    assert torch.equal(binding.dropout(x, 0.4, 8), want)
    binding.dropout(x, 0.4, 8, residual=r, out=out)
    assert torch.equal(out, want_res)
    outside = buf.clone()
    outside[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols] = 7.0
    assert bool((outside == 7).all())


def test_columns_of_one_buffer_are_told_apart():
    buf = values((6, 3 * 32), BF, 1)
    x, out = buf[:, :32], buf[:, 64:]
    want = binding.dropout(x.contiguous(), 0.5, 3)
    binding.dropout(x, 0.5, 3, out=out)
    assert torch.equal(out, want)
    for bad in (buf[:, 31:63], buf[1:, :32]):
        with pytest.raises((binding.PctcError, ValueError)):
            binding.dropout(x, 0.5, 3, out=bad)


def test_dropped_values_are_zero_whatever_they_were():
    x = torch.full((4, 64), float("nan"), device=DEV)
    y = binding.dropout(x, 0.5, 1)
    keep, _ = kept(0, 256, 0.5, 1, 0)
    keep = torch.from_numpy(keep).to(DEV).view(4, 64)
    assert bool(y[keep].isnan().all()) and bool((y[~keep] == 0).all())
    assert not binding.dropout(torch.full_like(x, float("inf")), 1.0, 1).any()      # p = 1: nothing is left
    x = values((4, 64), FP, 1)
    assert torch.equal(binding.dropout(x, 0.0, 1), x)


def test_no_values_at_all():
    for shape in ((0,), (0, 8), (3, 0)):
        assert binding.dropout(torch.zeros(shape, device=DEV), 0.5, 1).shape == shape


def test_the_backward_pass_is_the_same_call():
    x, g = values((9, 77), FP, 1).requires_grad_(), values((9, 77), FP, 2)
    keep, scale = kept(0, x.numel(), 0.35, 11, 12)
    y = x * torch.from_numpy(keep * scale).float().to(DEV).view(9, 77)
    y.backward(g)
    got = binding.dropout(g, 0.35, 11, offset=12)
    assert bool(((got - x.grad).abs() <= 2 * EPS * x.grad.abs()).all())
    # along a direction, by differences: the call is linear in its values
    v = values((9, 77), FP, 3)
    a, b = (binding.dropout((x.detach() + s * v), 0.35, 11, offset=12).double() for s in (1, -1))
    left, right = float(((a - b) / 2 * g).sum()), float((v.double() * got).sum())
    size = float((got.abs().double() * (v.abs() + x.detach().abs())).sum())
    assert abs(left - right) <= 8 * EPS * size


def test_step_counts_the_offset_up_in_a_captured_call():
    x, out = values((50, 96), BF, 1), torch.empty(50, 96, device=DEV, dtype=BF)
    step = torch.zeros(1, dtype=torch.int64, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        binding.dropout(x, 0.3, 4, offset=10, step=step, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.dropout(x, 0.3, 4, offset=10, step=step, out=out)
    masks = []
    for i in range(3):
        step.fill_(i)
        graph.replay()
        assert torch.equal(out, binding.dropout(x, 0.3, 4, offset=10 + i))
        masks.append(out.clone())
    assert not torch.equal(masks[0], masks[1]) and not torch.equal(masks[1], masks[2])


def test_more_than_2_32_values():
    n = 2 ** 32 + 4096 + 5
    x = torch.ones(n, device=DEV, dtype=BF)
    binding.dropout(x, 0.5, 21, out=x)
    for first in (2 ** 31 - 8, 2 ** 32 - 8, (n - 30) // 8 * 8):
        count = min(30, n - first)
        keep, _ = kept(first, count, 0.5, 21, 0)
        assert np.array_equal((x[first:first + count] != 0).cpu().numpy(), keep)
