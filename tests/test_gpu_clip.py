"""Gradient clipping on the GPU against 64-bit arithmetic on the same values.

Tolerances: the norm is a sum of non-negative squares.  Up to eight values are squared and added in fp32
(at most 8 roundings of 2^-24 relative), all else in 64 bits, so S is off by less than 8 * 2^-24 and the norm by
half of that, and then rounded once: 5 * 2^-24.  A scaled value is g * f with f off by the norm's error and one
rounding to fp32, times one fp32 rounding (7 * 2^-24), then rounded to its type (bf16: 2^-8)."""

import math

import pytest
import torch

from paper_2609_33645_b200 import binding, data_parallel

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NORM_TOL = 5 * 2.0 ** -24
VALUE_TOL = {torch.float32: 8 * 2.0 ** -24, torch.bfloat16: 2.0 ** -8 + 8 * 2.0 ** -24}


def reference(grads, max_norm, eps=1e-6):
    norm = math.sqrt(sum(float((g.double() ** 2).sum()) for g in grads))
    fits = math.isfinite(norm) and norm <= torch.finfo(torch.float32).max
    f = min(1.0, max_norm / (norm + eps)) if fits else 1.0
    return norm, [g.double() * f for g in grads]


def close(got, want, dtype):
    tiny = torch.finfo(dtype).tiny
    assert bool(((got.double() - want).abs() <= VALUE_TOL[dtype] * want.abs() + tiny * 2.0 ** -7).all())


def make(sizes, dtypes, scale, seed, offset=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    out = []
    for i, s in enumerate(sizes):
        dt = dtypes[i % len(dtypes)]
        buf = torch.zeros(s + 16, device=DEV, dtype=dt)
        v = buf[offset:offset + s]
        v.normal_(std=scale * (1 + i % 3), generator=g)
        out.append(v)
    return out


SIZES = [[1], [7], [8], [8191, 8192, 8193], [1000 * 64, 64, 1, 0, 3], [5] * 60, [300_001, 17, 65_536], [2, 3] * 700]


@pytest.mark.parametrize("offset", [0, 1, 5])
@pytest.mark.parametrize("dtypes", [(torch.float32,), (torch.bfloat16,), (torch.bfloat16, torch.float32)])
@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}x{max(s)}")
def test_norm_and_values(sizes, dtypes, offset):
    for over in (True, False):
        grads = make(sizes, dtypes, 0.5, len(sizes), offset)
        total = max(1, sum(sizes))
        max_norm = (0.05 if over else 50.0) * math.sqrt(total)
        before = [g.clone() for g in grads]
        norm, want = reference(before, max_norm)
        assert (norm > max_norm) == over
        for mode in ("same", "fp32", "shifted", "place"):
            if mode == "place":
                r = binding.clip_grad_norm(grads, max_norm)
                outs = grads
            else:
                outs = [torch.empty(g.numel() + 16, device=DEV, dtype=torch.float32 if mode == "fp32" else g.dtype)
                        [3 if mode == "shifted" else 0:][:g.numel()] for g in grads]
                r = binding.clip_grad_norm(grads, max_norm, out=outs)
                for g, b in zip(grads, before):
                    assert torch.equal(g, b)
            assert float(r["norm"]) == pytest.approx(norm, rel=NORM_TOL)
            for o, w, b in zip(outs, want, before):
                close(o, w, o.dtype)
                if not over:
                    assert torch.equal(o.double(), b.double())


def test_neighbours_of_the_gradients_are_left_alone():
    for dt in (torch.bfloat16, torch.float32):
        for off in range(8):
            for n in (0, 1, 6, 7, 8, 9, 8200):
                buf = torch.full((n + 32,), 7.0, device=DEV, dtype=dt)
                buf[off:off + n] = 1.0
                keep = buf.clone()
                binding.clip_grad_norm([buf[off:off + n]], 1e-3)
                assert torch.equal(buf[:off], keep[:off]) and torch.equal(buf[off + n:], keep[off + n:])
                if n:
                    assert float(buf[off:off + n].max()) < 1.0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("value", [0.0, 1e-30, 1e-38, 1e30, 3e38])
def test_values_whose_squares_leave_fp32(dtype, value):
    g = torch.full((1001,), value, device=DEV, dtype=dtype)
    g[500:] = 0
    norm, want = reference([g], 1.0)
    r = binding.clip_grad_norm([g], 1.0)
    if norm <= float(torch.finfo(torch.float32).max):
        assert float(r["norm"]) == pytest.approx(norm, rel=NORM_TOL, abs=2.0 ** -149)
    else:
        assert float(r["norm"]) == math.inf          # beyond fp32: counts as not finite
    close(g, want[0], dtype)


def test_a_factor_below_the_normal_range():
    g = torch.full((4,), 1.5e38, device=DEV)
    norm, want = reference([g], 1e-3)
    binding.clip_grad_norm([g], 1e-3)
    close(g, want[0], torch.float32)


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_a_norm_that_is_not_finite_scales_nothing(bad):
    g = torch.randn(10_000, device=DEV)
    g[1234] = bad
    keep = g.clone()
    r = binding.clip_grad_norm([g], 1e-3)
    assert torch.equal(g.nan_to_num(1.5), keep.nan_to_num(1.5))
    assert not math.isfinite(float(r["norm"]))
    out = [torch.zeros_like(g)]
    binding.clip_grad_norm([g], 1e-3, out=out)
    assert torch.equal(out[0].nan_to_num(1.5), keep.nan_to_num(1.5))


def test_two_halves_make_the_whole_and_repeats_agree_bitwise():
    a = make([40_000, 999, 64], (torch.bfloat16, torch.float32), 0.3, 3)
    b = [t.clone() for t in a]
    c = [t.clone() for t in a]
    ra = binding.clip_grad_norm(a, 2.0)
    rb = binding.clip_grad_norm(b, 2.0)
    sq = binding.grad_sqsum(c)["sqsum"]
    rc = binding.grad_scale(c, sq, 2.0)
    assert torch.equal(ra["norm"], rb["norm"]) and all(torch.equal(x, y) for x, y in zip(a, b))
    # the partial sums are added in another order: 64 bits, then one rounding
    assert float(rc["norm"]) == pytest.approx(float(ra["norm"]), rel=2.0 ** -23)
    for x, y in zip(a, c):
        close(y, x.double(), x.dtype)
    # a norm without clipping
    d = [t.clone() for t in c]
    binding.clip_grad_norm(d, math.inf)
    assert all(torch.equal(x, y) for x, y in zip(c, d))


def test_data_parallel_form_without_a_group_is_the_plain_call():
    a = make([1000, 64], (torch.float32,), 1.0, 5)
    b = [t.clone() for t in a]
    r = data_parallel.clip_grad_norm_data_parallel(a, 1.0, sharded=True)
    s = binding.clip_grad_norm(b, 1.0)
    assert torch.equal(r["norm"], s["norm"]) and all(torch.equal(x, y) for x, y in zip(a, b))


def test_captured_into_a_graph_and_on_another_stream():
    g = make([70_000, 33], (torch.bfloat16,), 0.2, 9)
    out = [torch.zeros_like(t) for t in g]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        binding.clip_grad_norm(g, 1.0, out=out)
    torch.cuda.current_stream().wait_stream(side)
    first = [t.clone() for t in out]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = binding.clip_grad_norm(g, 1.0, out=out)
    for t in g:
        t.mul_(2.0)
    graph.replay()
    torch.cuda.synchronize()
    norm, want = reference(g, 1.0)
    assert float(r["norm"]) == pytest.approx(norm, rel=NORM_TOL)
    for o, w, f in zip(out, want, first):
        close(o, w, o.dtype)


def test_gradients_of_the_head_are_clipped():
    """The call as a training step makes it: gradients of the head, then clipping, then the update."""
    g = torch.Generator(device=DEV).manual_seed(0)
    hidden = torch.randn(2, 30, 64, device=DEV, generator=g)
    W = torch.randn(500, 64, device=DEV, generator=g) / 8
    bias = torch.zeros(500, device=DEV)
    targets = torch.randint(1, 500, (2, 5), device=DEV, generator=g, dtype=torch.int32)
    r = binding.pruned_ctc_fwd_bwd(hidden, W, bias, targets, [30, 20], [5, 3], 0)
    grads = [r["dW"], r["dbias"], r["dH"]]
    norm, want = reference(grads, 0.5)
    c = binding.clip_grad_norm(grads, 0.5)
    assert float(c["norm"]) == pytest.approx(norm, rel=NORM_TOL) and norm > 0.5
    for x, w in zip(grads, want):
        close(x, w, x.dtype)


@pytest.mark.parametrize("count", [48, 49, 192, 193, 512, 513, 1024, 1025, 2100])
def test_lists_of_every_table_size(count):
    for dtypes in ((torch.float32,), (torch.bfloat16, torch.float32)):
        grads = make([1 + i % 37 for i in range(count)], dtypes, 0.5, count, offset=count % 3)
        norm, want = reference([g.clone() for g in grads], 1.0)
        r = binding.clip_grad_norm(grads, 1.0)
        assert float(r["norm"]) == pytest.approx(norm, rel=NORM_TOL) and norm > 1.0
        for g, w in zip(grads, want):
            close(g, w, g.dtype)


@pytest.mark.parametrize("offset", [0, 3])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_many_values(dtype, offset):
    """Enough for a CTA a chunk in the second pass (32 MB and more), odd sizes, every kind of output."""
    grads = make([17_000_001, 5, 12_345_677, 1], (dtype,), 0.01, 2, offset)
    before = [g.clone() for g in grads]
    norm, want = reference(before, 1.0)
    for kind in ("same", "fp32", "shifted", "place"):
        start = 1 if kind == "shifted" else offset
        whole = [torch.full((g.numel() + 16,), 9.0, device=DEV, dtype=torch.float32 if kind == "fp32" else dtype) for g in grads]
        outs = grads if kind == "place" else [o[start:start + g.numel()] for o, g in zip(whole, grads)]
        r = binding.clip_grad_norm(grads, 1.0, out=None if kind == "place" else outs)
        assert float(r["norm"]) == pytest.approx(norm, rel=NORM_TOL) and norm > 1.0
        for x, w in zip(outs, want):
            close(x, w, x.dtype)
        if kind != "place":                                 # what lies around the outputs is left alone
            for o, g in zip(whole, grads):
                assert bool((o[:start] == 9.0).all()) and bool((o[start + g.numel():] == 9.0).all())


def test_more_values_than_32_bits_count():
    n = (1 << 31) + 4099
    g = torch.zeros(n, device=DEV, dtype=torch.bfloat16)
    at = [0, 5, (1 << 31) - 1, 1 << 31, n - 1]
    for i in at:
        g[i] = 2.0
    r = binding.clip_grad_norm([g], 1.0)
    assert float(r["norm"]) == pytest.approx(math.sqrt(20.0), rel=NORM_TOL)
    want = 2.0 / (math.sqrt(20.0) + 1e-6)
    for i in at:
        assert abs(float(g[i]) - want) <= VALUE_TOL[torch.bfloat16] * want
    assert float(g[1]) == 0.0 and float(g[n - 2]) == 0.0


def test_capture_of_the_two_pass_form():
    g = make([9_000_000, 33], (torch.float32,), 0.02, 9)
    out = [torch.zeros_like(t) for t in g]
    binding.clip_grad_norm(g, 1.0, out=out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = binding.clip_grad_norm(g, 1.0, out=out)
    for t in g:
        t.mul_(3.0)
    graph.replay()
    torch.cuda.synchronize()
    norm, want = reference(g, 1.0)
    assert float(r["norm"]) == pytest.approx(norm, rel=NORM_TOL)
    for o, w in zip(out, want):
        close(o, w, o.dtype)


def test_refusals_on_the_device():
    g = torch.ones(64, device=DEV)
    for grads, kw in [([g, g], {}), ([g, g[8:16]], {}), ([g[:32], g[16:48]], {}), ([g[:32]], dict(out=[g[8:40]]))]:
        with pytest.raises(binding.PctcError):
            binding.clip_grad_norm(grads, 1.0, **kw)
    for grads, kw, match in [([g.double()], {}, "bf16 or fp32"), ([g.view(8, 8).t()], {}, "contiguous"),
                             ([g, torch.ones(3)], {}, "one device"), ([g], dict(out=[]), "same shape"),
                             ([g], dict(out=[g[:32]]), "same shape")]:
        with pytest.raises(ValueError, match=match):
            binding.clip_grad_norm(grads, 1.0, **kw)
    for bad in (0.0, -1.0, math.nan):
        with pytest.raises(binding.PctcError):
            binding.clip_grad_norm([g], bad)
    with pytest.raises(binding.PctcError):                  # bf16 gradients go to bf16 or fp32, fp32 ones to fp32
        binding.clip_grad_norm([g], 1.0, out=[torch.empty(64, device=DEV, dtype=torch.bfloat16)])
    assert bool((g == 1.0).all())
    r = binding.clip_grad_norm([g, g[:0]], 100.0)           # an empty tensor is nothing
    assert float(r["norm"]) == 8.0
    assert float(binding.clip_grad_norm([g[:0]], 1.0)["norm"]) == 0.0


def test_written_gradients_count_up():
    """As by torch's own in-place operations, so that autograd notices a saved tensor that was scaled."""
    g, out = torch.ones(100, device=DEV), torch.empty(100, device=DEV)
    binding.clip_grad_norm([g], 1.0, out=[out])
    assert g._version == 0 and out._version == 1
    binding.clip_grad_norm([g], 1.0)
    sq = binding.grad_sqsum([g])["sqsum"]
    assert g._version == 1 and sq._version == 0
    binding.grad_scale([g], sq, 1.0)
    assert g._version == 2 and sq._version == 0
    x = torch.ones(100, device=DEV, requires_grad=True)
    y = x * 3
    loss = (y * y).sum()
    binding.clip_grad_norm([y.detach()], 1.0)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("size", [50_000, 5_000_000])
def test_replicas_agree_bit_for_bit_when_equally_aligned(size, dtype):
    whole = torch.randn(size, device=DEV).to(dtype)

    def copy(offset):
        buf = torch.empty(size + 64, device=DEV, dtype=dtype)
        v = buf[offset:offset + size]
        v.copy_(whole)
        return v

    group = 16 // dtype.itemsize
    one, two, other = copy(1), copy(1 + 3 * group), copy(2)
    norms = [binding.clip_grad_norm([t], 1.0)["norm"] for t in (one, two, other)]
    assert torch.equal(norms[0], norms[1]) and torch.equal(one, two)
    assert abs(float(norms[2]) - float(norms[0])) <= 2 * NORM_TOL * float(norms[0])
    # the sum of one replica scales all of them alike, wherever they lie
    one, other = copy(1), copy(2)
    sq = binding.grad_sqsum([one])["sqsum"]
    norms = [binding.grad_scale([t], sq, 1.0)["norm"] for t in (one, other)]
    assert torch.equal(norms[0], norms[1]) and torch.equal(one, other)
