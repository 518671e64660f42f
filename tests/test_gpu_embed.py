"""Lookup in the vocabulary matrix and its gradient on the GPU, against 64-bit arithmetic on the same values.

Tolerances: a looked-up value is one fp32 product (8 bits: two), then rounded to its type: half a step (bf16 2^-8, fp32 none
further).  A gradient is a sum of c fp32 terms times the scale: c - 1 additions and a product of half a step 2^-24 each, on
partial sums of at most the sum of magnitudes (one more where it is added to a gradient that is there), then
rounded to its type."""

import pytest
import torch

from paper_2609_33645_b200 import binding, workloads as wl
from tests import helpers as H

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 2.0 ** -24
HALF = {torch.float32: EPS, torch.bfloat16: 2.0 ** -8}
TINY = 2.0 ** -126
BF, FP = torch.bfloat16, torch.float32


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def ids(shape, V, seed, none=0.2, hot=0.0):
    g = gen(seed)
    t = torch.randint(0, V, shape, generator=g, device=DEV, dtype=torch.int32)
    t = torch.where(torch.rand(shape, generator=g, device=DEV) < hot, V // 3, t)
    return torch.where(torch.rand(shape, generator=g, device=DEV) < none, -1, t).int()


def rows(n, D, dtype, seed, pad=0, shift=0):
    """[n, D] whose rows are D + pad apart and start `shift` values behind a 16-byte boundary."""
    buf = torch.full((n * (D + pad) + shift + 16,), float("nan"), device=DEV, dtype=dtype)
    v = buf[shift:shift + n * (D + pad)].view(n, D + pad)[:, :D]
    v.copy_(torch.randn(n, D, generator=gen(seed), device=DEV))
    return v


@pytest.mark.parametrize("M,V,D,pad,shift", [(1, 1, 1, 0, 0), (1, 151936, 1024, 0, 0), (7, 33, 8, 0, 0), (64, 500, 510, 0, 0),
                                            (65, 1001, 64, 8, 0), (130, 77, 96, 3, 0), (33, 50, 40, 0, 1), (257, 3000, 2056, 8, 8),
                                            (5000, 129, 72, 0, 0)])
@pytest.mark.parametrize("table,out", [(BF, BF), (BF, FP), (FP, BF), (FP, FP)])
def test_lookup(M, V, D, pad, shift, table, out):
    W, t = rows(V, D, table, 1, pad, shift), ids((M,), V, 2)
    for scale in (1.0, D ** 0.5):
        got = binding.embed(t, W, scale=scale, dtype=out)
        want = torch.where((t >= 0)[:, None], W[t.clamp(min=0).long()].float() * torch.tensor(scale, device=DEV), 0.0).to(out)
        assert got.dtype == out and torch.equal(got, want)         # one product, one rounding: the same bits
    to = rows(M, D, out, 3, pad, shift)
    assert binding.embed(t, W, scale=scale, out=to) is to and torch.equal(to, want)


@pytest.mark.parametrize("M,V,D", [(1, 1, 1), (64, 5000, 1024), (33, 100, 516), (257, 3000, 2056)])
@pytest.mark.parametrize("out", [BF, FP])
def test_lookup_in_8_bits(M, V, D, out):
    head = binding.quantize_rows(rows(V, D, FP, 1))
    t = ids((M,), V, 2)
    got = binding.embed(t, head, scale=1.7, dtype=out).double()
    want = torch.where((t >= 0)[:, None], head.q[t.clamp(min=0).long()].double() * head.scales[t.clamp(min=0).long()].double()[:, None], 0.0)
    want = want * float(torch.tensor(1.7))
    assert bool(((got - want).abs() <= want.abs() * (2 * EPS + HALF[out] * (1 + 2 * EPS)) + TINY).all())
    assert binding.embed(t, head).dtype == BF


def test_lookup_keeps_the_shape_of_the_tokens_and_takes_none_at_all():
    W = rows(50, 24, BF, 1)
    t = ids((2, 3, 5), 50, 2)
    assert binding.embed(t, W).shape == (2, 3, 5, 24)
    assert torch.equal(binding.embed(t, W)[1, 2], binding.embed(t[1, 2].contiguous(), W))
    for shape in ((0,), (4, 0)):
        assert binding.embed(torch.zeros(shape, dtype=torch.int32, device=DEV), W).shape == (*shape, 24)


def test_tokens_outside_the_vocabulary_give_zeros_and_no_gradient():
    bad = torch.tensor([-1, 50, 51, -2 ** 31, 2 ** 31 - 1, 0], dtype=torch.int32, device=DEV)
    for D in (24, 23):
        W = torch.full((50, D), float("nan"), device=DEV)
        got = binding.embed(bad, W)
        assert bool((got[:5] == 0).all()) and bool(got[5].isnan().all())
        g = torch.full((6, D), float("inf"), device=DEV)
        g[5] = 2.0
        dW = binding.embed_grad(bad, g, 50)["dW"]
        assert bool((dW[0] == 2).all()) and bool((dW[1:] == 0).all())


@pytest.mark.parametrize("M", [4, 300, 20_000])
def test_tokens_of_any_32_bits(M):
    V, D = 5000, 24
    t = torch.randint(-2 ** 31, 2 ** 31, (M,), generator=gen(1), device=DEV, dtype=torch.int64)
    t[::3] %= V
    t[:4] = torch.tensor([-2 ** 31, 2 ** 31 - 1, V, V - 1], device=DEV)
    t, there = t.int(), (t >= 0) & (t < V)
    W, g = rows(V, D, FP, 2), rows(M, D, FP, 3)
    assert torch.equal(binding.embed(t, W), torch.where(there[:, None], W[torch.where(there, t, 0).long()], 0.0))
    want = torch.zeros(V, D, device=DEV, dtype=torch.float64).index_add_(0, t[there].long(), g[there].double())
    sums = torch.zeros(V, D, device=DEV, dtype=torch.float64).index_add_(0, t[there].long(), g[there].double().abs())
    got = binding.embed_grad(t, g, V)["dW"].double()
    assert bool(((got - want).abs() <= M * EPS * sums).all())


def test_lookup_leaves_its_neighbours_alone():
    for D, dt in ((24, BF), (23, BF), (9, FP)):
        buf = torch.full((7, D + 9), 5.0, device=DEV, dtype=dt)
        W = rows(10, D, dt, 1)
        binding.embed(ids((5,), 10, 1), W, out=buf[1:6, 4:4 + D])
        keep = torch.ones_like(buf, dtype=torch.bool)
        keep[1:6, 4:4 + D] = False
        assert bool((buf[keep] == 5).all())


def test_matrices_of_more_than_2_31_values():
    V, D = 140_000, 16_384
    W = torch.empty(V, D, device=DEV, dtype=BF)
    t = torch.tensor([V - 1, 131_073, 0], dtype=torch.int32, device=DEV)
    x = rows(3, D, BF, 1)
    W[t.long()] = x
    assert torch.equal(binding.embed(t, W), x)
    dW = binding.embed_grad(t, x, dW=W)["dW"]
    assert torch.equal(dW[t.long()], x)
    assert not dW[131_074].any() and not dW[1].any() and not dW[V - 2].any()


def want_grad(t, g, V, scale):
    """The sum, the sum of magnitudes and the number of terms for every row, in 64 bits."""
    at = torch.where((t >= 0) & (t < V), t, V).long().reshape(-1)
    g = g.reshape(-1, g.shape[-1]).double()
    out = torch.zeros(V + 1, g.shape[-1], dtype=torch.float64, device=DEV)
    sums, mags = out.index_add(0, at, g)[:V], out.index_add(0, at, g.abs())[:V]
    return sums * scale, mags * abs(scale), torch.bincount(at, minlength=V + 1)[:V].double()[:, None]


def check_grad(got, t, g, V, scale, base=None):
    s = float(torch.tensor(scale, dtype=FP))
    want, mags, count = want_grad(t, g, V, s)
    near = (count + 1) * EPS * mags
    if base is not None:
        want, near = want + base.double(), near + EPS * (want + base.double()).abs()
    assert bool(((got.double() - want).abs() <= near + HALF[got.dtype] * (want.abs() + near) + TINY).all())


@pytest.mark.parametrize("M,V,D,none,hot", [
    (1, 1, 1, 0.0, 0.0), (1, 1000, 64, 0.0, 0.0), (5, 3, 24, 0.0, 0.0), (100, 1, 40, 0.0, 0.0), (513, 40, 8, 0.2, 0.0),
    (1000, 5003, 510, 0.1, 0.0), (2049, 300, 72, 0.0, 0.7), (3000, 151936, 16, 0.2, 0.0), (4097, 500_000, 8, 0.0, 0.3),
    (20_000, 2000, 256, 0.2, 0.0), (70_001, 50, 33, 0.5, 0.0), (9000, 1000, 128, 0.0, 1.0), (300, 700, 100, 1.0, 0.0),
    (262_145, 7, 8, 0.0, 0.5), (40_000, 3, 64, 0.3, 0.0), (2600, 2, 512, 0.0, 0.0), (66_000, 30, 1, 0.1, 0.3)])
@pytest.mark.parametrize("dtype,to", [(BF, BF), (FP, FP), (BF, FP), (FP, BF)])
def test_gradient(M, V, D, none, hot, dtype, to):
    t, g = ids((M,), V, 3, none, hot), rows(M, D, dtype, 4)
    for scale in (1.0, -D ** 0.5):
        r = binding.embed_grad(t, g, V, scale=scale, dtype=to)
        assert r["dW"].dtype == to and r["dW"].shape == (V, D)
        check_grad(r["dW"], t, g, V, scale)
        again = binding.embed_grad(t, g, dW=torch.full((V, D), float("nan"), device=DEV, dtype=to), scale=scale, workspace=r["workspace"])
        assert torch.equal(again["dW"], r["dW"])


def test_gradient_of_very_many_tokens():
    """More than a warp of the sort has bits for the positions of."""
    M, V = 40_000_000, 5
    t, g = ids((M,), V, 1, 0.1, 0.2), rows(M, 1, FP, 2)
    r = binding.embed_grad(t, g, V)
    check_grad(r["dW"], t, g, V, 1.0)
    assert torch.equal(binding.embed_grad(t, g, V, workspace=r["workspace"])["dW"], r["dW"])


@pytest.mark.parametrize("M,V,D", [(700, 500, 64), (700, 500, 63), (5000, 37, 40)])
@pytest.mark.parametrize("dtype,to", [(BF, BF), (FP, FP), (BF, FP)])
def test_gradient_adds_to_what_is_there_and_touches_nothing_else(M, V, D, dtype, to):
    t, g = ids((M,), V, 5, 0.3), rows(M, D, dtype, 6)
    base = rows(V, D, to, 7)
    there = torch.zeros(V, dtype=torch.bool, device=DEV)
    there[t[t >= 0].long()] = True
    base[~there] = float("nan")                                   # rows without a token are not even read
    dW = base.clone()
    version = dW._version
    assert binding.embed_grad(t, g, dW=dW, scale=0.5, accumulate=True)["dW"] is dW and dW._version > version
    assert bool(dW[~there].isnan().all())
    clean = torch.where(there[:, None], base, torch.zeros_like(base))
    check_grad(torch.where(there[:, None], dW, torch.zeros_like(dW)), t, g, V, 0.5, clean)


@pytest.mark.parametrize("pad,shift", [(8, 0), (3, 0), (0, 1)])
def test_gradient_with_strides(pad, shift):
    t = ids((900,), 123, 8)
    for D in (64, 61):
        for dt in (BF, FP):
            g, dW = rows(900, D, dt, 9, pad, shift), rows(123, D, dt, 10, pad, shift)
            binding.embed_grad(t, g, dW=dW)
            check_grad(dW, t, g, 123, 1.0)
            whole = torch.full((125, D + 10), 3.0, device=DEV, dtype=dt)
            binding.embed_grad(t, g, dW=whole[1:124, 5:5 + D])
            assert torch.equal(whole[1:124, 5:5 + D], dW)
            assert bool((whole[0] == 3).all() and (whole[124] == 3).all() and (whole[:, :5] == 3).all() and (whole[:, 5 + D:] == 3).all())


def test_gradient_without_tokens():
    t, g = torch.zeros((0,), dtype=torch.int32, device=DEV), torch.zeros((0, 24), device=DEV)
    assert not binding.embed_grad(t, g, 11)["dW"].any()
    dW = torch.ones(11, 24, device=DEV)
    binding.embed_grad(t, g, dW=dW, accumulate=True)
    assert bool((dW == 1).all())
    binding.embed_grad(t, g, dW=dW)
    assert not dW.any()


def test_gradient_is_the_lookups():
    """<embed(W), g> = <W, embed_grad(g)>, and the difference quotient along a direction, in 64 bits on whole numbers."""
    t = ids((400,), 90, 11)
    W = torch.randint(-8, 9, (90, 48), generator=gen(1), device=DEV).float()
    V = torch.randint(-8, 9, (90, 48), generator=gen(2), device=DEV).float()
    g = torch.randint(-8, 9, (400, 48), generator=gen(3), device=DEV).float()
    dW = binding.embed_grad(t, g, 90, scale=2.0)["dW"]
    assert float((binding.embed(t, W, scale=2.0).double() * g).sum()) == float((W.double() * dW).sum())
    step = binding.embed(t, W + V, scale=2.0) - binding.embed(t, W - V, scale=2.0)
    assert float((step.double() * g).sum()) / 2 == float((V.double() * dW).sum())


def test_not_finite_values_stay_in_their_rows():
    t = torch.tensor([4, 4, 7, 9, 9], dtype=torch.int32, device=DEV)
    g = torch.ones(5, 16, device=DEV)
    g[0, 3], g[2, 5], g[3, 6], g[4, 6] = float("nan"), float("inf"), float("inf"), float("-inf")
    dW = binding.embed_grad(t, g, 12)["dW"]
    assert bool(dW[4, 3].isnan()) and float(dW[7, 5]) == float("inf") and bool(dW[9, 6].isnan())
    assert int((~dW.isfinite()).sum()) == 3


def test_captured_into_a_graph_and_on_another_stream():
    t, g, W = ids((300,), 400, 1), rows(300, 64, BF, 2), rows(400, 64, BF, 3)
    dW, y = torch.empty(400, 64, device=DEV, dtype=BF), torch.empty(300, 64, device=DEV, dtype=BF)
    ws = binding.embed_grad(t, g, 400)["workspace"]

    def both():
        binding.embed(t, W, out=y)
        binding.embed_grad(t, g, dW=dW, workspace=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for seed in (5, 6):
        t.copy_(ids((300,), 400, seed, hot=0.3))
        g.copy_(rows(300, 64, BF, seed + 10))
        dW.fill_(9.0)
        graph.replay()
        torch.cuda.synchronize()
        check_grad(dW, t, g, 400, 1.0)
        assert torch.equal(y, binding.embed(t, W))


def test_the_gradient_of_a_tied_head():
    """What the head's backward pass has left in dW, plus the lookup's: one matrix on both sides of the model."""
    batch = wl.make_batch(wl.reduced(wl.CONFIGS["c2"], name="tied", V=2048, D=64, N=4, T_div=8, U_div=2), permute_ids=True)
    dev = torch.device(DEV)
    hidden, W = (torch.from_numpy(x).to(dev).to(BF) for x in (batch.hidden, batch.W))
    targets = torch.from_numpy(batch.targets).to(dev)
    r = binding.pruned_ctc_fwd_bwd(hidden, W, None, targets, batch.input_lengths, batch.target_lengths, batch.blank, check_status=True)
    before = r["dW"].clone()
    live = torch.arange(targets.shape[1], device=dev) < torch.tensor(list(batch.target_lengths), device=dev)[:, None]
    t = torch.where(live, targets, -1).int()
    x = binding.embed(t, W, scale=8.0)
    assert torch.equal(x, torch.where(live[..., None], (W[t.clamp(min=0).long()].float() * 8).to(BF), 0))
    g = torch.randn(x.shape, generator=gen(1), device=dev).to(BF)
    binding.embed_grad(t, g, dW=r["dW"], scale=8.0, accumulate=True)
    check_grad(r["dW"], t, g, 2048, 8.0, before)
    assert H.rel_fro(before.double().cpu().numpy(), H.run_oracle(batch)["dW"]) < 1e-2


def around(V, D, dtype, left, right, value):
    """A [V, D] view in the middle of a buffer of `value`, and a mask of what lies around it."""
    whole = torch.full((V + 2, D + left + right), value, device=DEV, dtype=dtype)
    outside = torch.ones(whole.shape, dtype=torch.bool, device=DEV)
    outside[1:-1, left:left + D] = False
    return whole, whole[1:-1, left:left + D], outside


@pytest.mark.parametrize("M", [1, 37, 255, 256, 257])
@pytest.mark.parametrize("D", [1023, 1024, 1025, 1026, 2050, 2056])
@pytest.mark.parametrize("dtype,to", [(BF, BF), (FP, FP), (BF, FP), (FP, BF)])
def test_gradient_of_few_tokens_in_one_and_several_slices(M, D, dtype, to):
    """Up to 256 tokens are one launch of blocks that have up to 1,024 columns each; 257 are sorted."""
    for V, hot in ((90, 0.0), (5003, 0.5), (1, 0.0)):
        t, g = ids((M,), V, 3, 0.2, hot), rows(M, D, dtype, 4)
        dW = binding.embed_grad(t, g, V, scale=0.7, dtype=to)["dW"]
        check_grad(dW, t, g, V, 0.7)
        given = torch.full((V, D), float("nan"), device=DEV, dtype=to)
        assert torch.equal(binding.embed_grad(t, g, dW=given, scale=0.7)["dW"], dW)


@pytest.mark.parametrize("M", [1, 37, 255, 256, 257])
@pytest.mark.parametrize("D,left,right", [(64, 8, 8), (61, 3, 2), (1025, 8, 7), (2050, 1, 1), (2056, 0, 8), (2048, 8, 0)])
@pytest.mark.parametrize("dtype", [BF, FP])
def test_gradient_of_few_tokens_with_strides(M, D, left, right, dtype):
    V = 301
    t, g = ids((M,), V, 5, 0.1), rows(M, D, dtype, 6, pad=left + right, shift=left)
    whole, dW, outside = around(V, D, dtype, left, right, 3.0)
    binding.embed_grad(t, g, dW=dW)
    check_grad(dW, t, g, V, 1.0)
    assert bool((whole[outside] == 3).all())


@pytest.mark.parametrize("M", [1, 37, 255, 256, 257])
@pytest.mark.parametrize("D,left,right", [(64, 0, 0), (63, 0, 0), (1025, 4, 3), (2050, 0, 0), (2056, 8, 8)])
@pytest.mark.parametrize("dtype,to", [(BF, BF), (FP, FP), (BF, FP)])
def test_gradient_of_few_tokens_adds_to_what_is_there(M, D, left, right, dtype, to):
    V = 301
    t, g = ids((M,), V, 7, 0.1, 0.3), rows(M, D, dtype, 8)
    there = torch.zeros(V, dtype=torch.bool, device=DEV)
    there[t[t >= 0].long()] = True
    whole, dW, outside = around(V, D, to, left, right, 3.0)
    dW.copy_(torch.randn(V, D, generator=gen(9), device=DEV))
    dW[~there] = float("nan")                                     # rows without a token are not even read
    base = dW.clone()
    binding.embed_grad(t, g, dW=dW, scale=0.5, accumulate=True)
    assert bool(dW[~there].isnan().all()) and bool((whole[outside] == 3).all())
    check_grad(torch.where(there[:, None], dW, 0.0), t, g, V, 0.5, torch.where(there[:, None], base, 0.0))


@pytest.mark.parametrize("M", [200, 3000])
def test_gradient_is_the_one_that_autograd_takes(M):
    """In 64 bits, through torch's own lookup."""
    V, D = 301, 72
    t, g = ids((M,), V, 10, 0.0), rows(M, D, FP, 11)
    W = torch.randn(V, D, generator=gen(12), device=DEV, dtype=torch.float64, requires_grad=True)
    (torch.nn.functional.embedding(t.long(), W) * 1.5).backward(g.double())
    dW = binding.embed_grad(t, g, V, scale=1.5)["dW"]
    mags = want_grad(t, g, V, 1.5)[1]
    count = torch.bincount(t.long(), minlength=V)[:, None]
    assert bool(((dW.double() - W.grad).abs() <= (count + 1) * EPS * mags + TINY).all())
