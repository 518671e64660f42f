"""The clipped policy loss on the GPU against the same formula in 64 bits, and its gradient against differences of that.

Tolerances, in roundings of 2^-24 (EPS): a ratio is 64 bits (where |d| < 1: with a series of fourteen fp32
operations for what goes beyond 1 + d, at most 0.72 of it) and rounded once; a gradient two products and a sum more, the KL
terms expm1f (one step: 2 EPS) or that series and two products; the weight 2^-48 and a rounding.  16 EPS of the sum of the terms' magnitudes covers them all; sums are 64 bits."""

import math

import pytest
import torch

from paper_2609_33645_b200 import binding, workloads as wl
from tests import helpers as H

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 2.0 ** -24
TOL = 16 * EPS
TINY = 2.0 ** -126


def counted(logp, mask, lengths):
    count = torch.ones_like(logp, dtype=torch.bool) if mask is None else mask.clone()
    if lengths is not None:
        count &= torch.arange(logp.shape[1], device=DEV) < lengths.clamp(0, logp.shape[1])[:, None]
    return count


def reference(logp, old, adv, ref=None, mask=None, lengths=None, clip=(0.2, 0.2), kl_weight=0.0, reduction="tokens", negated=False):
    """loss, grad, kl, clipped, count, and how large the terms of a token are, all in 64 bits."""
    sign = -1.0 if negated else 1.0
    count = counted(logp, mask, lengths)
    at = count.nonzero(as_tuple=True)
    new, was = (sign * x.double()[at] for x in (logp, old))
    A = adv.double()[at] if adv.dim() == 2 else adv.double()[at[0]]
    r = torch.exp(new - was)
    cut = torch.clamp(r, 1 - clip[0], 1 + clip[1])
    clipped = A * r > A * cut
    token = -torch.minimum(A * r, A * cut)
    grad = torch.where(clipped, 0.0, -A * r)
    size, kl = (A * r).abs().clamp(max=1e300) * ~clipped + (A * cut).abs(), torch.zeros_like(new)
    if ref is not None:
        f = sign * ref.double()[at] - new
        kl = torch.expm1(f) - f
        token, grad = token + kl_weight * kl, grad - kl_weight * torch.expm1(f)
        size = size + abs(kl_weight) * (kl.abs() + torch.expm1(f).abs())
    rows = count.sum(1)
    n = max(1, int(count.sum()))
    if reduction == "tokens":
        w = torch.full_like(new, 1 / n)
    elif reduction == "sequences":
        w = 1.0 / (rows[at[0]].double() * max(1, int((rows > 0).sum())))
    else:
        w = torch.ones_like(new)
    full = torch.zeros(logp.shape, dtype=torch.float64, device=DEV)
    sizes = full.clone()
    full[at], sizes[at] = sign * w * grad, w * size
    return dict(loss=float((w * token).sum()), grad=full, kl=float(kl.sum() / n), clipped=int(clipped.sum()) / n,
                count=int(count.sum()), size=sizes, kl_size=float(kl.abs().sum() / n))


def check(r, want):
    total = float(want["size"].sum())
    assert abs(float(r["loss"]) - want["loss"]) <= TOL * total + TINY
    assert bool(((r["grad"].double() - want["grad"]).abs() <= TOL * want["size"] + TINY).all())
    assert bool((r["grad"][want["size"] == 0] == 0).all())
    assert abs(float(r["kl"]) - want["kl"]) <= TOL * want["kl_size"] + TINY
    assert abs(float(r["clipped"]) - want["clipped"]) <= EPS * want["clipped"]
    assert int(r["count"]) == want["count"] and r["count"].dtype == torch.int32


def inputs(N, T, seed, each=False, ref=True, mask=False, lengths=False, moved=0.2, garbage=True, spread=0.3):
    g = torch.Generator(device=DEV).manual_seed(seed)
    old = torch.log(torch.rand(N, T, generator=g, device=DEV).clamp(min=1e-6))
    k = dict(logp=old + moved * torch.randn(N, T, generator=g, device=DEV), old=old,
             adv=torch.randn((N, T) if each else (N,), generator=g, device=DEV))
    k["ref"] = old + spread * torch.randn(N, T, generator=g, device=DEV) if ref else None
    k["mask"] = torch.rand(N, T, generator=g, device=DEV) < 0.6 if mask else None
    if mask and N > 1:
        k["mask"][N // 2] = False                                 # a row of which nothing counts
    k["lengths"] = torch.randint(0, T + 1, (N,), generator=g, device=DEV, dtype=torch.int32) if lengths else None
    if garbage:
        count = counted(k["logp"], k["mask"], k["lengths"])
        for i, name in enumerate(("logp", "old", "ref")):
            if k[name] is not None:
                k[name][~count] = (math.nan, math.inf, -torch.finfo(torch.float32).max)[i]
    return k


def call(k, **kw):
    return binding.policy_loss(k["logp"], k["old"], k["adv"], ref_logp=k["ref"], mask=k["mask"], lengths=k["lengths"], **kw)


SHAPES = [(1, 1), (3, 1), (64, 1), (5, 7), (4, 33), (1, 2048), (17, 501), (2, 40_000), (3000, 11), (300, 300), (4096, 1), (70_001, 1)]


@pytest.mark.parametrize("N,T", SHAPES)
@pytest.mark.parametrize("reduction", binding.POLICY_REDUCTIONS)
@pytest.mark.parametrize("mask,lengths", [(False, False), (True, False), (False, True), (True, True)])
def test_loss_and_gradient(N, T, reduction, mask, lengths):
    for each, ref, negated in ((False, True, False), (True, False, True)):
        k = inputs(N, T, N + T, each, ref, mask, lengths)
        if negated:
            for name in ("logp", "old"):
                k[name] = -k[name]
        kw = dict(clip=(0.2, 0.3), kl_weight=0.05, reduction=reduction, negated=negated)
        r = call(k, **kw)
        check(r, reference(**k, **kw))
        again = call(k, workspace=r["workspace"], **kw)
        for name in ("loss", "grad", "kl", "clipped", "count"):
            assert torch.equal(r[name], again[name])
        alone = call(k, want_grad=False, **kw)
        assert "grad" not in alone and torch.equal(alone["loss"], r["loss"]) and torch.equal(alone["count"], r["count"])


@pytest.mark.parametrize("shape", [(6, 50), (200, 400)])
def test_gradient_against_differences(shape):
    k = inputs(*shape, 5, each=True, mask=True, moved=0.5, garbage=False)
    kw = dict(clip=(0.1, 0.3), kl_weight=0.2)
    r = call(k, **kw)
    step = 1e-6
    ratio = torch.exp(k["logp"].double() - k["old"].double())
    for seed in range(3):
        v = torch.randn(shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV).double()
        v[((ratio - 0.9).abs() < 1e-4) | ((ratio - 1.3).abs() < 1e-4)] = 0      # not across a bend
        up, down = (reference(**{**k, "logp": k["logp"].double() + s * step * v}, **kw)["loss"] for s in (1, -1))
        left, right = (up - down) / (2 * step), float((v * r["grad"].double()).sum())
        # central differences: step^2 / 6 of the third derivative, and 2^-53 of the loss over the step
        size = float((v.abs() * reference(**k, **kw)["size"]).sum())
        assert abs(left - right) <= TOL * size + 10 * step ** 2 * size + 1e-9 * size


def test_borders_and_ties():
    """At a ratio of exactly 1 + high or 1 - low the gradient is the ratio's; with low = high = 0 and unmoved tokens, too."""
    z = torch.zeros(1, 4, device=DEV)
    adv = torch.tensor([[1.0, -1.0, 0.0, 2.0]], device=DEV)
    r = binding.policy_loss(z, z, adv, clip=(0.0, 0.0), reduction="sum")
    assert r["grad"].tolist() == [[-1.0, 1.0, 0.0, -2.0]] and float(r["clipped"]) == 0 and float(r["loss"]) == -2
    tiny = torch.full_like(z, 2.0 ** -20)
    r = binding.policy_loss(tiny, z, adv, clip=(0.0, 0.0), reduction="sum")
    assert r["grad"][0, 0] == 0 and r["grad"][0, 3] == 0 and r["grad"][0, 1] > 0.9 and float(r["clipped"]) == 0.5
    r = binding.policy_loss(tiny, z, adv, clip=(1.0, math.inf), reduction="sum")
    assert float(r["clipped"]) == 0


def test_small_kl_terms_keep_their_digits():
    f = torch.cat([10.0 ** torch.arange(-6, 1, 0.01), -10.0 ** torch.arange(-6, 1, 0.01)]).to(DEV)[:, None].contiguous()
    z, adv = torch.zeros_like(f), torch.zeros(f.shape[0], device=DEV)
    for i in range(0, f.shape[0], 7):
        r = binding.policy_loss(z[i:i + 1], z[i:i + 1], adv[i:i + 1], ref_logp=f[i:i + 1], kl_weight=1.0)
        x = f[i].double()
        want = float(torch.expm1(x) - x) if abs(float(x)) > 1e-2 else float(x * x / 2 * (1 + x / 3 * (1 + x / 4 * (1 + x / 5))))
        # from 1/4 on a difference of rounded numbers: at most 4 EPS (|e^f - 1| + |f|), at most 14 times the result
        assert abs(float(r["kl"]) - want) <= 64 * EPS * want
        assert abs(float(r["grad"]) + float(torch.expm1(x))) <= TOL * float(torch.expm1(x).abs())


def test_values_that_are_not_finite():
    inf = math.inf
    new = torch.tensor([[-inf, -1.0, 200.0, 200.0, -1.0, math.nan]], device=DEV)
    old = torch.tensor([[-1.0, -inf, 0.0, 0.0, -1.0, -1.0]], device=DEV)
    for at, adv, loss, grad in ((0, 1.0, 0.0, 0.0), (0, -1.0, 0.8, 0.0), (1, 1.0, -1.2, 0.0), (1, -1.0, inf, inf), (2, 1.0, -1.2, 0.0),
                                (2, -1.0, inf, inf), (3, 0.0, 0.0, 0.0), (4, 1.0, -1.0, -1.0)):
        r = binding.policy_loss(new[:, at:at + 1], old[:, at:at + 1], torch.tensor([adv], device=DEV))
        assert float(r["loss"]) == pytest.approx(loss, rel=TOL) and float(r["grad"]) == pytest.approx(grad, rel=TOL), (at, adv)
    r = binding.policy_loss(new, old, torch.ones(1, device=DEV))
    assert math.isnan(float(r["loss"])) and bool(r["grad"][0, 5].isnan()) and bool(r["grad"][0, :5].isfinite().all())
    # a reference that has no such token, a model that has none
    one = torch.full((1, 1), -1.0, device=DEV)
    r = binding.policy_loss(one, one, torch.ones(1, device=DEV), ref_logp=one - inf, kl_weight=1.0)
    assert float(r["kl"]) == inf and float(r["grad"]) == 0.0     # exp(-inf) - 1 + inf; -A r - (0 - 1)
    r = binding.policy_loss(one - inf, one, torch.ones(1, device=DEV), ref_logp=one, kl_weight=1.0)
    assert float(r["kl"]) == inf and float(r["grad"]) == -inf
    # no advantage: nothing times the ratio of a finite difference, however large; 0 * inf of an infinite one
    for x, o, nan in ((1000.0, 0.0, False), (-1.0, -inf, True), (-inf, -1.0, False), (-inf, -inf, True)):
        r = binding.policy_loss(torch.full((1, 1), x, device=DEV), torch.full((1, 1), o, device=DEV), torch.zeros(1, device=DEV))
        assert all(math.isnan(float(r[k])) == nan and (nan or float(r[k]) == 0.0) for k in ("loss", "grad")), (x, o)


def test_nothing_counted():
    k = inputs(4, 9, 1)
    for kw in (dict(mask=torch.zeros(4, 9, dtype=torch.bool, device=DEV)), dict(lengths=torch.zeros(4, dtype=torch.int32, device=DEV)),
               dict(lengths=torch.full((4,), -3, dtype=torch.int32, device=DEV))):
        for reduction in binding.POLICY_REDUCTIONS:
            r = call({**k, **{**dict(mask=None, lengths=None), **kw}}, reduction=reduction, kl_weight=1.0)
            assert [float(r[n]) for n in ("loss", "kl", "clipped", "count")] == [0, 0, 0, 0] and not r["grad"].any()
    long = call({**k, "lengths": torch.full((4,), 100, dtype=torch.int32, device=DEV)})
    assert torch.equal(long["grad"], call(k)["grad"])


@pytest.mark.parametrize("N,T", [(9, 40), (130, 400)])
def test_strides(N, T):
    k = inputs(N, T + 3, 7, each=True, mask=True)
    narrow = {n: (v[:, 2:2 + T] if v is not None and v.dim() == 2 else v) for n, v in k.items()}
    dense = {n: (v.contiguous() if v is not None else None) for n, v in narrow.items()}
    a, b = (call(x, kl_weight=0.1, reduction="sequences") for x in (narrow, dense))
    for name in ("loss", "grad", "kl", "clipped", "count"):
        assert torch.equal(a[name], b[name])
    col = {n: (v[:, 3] if v is not None and v.dim() == 2 else v) for n, v in k.items()}     # [N], one a row
    want = {n: (v.contiguous()[:, None] if v is not None and v.dim() == 1 else v) for n, v in col.items()}
    a = call(col)
    assert a["grad"].shape == (N,)
    check({**a, "grad": a["grad"][:, None]}, reference(**want))


def test_refusals():
    k = inputs(4, 9, 1, mask=True, lengths=True)
    for change in (dict(logp=k["logp"].double()), dict(logp=k["logp"].t()), dict(old=k["old"][:3]), dict(ref=k["ref"].bfloat16()),
                   dict(mask=k["mask"].int()), dict(lengths=k["lengths"].long()), dict(adv=k["adv"][:3]), dict(adv=k["adv"][:, None]),
                   dict(adv=k["adv"].double()), dict(old=k["old"].cpu())):
        with pytest.raises(ValueError):
            call({**k, **change})
    with pytest.raises(binding.PctcError):
        call(k, clip=(1.5, 0.2))
    with pytest.raises(binding.PctcError):
        call({n: (None if n in ("ref", "mask", "lengths") else v[:0]) for n, v in k.items()})


def test_captured_into_a_graph_and_on_another_stream():
    for N, T in ((8, 30), (200, 300)):
        k = inputs(N, T, 3, mask=True, lengths=True)
        kw = dict(kl_weight=0.1, reduction="sequences")
        ws = call(k, **kw)["workspace"]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            check(call(k, workspace=ws, **kw), reference(**k, **kw))
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            r = call(k, workspace=ws, **kw)
        for seed in (4, 5):
            for name, v in inputs(N, T, seed, mask=True, lengths=True).items():
                k[name].copy_(v)
            graph.replay()
            torch.cuda.synchronize()
            check(r, reference(**k, **kw))


def test_a_policy_step_over_transcripts():
    """Losses from the head, weights from the policy loss, gradients from the head: those of the weighted losses."""
    batch = wl.make_batch(wl.reduced(wl.CONFIGS["c2"], name="policy", V=1024, D=64, N=6, T_div=8, U_div=2), permute_ids=True)
    batch.input_lengths[3] = 2                                     # too short for its labels: not counted
    dev = torch.device(DEV)
    hidden, W = (torch.from_numpy(x).to(dev).to(torch.bfloat16) for x in (batch.hidden, batch.W))
    targets = torch.from_numpy(batch.targets).to(dev)
    args = (hidden, W, None, targets, batch.input_lengths, batch.target_lengths, batch.blank)
    loss = binding.pruned_ctc_fwd_bwd(*args, forward_only=True)["loss"]
    old = loss + torch.tensor([0.1, -0.4, 0.02, 5.0, 0.5, -0.1], device=dev)
    adv = torch.tensor([1.0, -1.0, 0.5, 9.0, 2.0, -0.3], device=dev)
    r = binding.ctc_policy_fwd_bwd(*args, old, adv, ref_losses=old - 0.2, kl_weight=0.1, check_status=True)
    live = torch.tensor([[True]] * 3 + [[False]] + [[True]] * 2, device=dev)
    want = reference(loss[:, None], old[:, None], adv, (old - 0.2)[:, None], live, None, (0.2, 0.2), 0.1, "sequences", True)
    check({**r["policy"], "grad": r["policy"]["grad"][:, None]}, want)
    assert want["clipped"] > 0 and int(r["policy"]["count"]) == 5 and torch.equal(r["loss"], loss)
    ref = H.run_oracle(batch, utt_weights=want["grad"][:, 0].cpu().numpy())
    for name in ("dH", "dW"):
        assert H.rel_fro(r[name].double().cpu().numpy(), ref[name]) < 1e-2


@pytest.mark.parametrize("N,T", [(2000, 1), (40, 400), (300, 300)])
def test_gains_that_cancel(N, T):
    """Advantages of both signs whose gains add up to almost nothing: the sum is no worse than its last rounding and the
    32-bit part of each token, exp(d) - 1 - d within 4 EPS."""
    k = inputs(N, T, 11, each=True, ref=False, garbage=False, moved=0.1)
    r = torch.exp(k["logp"].double() - k["old"].double()).clamp(0.8, 1.2)
    k["adv"] = k["adv"] - ((k["adv"].double() * r).sum() / r.sum()).float()
    for reduction in binding.POLICY_REDUCTIONS:
        want = reference(**k, reduction=reduction)
        d = k["logp"].double() - k["old"].double()
        w = 1.0 if reduction == "sum" else 1.0 / (N * T)
        part = float((k["adv"].double().abs() * (torch.expm1(d) - d)).sum()) * w
        got = float(call(k, reduction=reduction)["loss"])
        assert abs(want["loss"]) < 1e-3 * float(want["size"].sum())
        assert abs(got - want["loss"]) <= EPS * abs(want["loss"]) + 4 * EPS * part


def test_a_policy_step_with_the_defaults_spelt_out():
    batch = wl.make_batch(wl.reduced(wl.CONFIGS["c2"], name="policy", V=512, D=64, N=4, T_div=8, U_div=2), permute_ids=True)
    dev = torch.device(DEV)
    hidden, W = (torch.from_numpy(x).to(dev).to(torch.bfloat16) for x in (batch.hidden, batch.W))
    args = (hidden, W, None, torch.from_numpy(batch.targets).to(dev), batch.input_lengths, batch.target_lengths, batch.blank,
            torch.full((4,), 100.0, device=dev), torch.ones(4, device=dev))
    a, b = binding.ctc_policy_fwd_bwd(*args), binding.ctc_policy_fwd_bwd(*args, forward_only=False, utt_weights=None, skip_dW=False)
    for name in ("loss", "dH", "dW"):
        assert torch.equal(a[name], b[name])


@pytest.mark.parametrize("N,T", [(1, 40), (7, 33), (40, 100), (5, 4001), (300, 300)])
@pytest.mark.parametrize("reduction", binding.POLICY_REDUCTIONS)
def test_exponentials_beyond_fp32(N, T, reduction):
    """Ratios and KL terms that fp32 does not hold, with weights that bring them back; kl_weight = 0 takes nothing of a KL term."""
    for mask, kl_weight, small in ((False, 0.0, 1.0), (True, 0.0, 1.0), (False, 1e-6, 1e-3), (True, -1e-30, 1e-30)):
        k = inputs(N, T, N + T, each=True, mask=mask, garbage=False)
        g = torch.Generator(device=DEV).manual_seed(3)
        far = torch.rand(N, T, generator=g, device=DEV) < 4 / (N * T)
        far[N // 2 - 1 if mask else 0, :2] = True
        if mask:
            k["mask"][N // 2 - 1, :2] = True
        k["logp"] = torch.where(far, k["old"] + 89.0, k["logp"])         # e^89 = 4.5e38
        k["adv"] = torch.where(far, -small * 1e-3 * k["adv"].abs(), k["adv"])
        up = torch.rand(N, T, generator=g, device=DEV) < 4 / (N * T)
        up[N // 2 - 1 if mask else 0, 1:4] = True
        k["ref"] = torch.where(up, k["logp"] + (88.9 if kl_weight == 0 else 95.0), k["ref"])
        kw = dict(kl_weight=kl_weight, reduction=reduction, clip=(0.2, 0.2))
        want = reference(**k, **kw)
        r = call(k, **kw)
        if want["kl"] > 3e38:                                            # the mean of the KL terms is beyond fp32 itself
            assert math.isinf(float(r["kl"]))
            want["kl"], want["kl_size"] = 0.0, 0.0
            r["kl"] = torch.zeros(1)
        assert want["grad"].abs().max() < 3e38 and abs(want["loss"]) < 3e38
        check(r, want)


def test_a_reference_that_is_only_watched_leaves_the_loss_alone():
    """kl_weight = 0: the loss and its gradient are those without a reference, however far that is."""
    for N, T in ((3, 5), (300, 300)):
        k = inputs(N, T, 1, garbage=False)
        far = k["logp"] + torch.linspace(-3000.0, 3000.0, N, device=DEV)[:, None]
        r = call({**k, "ref": far}, kl_weight=0.0)
        assert math.isinf(float(r["kl"]))
        check({**r, "kl": torch.zeros(1)}, reference(**{**k, "ref": None}))


@pytest.mark.parametrize("N,T", [(64, 1), (8, 30), (3, 1600), (256, 4096)])
def test_the_loss_does_not_hold_on_to_the_gradient_and_the_workspace(N, T):
    k = inputs(N, T, 1, mask=True)
    for r in (call(k), call(k, want_grad=False), call(k, workspace=call(k)["workspace"])):
        for name in ("loss", "kl", "clipped", "count"):
            assert r[name].untyped_storage().nbytes() <= 64 and r[name].shape == (1,)
            assert all(r[name].untyped_storage().data_ptr() != r[o].untyped_storage().data_ptr() for o in ("grad", "workspace") if o in r)
