"""What is measured of the operators around the head: clipping before the weight update, and beam search after it.

Four operators, each once in elementary torch operations (``own`` false) and once through the
package's binding (``own`` true):

  clip    global gradient norm over many tensors, and clipping
  select  beam search's selection over beams and vocabulary
  move    reordering of the decoder states of the selected beams
  prefix  CTC prefix beam search over the k best classes of every frame

``listed()`` and ``draw()`` give cases, ``prepare()`` their inputs, ``run()`` one pass, ``work()`` the
bytes and operations of a pass, ``exact()`` the results in 64 bits on the host.
"""

import math

import numpy as np
import torch

own = False

FLAG_EMPTY, FLAG_NONFINITE = 1, 2      # no hypothesis is left; an input was NaN or infinite
RESCALE_EVERY = 16                     # frames between rescalings of the prefix probabilities
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


# ---------------------------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------------------------

def listed():
    return [
        # The gradients of a tiny fp32 head and what feeds it: V=1000, D=64, and a few odd-sized parameters.
        dict(name="clip tiny fp32", op="clip", dtype="fp32", tensors=7, total=99_991, packed=False, place="out", over=True),
        # An encoder's parameters in one packed bucket (odd offsets), in place, in the usual step that needs no clipping.
        dict(name="clip encoder in place", op="clip", dtype="bf16", tensors=384, total=64_000_001, packed=True,
             place="in", over=False),
        # Head dW [151936, 1024] with its bias and a few others, clipped into another buffer.
        dict(name="clip head bf16", op="clip", dtype="bf16", tensors=6, total=156_000_000, packed=False,
             place="out", over=True),
        # One utterance, the paper's beam of 4, fp32 logits.
        dict(name="select 1x4 fp32", op="select", dtype="fp32", N=1, B=4, K=4, V=151936, pad=0, done=0.0, masked=0.0),
        # A batch with ended hypotheses and a vocabulary of odd size, so that rows start on odd addresses.
        dict(name="select 16x4 odd", op="select", dtype="bf16", N=16, B=4, K=4, V=50_001, pad=0, done=0.25, masked=0.1),
        # A large serving batch over the full vocabulary in padded rows.
        dict(name="select 64x8 bf16", op="select", dtype="bf16", N=64, B=8, K=8, V=151936, pad=128, done=0.1, masked=0.0),
        # Token histories and small recurrent states of one utterance.
        dict(name="move 1x4 small", op="move", dtype="fp32", N=1, B=4, heads=1, L=150, D=16, caches=2, recurrent=512,
             place="out", moved=1.0),
        # Decoder caches [N, B, heads, L, D]; half of the hypotheses stay in their slot.
        dict(name="move caches in place", op="move", dtype="bf16", N=8, B=4, heads=8, L=300, D=64, caches=12, recurrent=0,
             place="in", moved=0.5),
        # The same for a batch of 16, into a second set of buffers, every slot from its parent.
        dict(name="move caches 16x8", op="move", dtype="bf16", N=16, B=8, heads=8, L=151, D=64, caches=16, recurrent=0,
             place="out", moved=1.0),
        # One second of speech at 25 frames a second.
        dict(name="prefix 1x25 beam 4", op="prefix", N=1, T_lo=25, T_hi=25, k=8, B=4, V=1000, sharp=4.0),
        # A batch of utterances of 300 to 500 frames with the paper's beam.
        dict(name="prefix 16x500 beam 4", op="prefix", N=16, T_lo=300, T_hi=500, k=8, B=4, V=180000, sharp=3.0),
        # Long utterances, a wide beam and flat posteriors, where most candidates compete.
        dict(name="prefix 8x1500 beam 16", op="prefix", N=8, T_lo=800, T_hi=1500, k=8, B=16, V=151936, sharp=1.0),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["clip", "select", "move", "prefix"])
    dtype = rng.choice(["bf16", "fp32"])
    if op == "clip":
        total = _log_int(rng, 50_000, 150_000_000 if dtype == "bf16" else 75_000_000)
        place = rng.choice(["in", "out"])
        return dict(op=op, dtype=dtype, tensors=_log_int(rng, 1, 384), total=total, packed=rng.random() < 0.5,
                    place=place, over=place == "out" and rng.random() < 0.7)
    if op == "select":
        V = _log_int(rng, 500, 180_000)
        if rng.random() < 0.6:
            V = (V + 7) // 8 * 8
        B = rng.choice([1, 2, 3, 4, 5, 8, 16])
        N = _log_int(rng, 1, max(1, min(64, (70_000_000 if dtype == "bf16" else 35_000_000) // (B * V))))
        return dict(op=op, dtype=dtype, N=N, B=B, K=B if rng.random() < 0.7 else rng.choice([1, 4, 10, 16]), V=V,
                    pad=rng.choice([0, 0, 64, 128]), done=rng.choice([0.0, 0.1, 0.3]) if B > 1 else 0.0,
                    masked=rng.choice([0.0, 0.1]))
    if op == "move":
        B = rng.choice([2, 3, 4, 8])
        heads, D, caches = rng.choice([1, 4, 8]), rng.choice([32, 64, 128]), rng.randint(1, 16)
        L = _log_int(rng, 2, 600)
        N = _log_int(rng, 1, max(1, min(16, 120_000_000 // (B * heads * L * D * caches))))
        place = rng.choice(["in", "out"])
        return dict(op=op, dtype=dtype, N=N, B=B, heads=heads, L=L, D=D, caches=caches,
                    recurrent=rng.choice([0, 0, 257, 512]), place=place, moved=0.5 if place == "in" else 1.0)
    N, T = rng.choice([1, 2, 4, 8, 16]), _log_int(rng, 10, 700)
    return dict(op=op, N=N, T_lo=max(1, T // 2), T_hi=T, k=rng.choice([1, 2, 4, 8, 8, 8]), B=rng.choice([1, 2, 4, 8, 10, 16]),
                V=rng.choice([1000, 151936, 180000]), sharp=rng.choice([0.5, 1.0, 2.0, 4.0]))


# ---------------------------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------------------------

def _sizes(case):
    """Element counts of the gradient tensors: a few large matrices and many small vectors."""
    n, total = case["tensors"], case["total"]
    w = [1.0 / (1 + i) ** 0.7 for i in range(n)]
    sizes = [max(1, int(total * x / sum(w))) for x in w]
    sizes[0] += total - sum(sizes)
    return sizes


def _views(flat, sizes, packed):
    out, at = [], 0
    for s in sizes:
        out.append(flat[at:at + s])
        at += s if packed else (s + 63) // 64 * 64
    return out


def _prepare_clip(case, g):
    sizes, dtype = _sizes(case), DTYPES[case["dtype"]]
    room = sum(s if case["packed"] else (s + 63) // 64 * 64 for s in sizes)
    flat = torch.zeros(room, dtype=dtype, device="cuda")
    grads = _views(flat, sizes, case["packed"])
    # the norm of standard normal values is sqrt(total); gradients of one tensor share a scale
    scale = (8.0 if case["over"] else 0.5) / math.sqrt(case["total"])
    for i, t in enumerate(grads):
        t.normal_(std=scale * (0.5 + (i * 7 % 11) / 11.0), generator=g)
    s = dict(flat=flat, grads=grads, max_norm=1.0, out=None, out_flat=None)
    if case["place"] == "out":
        s["out_flat"] = torch.zeros_like(flat)
        s["out"] = _views(s["out_flat"], sizes, case["packed"])
    return s


def _prepare_select(case, g):
    N, B, V = case["N"], case["B"], case["V"]
    full = torch.randn(N, B, V + case["pad"], generator=g, device="cuda").mul_(2.5).to(DTYPES[case["dtype"]])
    logits = full[:, :, :V]
    if case["masked"]:
        logits.masked_fill_(torch.rand(V, generator=g, device="cuda") < case["masked"], -math.inf)
    scores = -20.0 - 10.0 * torch.rand(N, B, generator=g, device="cuda")
    if case["done"]:
        finished = torch.rand(N, B, generator=g, device="cuda") < case["done"]
    else:
        finished = None
    return dict(logits=logits, scores=scores, finished=finished, eos=2 if finished is not None else None, K=case["K"])


def _prepare_move(case, g):
    N, B, H, L, D = (case[x] for x in ("N", "B", "heads", "L", "D"))
    dtype = DTYPES[case["dtype"]]
    slots = torch.arange(B, device="cuda", dtype=torch.int32).expand(N, B).contiguous()
    if case["place"] == "in":
        # survivors stay where they are; the other slots copy one of the survivors
        keep = B - max(1, int(B * case["moved"])) if B > 1 else 1
        pick = torch.randint(0, keep, (N, B), generator=g, device="cuda", dtype=torch.int32)
        parents = torch.where(slots < keep, slots, pick)
    else:
        parents = torch.randint(0, B, (N, B), generator=g, device="cuda", dtype=torch.int32)
    lengths = torch.randint((L + 1) // 2, L + 1, (N,), generator=g, device="cuda", dtype=torch.int32)
    states = [torch.randint(0, 1000, (N, B, L), generator=g, device="cuda", dtype=torch.int32)]
    axes = [2]
    for _ in range(case["caches"]):
        states.append(torch.randn(N, B, H, L, D, generator=g, device="cuda").to(dtype))
        axes.append(3)
    if case["recurrent"]:
        states.append(torch.randn(N, B, case["recurrent"], generator=g, device="cuda").to(dtype))
        axes.append(None)
    out = [torch.zeros_like(x) for x in states] if case["place"] == "out" else None
    return dict(states=states, axes=axes, parents=parents, lengths=lengths, out=out)


def _prepare_prefix(case, g):
    """What a head gives for speech: confusion sets that last some frames, blank in most of them."""
    N, T, k, V = case["N"], case["T_hi"], case["k"], case["V"]
    dev = "cuda"
    seg = (T + 7) // 8
    base = torch.randint(0, V - 1, (N, seg, 1), generator=g, device=dev)
    step = torch.randint(1, max(2, (V - 1) // k), (N, seg, 1), generator=g, device=dev)
    sets = 1 + (base + step * torch.arange(k, device=dev)) % (V - 1)           # k different classes, none of them blank
    if k > 1:
        has_blank = torch.rand(N, seg, generator=g, device=dev) < 0.9
        sets[:, :, 0] = torch.where(has_blank, torch.zeros_like(sets[:, :, 0]), sets[:, :, 0])
    sets = sets.repeat_interleave(8, dim=1)[:, :T]
    bias = torch.randn(N, seg, k, generator=g, device=dev).repeat_interleave(8, dim=1)[:, :T]
    z = case["sharp"] * (torch.randn(N, T, k, generator=g, device=dev) + bias)
    z = z - torch.log(torch.exp(z.double()).sum(-1, keepdim=True) + 0.01).float()
    z, order = torch.sort(z, dim=-1, descending=True)
    span = case["T_hi"] - case["T_lo"] + 1
    lengths = [case["T_lo"] + int(v * span) for v in torch.rand(N, generator=g, device=dev).tolist()]
    lengths[0] = T
    return dict(classes=torch.gather(sets, -1, order).int().contiguous(), logprobs=z.contiguous(), lengths=lengths,
                blank=0, B=case["B"])


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    make = dict(clip=_prepare_clip, select=_prepare_select, move=_prepare_move, prefix=_prepare_prefix)[case["op"]]
    return dict(make(case, g), op=case["op"])


# ---------------------------------------------------------------------------------------------
# Plain forms
# ---------------------------------------------------------------------------------------------

def _plain_clip(s):
    # long sums in 64 bits; the factor is applied in 32 bits and rounded once
    total = torch.zeros((), dtype=torch.float64, device="cuda")
    for t in s["grads"]:
        total = total + t.double().square().sum()
    norm = total.sqrt()
    factor = torch.clamp(s["max_norm"] / (norm + 1e-6), max=1.0)
    factor = torch.where(torch.isfinite(norm), factor, torch.ones_like(factor)).float()
    for t, o in zip(s["grads"], s["out"] or s["grads"]):
        o.copy_(t.float() * factor)
    return dict(norm=norm.float().reshape(1), grads=s["flat"] if s["out"] is None else s["out_flat"])


def _plain_select(s):
    # 64 bits: candidates of different beams are compared, and equal ones go to the lowest index
    x, scores, K = s["logits"].double(), s["scores"], s["K"]
    N, B, V = x.shape
    m = x.amax(-1, keepdim=True)
    m = torch.where(torch.isinf(m) & (m < 0), torch.zeros_like(m), m)
    lse = m + torch.log(torch.exp(x - m).sum(-1, keepdim=True))
    live = torch.isfinite(scores)
    done = torch.zeros_like(live) if s["finished"] is None else s["finished"]
    bad = (live & ~done & (torch.isnan(lse[..., 0]) | (lse[..., 0] == math.inf))) | torch.isnan(scores) | (scores == math.inf)
    use = live & ~done & torch.isfinite(lse[..., 0])
    cand = torch.where(use[..., None], scores.double()[..., None] + (x - lse), -math.inf)
    if s["finished"] is not None:
        cand[:, :, s["eos"]] = torch.where(live & done, scores.double(), cand[:, :, s["eos"]])
    best, at = torch.sort(cand.reshape(N, B * V), dim=-1, descending=True, stable=True)
    if B * V < K:
        best, at = torch.nn.functional.pad(best, (0, K - B * V), value=-math.inf), torch.nn.functional.pad(at, (0, K - B * V))
    best, at = best[:, :K], at[:, :K]
    none = best == -math.inf
    parents = torch.where(none, -1, at // V).int()
    tokens = torch.where(none, -1, at % V).int()
    ended = torch.gather(done, 1, parents.clamp(min=0).long()) & ~none
    if s["eos"] is not None:
        ended = ended | (tokens == s["eos"])
    return dict(scores=best.float(), parents=parents, tokens=tokens, finished=ended,
                flags=torch.where(bad.any(1), FLAG_NONFINITE, 0).int())


def _plain_move(s):
    rows = s["parents"].clamp(min=0).long()
    n = torch.arange(rows.shape[0], device="cuda")[:, None]
    for x, axis, o in zip(s["states"], s["axes"], s["out"] or s["states"]):
        new = x[n, rows]
        keep = (s["parents"] >= 0).reshape(rows.shape + (1,) * (x.dim() - 2))
        if axis is not None:
            t = torch.arange(x.shape[axis], device="cuda").reshape((-1,) + (1,) * (x.dim() - 1 - axis))
            keep = keep & (t < s["lengths"].reshape((-1,) + (1,) * (x.dim() - 1)))
        o.copy_(torch.where(keep, new, o))
    return list(s["out"] or s["states"])


def _probabilities(classes, logprobs):
    """exp(logprob - the frame's largest), to 24 significant bits, 0 for what does not count; and the shifts."""
    lp = logprobs.double()
    bad = (classes >= 0) & (torch.isnan(lp) | (lp == math.inf))
    ok = (classes >= 0) & torch.isfinite(lp)
    k = classes.shape[-1]
    twice = (classes[..., :, None] == classes[..., None, :]) & ok[..., None, :]
    twice = twice & torch.ones(k, k, dtype=torch.bool, device=lp.device).tril(-1)
    ok = ok & ~twice.any(-1)
    shift = torch.where(ok, lp, -math.inf).amax(-1)
    shift = torch.where(torch.isfinite(shift), shift, torch.zeros_like(shift))
    z = lp - shift[..., None]
    ok = ok & (z >= -700.0)
    p = torch.exp(torch.where(ok, z, torch.zeros_like(z)))
    bits = (p.view(torch.int64) + (1 << 28)) & ~((1 << 29) - 1)
    return torch.where(ok, bits.view(torch.float64), torch.zeros_like(p)), shift, bad.any(-1)


def _plain_prefix(s):
    classes, B, blank = s["classes"].long(), s["B"], s["blank"]
    N, T, k = classes.shape
    dev = classes.device
    lengths = torch.tensor(s["lengths"], device=dev)
    inside = torch.arange(T, device=dev) < lengths[:, None]
    prob, shift, bad = _probabilities(classes, s["logprobs"])
    flags = torch.where((bad & inside).any(1), FLAG_NONFINITE, 0)
    prob = prob * inside[..., None]
    p_blank = (prob * (classes == blank)).sum(-1)
    pb = torch.zeros(N, B, dtype=torch.float64, device=dev)
    pb[:, 0] = 1.0
    pn = torch.zeros_like(pb)
    last = torch.full((N, B), -1, device=dev)
    size = torch.zeros(N, B, dtype=torch.long, device=dev)
    toks = torch.full((N, B, T + 1), -1, dtype=torch.int32, device=dev)
    power = torch.zeros(N, dtype=torch.float64, device=dev)
    n = torch.arange(N, device=dev)[:, None]
    for t in range(T):
        cls, p, seen = classes[:, t], prob[:, t], toks[:, :, :t + 1]
        total = pb + pn
        again = (cls[:, None, :] == last[:, :, None]) & (p[:, None, :] > 0)                 # [N, B, k]
        grow = torch.where(again, pb[:, :, None], total[:, :, None]) * p[:, None, :] * (cls != blank)[:, None, :]
        stay_b = total * p_blank[:, t, None]
        stay_n = pn * (again * p[:, None, :]).sum(-1)
        # slot c holds the prefix of slot r and one label more: r's extension by that label is slot c's prefix
        short = seen.scatter(2, (size - 1).clamp(min=0)[..., None], -1)
        child = (short[:, :, None, :] == seen[:, None, :, :]).all(-1) & (size[:, :, None] == size[:, None, :] + 1)
        child = child & (total[:, :, None] > 0) & (total[:, None, :] > 0)                   # [N, c, r]
        same = child[..., None] & again[:, :, None, :]                                      # [N, c, r, j]
        stay_n = stay_n + (same * grow[:, None]).sum((2, 3))
        grow = torch.where(same.any(1), torch.zeros_like(grow), grow)
        stay = stay_b + stay_n
        value, at = torch.sort(torch.cat([stay, grow.reshape(N, B * k)], 1), dim=1, descending=True, stable=True)
        value, at = value[:, :B], at[:, :B]
        stays = at < B
        r = torch.where(stays, at, (at - B).clamp(min=0) // k)
        c = cls[n, (at - B).clamp(min=0) % k]
        go = inside[:, t, None]
        new_size = size[n, r] + (~stays & (value > 0))
        new_toks = toks[n, r]
        new_toks = new_toks.scatter(2, size[n, r][..., None], torch.where(stays, toks[n, r].gather(
            2, size[n, r][..., None])[..., 0], c.int())[..., None])
        new_b = torch.where(stays, stay_b[n, r], torch.zeros_like(value))
        new_n = torch.where(stays, stay_n[n, r], value)
        if t % RESCALE_EVERY == RESCALE_EVERY - 1:
            top = (new_b + new_n)[:, 0]
            e = torch.where(top > 0, torch.frexp(top).exponent, torch.zeros_like(top, dtype=torch.int32))
            scale = torch.ldexp(torch.ones_like(top), -e)[:, None]
            new_b, new_n = new_b * scale, new_n * scale
            power = power + torch.where(go[:, 0], e, torch.zeros_like(e))
        pb, pn = torch.where(go, new_b, pb), torch.where(go, new_n, pn)
        last = torch.where(go, torch.where(stays, last[n, r], c), last)
        size = torch.where(go, new_size, size)
        toks = torch.where(go[..., None], new_toks, toks)
    total = pb + pn
    live = total > 0
    score = torch.log(total) + (power * math.log(2.0) + (shift * inside).sum(1))[:, None]
    flags = flags | torch.where(live.any(1), 0, FLAG_EMPTY)
    size = torch.where(live, size, torch.zeros_like(size))
    toks = torch.where(torch.arange(T, device=dev) < size[..., None], toks[:, :, :T], -1)
    return dict(tokens=toks.int(), token_lengths=size.int(), scores=torch.where(live, score, -math.inf).float(),
                flags=flags.int())


def run(s):
    if own:
        from paper_2609_33645_b200 import binding
        if s["op"] == "clip":
            r = binding.clip_grad_norm(s["grads"], s["max_norm"], out=s["out"])
            return dict(norm=r["norm"], grads=s["flat"] if s["out"] is None else s["out_flat"])
        if s["op"] == "select":
            r = binding.beam_select(s["logits"], s["scores"], s["K"], finished=s["finished"], eos_id=s["eos"])
            return dict(scores=r["scores"], parents=r["parents"], tokens=r["tokens"], finished=r["finished"], flags=r["flags"])
        if s["op"] == "move":
            return binding.beam_reorder(s["states"], s["parents"], lengths=s["lengths"], time_axes=s["axes"], out=s["out"])
        r = binding.prefix_beam_decode(s["classes"], s["logprobs"], s["lengths"], s["blank"], s["B"])
        return dict(tokens=r["tokens"], token_lengths=r["token_lengths"], scores=r["scores"], flags=r["flags"])
    return dict(clip=_plain_clip, select=_plain_select, move=_plain_move, prefix=_plain_prefix)[s["op"]](s)


# ---------------------------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------------------------

def work(case):
    size = 2 if case.get("dtype") == "bf16" else 4
    if case["op"] == "clip":
        # every value read once; written where it changes or goes to another buffer
        written = case["total"] * size if case["place"] == "out" or case["over"] else 0
        return dict(bytes=case["total"] * size + written + 4, flops=3 * case["total"])
    if case["op"] == "select":
        live = case["N"] * case["B"] * (1 - case["done"])
        return dict(bytes=live * case["V"] * size + case["N"] * (case["B"] * 5 + case["K"] * 13), flops=4 * live * case["V"])
    if case["op"] == "move":
        rows = case["N"] * case["B"]
        if case["place"] == "in":
            rows = case["N"] * (max(1, int(case["B"] * case["moved"])) if case["B"] > 1 else 0)
        moved = 0.75 * case["L"] * (4 + case["caches"] * case["heads"] * case["D"] * size) + case["recurrent"] * size
        return dict(bytes=max(8.0, 2 * rows * moved), flops=0)
    frames = case["N"] * (case["T_lo"] + case["T_hi"]) / 2
    return dict(bytes=frames * case["k"] * 8 + case["N"] * case["B"] * (case["T_hi"] * 4 + 8),
                flops=frames * case["B"] * (case["k"] + 1) * 4)


# ---------------------------------------------------------------------------------------------
# The same in 64 bits on the host, written from the definitions
# ---------------------------------------------------------------------------------------------

def _host(t):
    return t.detach().float().cpu().numpy().astype(np.float64) if t.is_floating_point() else t.cpu().numpy()


def _exact_clip(case, s):
    squares = 0.0
    for t in s["grads"]:
        v = _host(t)
        squares += float(np.dot(v, v))
    norm = math.sqrt(squares)
    factor = min(1.0, s["max_norm"] / (norm + 1e-6)) if math.isfinite(norm) else 1.0
    return dict(norm=np.array([norm]), grads=_host(s["flat"]) * factor)      # the gaps between tensors are zero


def _exact_select(case, s):
    N, B, V = s["logits"].shape
    best = np.full((N, case["K"]), -np.inf)
    for n in range(N):
        x, sc = _host(s["logits"][n]), _host(s["scores"][n])
        found = []
        for b in range(B):
            if s["finished"] is not None and bool(s["finished"][n, b]):
                found.append(np.array([sc[b]]))
                continue
            top = x[b].max()
            lse = top + math.log(np.exp(x[b] - top).sum())
            row = x[b] if V <= case["K"] else np.partition(x[b], V - case["K"])[V - case["K"]:]
            found.append(sc[b] + (row - lse))
        found = np.sort(np.concatenate(found))[::-1][: case["K"]]
        best[n, : found.size] = found
    return dict(scores=best, parents=None, tokens=None, finished=None, flags=None)


def _exact_move(case, s):
    rows, lens = _host(s["parents"]), _host(s["lengths"])
    result = []
    for i, (x, axis) in enumerate(zip(s["states"], s["axes"])):
        if not x.is_floating_point():
            result.append(None)
            continue
        v = _host(x)
        o = v.copy() if s["out"] is None else np.zeros_like(v)
        for n in range(v.shape[0]):
            for b in range(rows.shape[1]):
                if axis is None:
                    o[n, b] = v[n, rows[n, b]]
                else:
                    o[n, b, :, : lens[n]] = v[n, rows[n, b], :, : lens[n]]
        result.append(o)
    return result


def _exact_prefix(case, s):
    """The search over dictionaries of prefixes, one utterance at a time; a prefix is a node of a tree of labels."""
    cls, lp = _host(s["classes"]), _host(s["logprobs"])
    scores = np.full((case["N"], s["B"]), -np.inf)
    for n in range(case["N"]):
        nodes, ends = {}, {0: None}
        beams = [(0, 1.0, 0.0)]                       # node, probability ending in blank, ending in a label
        log_scale = 0.0
        for t in range(s["lengths"][n]):
            shift = lp[n, t].max()
            p = [(int(c), math.exp(v - shift)) for c, v in zip(cls[n, t], lp[n, t])]
            found = {}
            for node, b, l in beams:
                here = found.setdefault(node, [0.0, 0.0])
                for c, q in p:
                    if c == s["blank"]:
                        here[0] += (b + l) * q
                        continue
                    if c == ends[node]:
                        here[1] += l * q
                    child = nodes.setdefault((node, c), len(nodes) + 1)
                    ends[child] = c
                    found.setdefault(child, [0.0, 0.0])[1] += (b if c == ends[node] else b + l) * q
            kept = sorted(found.items(), key=lambda e: -(e[1][0] + e[1][1]))[: s["B"]]
            top = kept[0][1][0] + kept[0][1][1]
            beams = [(node, b / top, l / top) for node, (b, l) in kept if b + l > 0]
            log_scale += shift + math.log(top)
        for i, (_, b, l) in enumerate(beams):
            scores[n, i] = math.log(b + l) + log_scale
    return dict(tokens=None, token_lengths=None, scores=scores, flags=None)


def exact(case, seed):
    s = prepare(case, seed)
    return dict(clip=_exact_clip, select=_exact_select, move=_exact_move, prefix=_exact_prefix)[case["op"]](case, s)
