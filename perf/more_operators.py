"""What is measured of the operators around the head's matrix and the loss: what feeds the head, what weighs its loss, and
the head in 8 bits.

Five operators, each once in elementary torch operations (``own`` false) and once through the package's
binding (``own`` true):

  embed    rows of the vocabulary matrix for tokens, scaled; the matrix in bf16 or fp32, or in 8 bits with a scale a row
  scatter  the gradient of that lookup with respect to the whole matrix
  dropout  zeroing by a counter-based generator, alone or with a residual
  policy   clipped policy loss over log-probabilities with a KL term, and its gradient
  head8    logits of the head in 8-bit integers, the states quantized a row at a time

``listed()`` and ``draw()`` give cases, ``prepare()`` their inputs, ``run()`` one pass, ``work()`` the
bytes and operations of a pass, ``exact()`` the results in 64 bits on the host.
"""

import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
TINY = 2.0 ** -100                     # rows whose largest value is below this are quantized as zeros


# ---------------------------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------------------------

def listed():
    return [
        # A step of beam search: the chosen tokens of 16 utterances with 4 beams, from the head in 8 bits.
        dict(name="embed 16x4 from 8 bits", op="embed", table="int8", dtype="bf16", M=64, V=151936, D=1024, scale=1.0, none=0.05),
        # The targets of a training batch (padded with -1) from a bf16 matrix, scaled by sqrt(D).
        dict(name="embed 64x512", op="embed", table="bf16", dtype="bf16", M=32768, V=151936, D=2560, scale=2560 ** 0.5, none=0.2),
        # A small vocabulary in fp32 with odd sizes.
        dict(name="scatter odd fp32", op="scatter", dtype="fp32", M=1999, V=5_003, D=510, scale=1.0, none=0.1, zipf=1.0),
        # A training batch into the gradient of the full-vocabulary matrix; tokens as frequent as in text.
        dict(name="scatter 64x512", op="scatter", dtype="bf16", M=32768, V=151936, D=1024, scale=1.0, none=0.2, zipf=1.0),
        # One second of speech in front of the head.
        dict(name="dropout 25x512 fp32", op="dropout", dtype="fp32", rows=25, cols=512, p=0.1, residual=False),
        # 640 utterances of 100 frames, added to the residual.
        dict(name="dropout 64000x1024", op="dropout", dtype="bf16", rows=64000, cols=1024, p=0.1, residual=True),
        # Losses of sampled hypotheses: one log-probability a sequence, as the CTC loss gives it.
        dict(name="policy 64 sequences", op="policy", N=64, T=1, ref=False, mask=False, lengths=False, each=False, kl=0.0,
             reduction="sequences", negated=True),
        # A batch of sampled transcripts, ragged, weighted by token.
        dict(name="policy 128x501 ragged", op="policy", N=128, T=501, ref=True, mask=False, lengths=True, each=False, kl=0.05,
             reduction="tokens", negated=False),
        # Long answers with a mask and advantages of their own for every token.
        dict(name="policy 256x4096", op="policy", N=256, T=4096, ref=True, mask=True, lengths=False, each=True, kl=0.02,
             reduction="sequences", negated=False),
        # A step of beam search with one utterance and 4 beams.
        dict(name="head8 4 rows", op="head8", dtype="bf16", out="fp32", M=4, V=151936, D=1024, bias=False),
        # A portion of streamed frames, with odd sizes and a bias.
        dict(name="head8 37 rows odd", op="head8", dtype="fp32", out="fp32", M=37, V=50_001, D=516, bias=True),
        # The frames of a batch against the full-vocabulary head.
        dict(name="head8 2048 rows", op="head8", dtype="bf16", out="bf16", M=2048, V=151936, D=4096, bias=False),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, hi):
    """A row's length: mostly a multiple of 64, sometimes any."""
    d = _log_int(rng, 64, hi)
    return d // 64 * 64 if rng.random() < 0.7 else d


def draw(rng):
    op = rng.choice(["embed", "scatter", "dropout", "policy", "head8"])
    dtype = rng.choice(["bf16", "fp32"])
    if op in ("embed", "scatter"):
        V = _log_int(rng, 500, 180_000)
        D = _width(rng, min(5120, 400_000_000 // V))
        M = _log_int(rng, 1, max(1, min(65_536, 80_000_000 // D)))
        c = dict(op=op, dtype=dtype, M=M, V=V, D=D, scale=rng.choice([1.0, D ** 0.5]), none=rng.choice([0.0, 0.2]))
        if op == "embed":
            return dict(c, table=rng.choice(["bf16", "fp32", "int8"]))
        return dict(c, zipf=rng.choice([0.0, 0.7, 1.0, 1.3]))
    if op == "dropout":
        cols = _width(rng, 5120)
        return dict(op=op, dtype=dtype, rows=_log_int(rng, 1, 60_000_000 // cols), cols=cols,
                    p=rng.choice([0.05, 0.1, 0.3, 0.5]), residual=rng.random() < 0.5)
    if op == "policy":
        T = rng.choice([1, _log_int(rng, 2, 8192), _log_int(rng, 2, 8192)])
        ref = rng.random() < 0.6
        return dict(op=op, N=_log_int(rng, 1, max(1, min(4096, 1_000_000 // T))), T=T, ref=ref, mask=rng.random() < 0.5,
                    lengths=rng.random() < 0.5, each=rng.random() < 0.3, kl=rng.choice([0.01, 0.1]) if ref else 0.0,
                    reduction=rng.choice(["tokens", "sequences", "sum"]), negated=rng.random() < 0.3)
    V = _log_int(rng, 500, 180_000)
    D = _width(rng, min(5120, 600_000_000 // V))
    M = _log_int(rng, 1, max(1, min(4096, 600_000_000 // V, 1_200_000_000_000 // (V * D))))
    return dict(op=op, dtype=dtype, out=rng.choice(["bf16", "fp32"]) if M * V < 300_000_000 else "bf16", M=M, V=V, D=D,
                bias=rng.random() < 0.5)


# ---------------------------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------------------------

def _tokens(case, g, zipf):
    """Token ids as frequent as 1 / rank^zipf, each rank a token of its own; -1 where there is none."""
    M, V = case["M"], case["V"]
    u = torch.rand(M, generator=g, device="cuda", dtype=torch.float64)
    if zipf == 1.0:
        rank = torch.exp(u * math.log(V)) - 1
    else:
        rank = (u * (float(V) ** (1 - zipf) - 1) + 1) ** (1 / (1 - zipf)) - 1
    rank = rank.long().clamp(0, V - 1)
    tokens = torch.randperm(V, generator=g, device="cuda")[rank]
    return torch.where(torch.rand(M, generator=g, device="cuda") < case["none"], -1, tokens).int()


def _quantized(w):
    """Rows in 8 bits: q = round(w * (127 / max|w|)), scale = max|w| / 127.  Rows of q start 16-byte aligned."""
    V, D = w.shape
    q = torch.zeros(V, (D + 15) // 16 * 16, dtype=torch.int8, device=w.device)[:, :D]
    q8, scales = _quantize(w.float())
    q.copy_(q8)
    return q, scales


def _quantize(x):
    top = x.abs().amax(-1)
    zero, most = top < TINY, torch.full_like(top, 127.0)          # a tensor: torch divides by a number only nearly
    inv = torch.where(zero, torch.zeros_like(top), most / top)
    return torch.round(x * inv[:, None]).clamp(-127, 127), torch.where(zero, torch.zeros_like(top), top / most)


def _prepare_embed(case, g):
    W = torch.randn(case["V"], case["D"], generator=g, device="cuda").mul_(case["D"] ** -0.5)
    s = dict(tokens=_tokens(case, g, 0.0), scale=case["scale"], dtype=DTYPES[case["dtype"]], scales=None)
    if case["table"] == "int8":
        s["W"], s["scales"] = _quantized(W)
    else:
        s["W"] = W.to(DTYPES[case["table"]])
    return s


def _prepare_scatter(case, g):
    grad = torch.randn(case["M"], case["D"], generator=g, device="cuda").to(DTYPES[case["dtype"]])
    return dict(tokens=_tokens(case, g, case["zipf"]), grad=grad, V=case["V"], scale=case["scale"])


def _prepare_dropout(case, g):
    shape, dtype = (case["rows"], case["cols"]), DTYPES[case["dtype"]]
    x = torch.randn(shape, generator=g, device="cuda").to(dtype)
    residual = torch.randn(shape, generator=g, device="cuda").to(dtype) if case["residual"] else None
    seed = int(torch.randint(0, 2 ** 62, (1,), generator=g, device="cuda"))
    return dict(x=x, residual=residual, p=case["p"], seed=seed, offset=seed % 100_003)


def _prepare_policy(case, g):
    N, T = case["N"], case["T"]

    def rand(*shape):
        return torch.rand(*shape, generator=g, device="cuda")

    def randn(*shape):
        return torch.randn(*shape, generator=g, device="cuda")
    spread = 20.0 if T == 1 else 1.0
    old = -spread * -torch.log(rand(N, T).clamp(min=1e-6))
    new = old + 0.15 * randn(N, T) * (rand(N, T) < 0.8)           # some tokens have not moved since they were sampled
    ref = old + 0.3 * randn(N, T) if case["ref"] else None
    sign = -1.0 if case["negated"] else 1.0
    s = dict(logp=sign * new, old=sign * old, ref=None if ref is None else sign * ref, mask=None, lengths=None,
             adv=randn(N, T) if case["each"] else randn(N), kl=case["kl"], reduction=case["reduction"], negated=case["negated"])
    if case["lengths"]:
        s["lengths"] = (rand(N) * T + 1).int().clamp(max=T)
    if case["mask"]:
        s["mask"] = rand(N, T) < 0.7
        s["mask"][rand(N) < 0.05] = False                         # rows with nothing to learn from
    count = _counted(s)
    for name in ("logp", "old", "ref"):                           # what lies in uncounted places does not matter
        if s[name] is not None:
            s[name] = torch.where(count, s[name], torch.full_like(s[name], math.nan))
    return s


def _prepare_head8(case, g):
    W = torch.randn(case["V"], case["D"], generator=g, device="cuda").mul_(case["D"] ** -0.5)
    q, scales = _quantized(W)
    hidden = torch.randn(case["M"], case["D"], generator=g, device="cuda").to(DTYPES[case["dtype"]])
    bias = torch.randn(case["V"], generator=g, device="cuda").to(DTYPES[case["dtype"]]) if case["bias"] else None
    return dict(hidden=hidden, q=q, scales=scales, bias=bias, out=DTYPES[case["out"]])


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    make = dict(embed=_prepare_embed, scatter=_prepare_scatter, dropout=_prepare_dropout, policy=_prepare_policy,
                head8=_prepare_head8)[case["op"]]
    return dict(make(case, g), op=case["op"])


# ---------------------------------------------------------------------------------------------
# Plain forms
# ---------------------------------------------------------------------------------------------

def _plain_embed(s):
    t = s["tokens"].long()
    there = (t >= 0) & (t < s["W"].shape[0])
    at = torch.where(there, t, torch.zeros_like(t))
    x = s["W"][at].float()
    factor = torch.full_like(x[:, :1], s["scale"]) if s["scales"] is None else (s["scales"][at] * s["scale"])[:, None]
    return torch.where(there[:, None], x * factor, torch.zeros_like(x)).to(s["dtype"])


def _plain_scatter(s):
    t, g = s["tokens"].long(), s["grad"].float()
    there = (t >= 0) & (t < s["V"])
    dW = torch.zeros(s["V"] + 1, g.shape[1], device="cuda")
    dW.index_add_(0, torch.where(there, t, torch.full_like(t, s["V"])), g)
    return (dW[:-1] * s["scale"]).to(s["grad"].dtype)


def _philox_words(blocks, seed, offset):
    """Four 32-bit words for each block number: Philox-4x32 with 10 rounds (Salmon et al., 2011), counter (block, offset), key seed."""
    low = 0xFFFFFFFF
    c0, c1 = blocks & low, (blocks >> 32) & low
    c2, c3 = torch.full_like(blocks, offset & low), torch.full_like(blocks, offset >> 32 & low)
    k0, k1 = seed & low, seed >> 32 & low
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57                   # wrapped to 64 bits: both halves are right
        c0, c1, c2, c3 = (b >> 32 & low) ^ c1 ^ k0, b & low, (a >> 32 & low) ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return torch.stack([c0, c1, c2, c3], -1)


def _plain_dropout(s):
    x = s["x"]
    n = x.numel()
    words = _philox_words(torch.arange((n + 7) // 8, device="cuda"), s["seed"], s["offset"])
    halves = torch.stack([words & 0xFFFF, words >> 16], -1).reshape(-1)[:n].reshape(x.shape)
    limit = int(math.floor(s["p"] * 65536 + 0.5))
    y = torch.where(halves >= limit, x.float() * (65536 / (65536 - limit)), torch.zeros((), device="cuda"))
    return (y if s["residual"] is None else y + s["residual"].float()).to(x.dtype)


def _counted(s):
    N, T = s["logp"].shape
    count = torch.ones(N, T, dtype=torch.bool, device="cuda") if s["mask"] is None else s["mask"]
    if s["lengths"] is not None:
        count = count & (torch.arange(T, device="cuda") < s["lengths"][:, None])
    return count


def _plain_policy(s):
    # 64 bits: whether a ratio is clipped is a comparison, and the sums are long
    count = _counted(s)
    zero = torch.zeros((), dtype=torch.float64, device="cuda")
    sign = -1.0 if s["negated"] else 1.0
    new, old = (torch.where(count, sign * s[k].double(), zero) for k in ("logp", "old"))
    adv = s["adv"].double() if s["adv"].dim() == 2 else s["adv"].double()[:, None].expand(new.shape)
    r = torch.exp(new - old)
    clipped = count & (((adv > 0) & (r > 1.2)) | ((adv < 0) & (r < 0.8)))
    loss = torch.where(clipped, -adv * torch.clamp(r, 0.8, 1.2), -adv * r)
    grad = torch.where(clipped, zero, -adv * r)
    kl = torch.zeros_like(new)
    if s["ref"] is not None:
        d = torch.where(count, sign * s["ref"].double() - new, zero)
        kl = torch.expm1(d) - d
        loss, grad = loss + s["kl"] * kl, grad - s["kl"] * torch.expm1(d)
    rows = count.sum(1, keepdim=True)
    if s["reduction"] == "tokens":
        w = torch.ones_like(new) / count.sum().clamp(min=1)
    elif s["reduction"] == "sequences":
        w = 1.0 / (rows.clamp(min=1) * (rows > 0).sum().clamp(min=1)).expand(new.shape)
    else:
        w = torch.ones_like(new)
    total = count.sum().clamp(min=1)
    return dict(loss=torch.where(count, w * loss, zero).sum().float().reshape(1),
                grad=torch.where(count, sign * w * grad, zero).float(),
                kl=(torch.where(count, kl, zero).sum() / total).float().reshape(1),
                clipped=(clipped.sum() / total.double()).float().reshape(1), count=count.sum().int().reshape(1))


def _plain_head8(s):
    q, scale = _quantize(s["hidden"].float())
    # sums of 8-bit products pass 2^24: 64 bits
    acc = q.double() @ s["q"].double().T
    y = acc * scale.double()[:, None] * s["scales"].double()
    return (y if s["bias"] is None else y + s["bias"].double()).to(s["out"])


def run(s):
    if own:
        from paper_2609_33645_b200 import binding
        if s["op"] == "embed":
            table = s["W"] if s["scales"] is None else binding.QuantizedHead(s["W"], s["scales"])
            return binding.embed(s["tokens"], table, scale=s["scale"], dtype=s["dtype"])
        if s["op"] == "scatter":
            return binding.embed_grad(s["tokens"], s["grad"], s["V"], scale=s["scale"])["dW"]
        if s["op"] == "dropout":
            return binding.dropout(s["x"], s["p"], s["seed"], offset=s["offset"], residual=s["residual"])
        if s["op"] == "policy":
            r = binding.policy_loss(s["logp"], s["old"], s["adv"], ref_logp=s["ref"], mask=s["mask"], lengths=s["lengths"],
                                    clip=(0.2, 0.2), kl_weight=s["kl"], reduction=s["reduction"], negated=s["negated"])
            return dict(loss=r["loss"], grad=r["grad"], kl=r["kl"], clipped=r["clipped"], count=r["count"])
        return binding.quantized_logits(s["hidden"], binding.QuantizedHead(s["q"], s["scales"]), bias=s["bias"], dtype=s["out"])
    return dict(embed=_plain_embed, scatter=_plain_scatter, dropout=_plain_dropout, policy=_plain_policy,
                head8=_plain_head8)[s["op"]](s)


# ---------------------------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------------------------

def work(case):
    size = {"bf16": 2, "fp32": 4, "int8": 1}
    if case["op"] == "embed":
        rows = case["M"] * (1 - case["none"])
        row = case["D"] * size[case["table"]] + (4 if case["table"] == "int8" else 0)
        return dict(bytes=case["M"] * (4 + case["D"] * size[case["dtype"]]) + rows * row, flops=rows * case["D"])
    if case["op"] == "scatter":
        rows, item = case["M"] * (1 - case["none"]), size[case["dtype"]]
        return dict(bytes=case["M"] * 4 + rows * case["D"] * item + case["V"] * case["D"] * item, flops=rows * case["D"])
    if case["op"] == "dropout":
        n = case["rows"] * case["cols"]
        return dict(bytes=n * size[case["dtype"]] * (3 if case["residual"] else 2), flops=2 * n)
    if case["op"] == "policy":
        n = case["N"] * case["T"]
        part = (0.5 + 0.5 / case["T"] if case["lengths"] else 1.0) * (0.67 if case["mask"] else 1.0)
        read = part * n * 4 * (2 + case["ref"] + case["each"]) + n * case["mask"] + 4 * case["N"]
        return dict(bytes=read + n * 4, flops=30 * part * n)
    M, V, D = case["M"], case["V"], case["D"]
    return dict(bytes=M * D * size[case["dtype"]] + V * (D + 4) + V * size[case["dtype"]] * case["bias"] + M * V * size[case["out"]],
                flops=2 * M * V * D)


# ---------------------------------------------------------------------------------------------
# The same in 64 bits on the host, written from the definitions
# ---------------------------------------------------------------------------------------------

def _host(t):
    return t.detach().float().cpu().numpy().astype(np.float64) if t.is_floating_point() else t.cpu().numpy()


def _exact_embed(case, s):
    tokens, W = _host(s["tokens"]), s["W"]
    y = np.zeros((case["M"], case["D"]))
    live = np.flatnonzero(tokens >= 0)
    rows = torch.from_numpy(tokens[live].astype(np.int64)).to(W.device)
    y[live] = _host(W[rows]) * s["scale"]
    if s["scales"] is not None:
        y[live] *= _host(s["scales"][rows])[:, None]
    return y


def _exact_scatter(case, s):
    tokens, g = _host(s["tokens"]), _host(s["grad"])
    y = np.zeros((case["V"], case["D"]))
    live = np.flatnonzero(tokens >= 0)
    if live.size:
        live = live[np.argsort(tokens[live], kind="stable")]
        first = np.flatnonzero(np.diff(tokens[live], prepend=-1))
        y[tokens[live[first]]] = np.add.reduceat(g[live], first, axis=0) * s["scale"]
    return y


def _exact_dropout(case, s):
    x = _host(s["x"]).reshape(-1)
    mask32, lo16 = np.uint64(0xFFFFFFFF), np.uint64(0xFFFF)
    half = np.uint64(32)
    block = np.arange((x.size + 7) // 8, dtype=np.uint64)
    c = [block & mask32, block >> half, np.full_like(block, s["offset"] & 0xFFFFFFFF), np.full_like(block, s["offset"] >> 32)]
    key = [s["seed"] & 0xFFFFFFFF, s["seed"] >> 32]
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> half) ^ c[1] ^ np.uint64(key[0]), b & mask32, (a >> half) ^ c[3] ^ np.uint64(key[1]), a & mask32]
        key = [(key[0] + 0x9E3779B9) % 2 ** 32, (key[1] + 0xBB67AE85) % 2 ** 32]
    u = np.stack([v for w in c for v in (w & lo16, w >> np.uint64(16))], 1).reshape(-1)[: x.size]
    t = math.floor(case["p"] * 65536 + 0.5)
    y = np.where(u < t, 0.0, x * (65536.0 / (65536 - t)))
    if s["residual"] is not None:
        y = y + _host(s["residual"]).reshape(-1)
    return y.reshape(s["x"].shape)


def _exact_policy(case, s):
    N, T = case["N"], case["T"]
    new, old, adv = _host(s["logp"]), _host(s["old"]), _host(s["adv"])
    ref = None if s["ref"] is None else _host(s["ref"])
    if case["negated"]:
        new, old, ref = -new, -old, None if ref is None else -ref
    counts, sums, grad = np.zeros(N), np.zeros(N), np.zeros((N, T))
    kl_sum, clipped = 0.0, 0
    for n in range(N):
        take = np.arange(T) < (T if s["lengths"] is None else int(s["lengths"][n]))
        if s["mask"] is not None:
            take &= _host(s["mask"][n])
        at = np.flatnonzero(take)
        A = adv[n][at] if adv.ndim == 2 else np.full(at.size, adv[n])
        ratio = np.exp(new[n, at] - old[n, at])
        plain, cut = A * ratio, A * np.minimum(np.maximum(ratio, 0.8), 1.2)
        token = -np.minimum(plain, cut)
        grad[n, at] = np.where(plain <= cut, -plain, 0.0)
        clipped += int((plain > cut).sum())
        if ref is not None:
            gap = ref[n, at] - new[n, at]
            k = np.expm1(gap) - gap
            token += case["kl"] * k
            grad[n, at] -= case["kl"] * np.expm1(gap)
            kl_sum += k.sum()
        counts[n], sums[n] = at.size, token.sum()
    total = max(1.0, counts.sum())
    if case["reduction"] == "tokens":
        loss, grad = sums.sum() / total, grad / total
    elif case["reduction"] == "sequences":
        share = 1.0 / (np.maximum(counts, 1) * max(1, (counts > 0).sum()))
        loss, grad = (sums * share).sum(), grad * share[:, None]
    else:
        loss = sums.sum()
    return dict(loss=np.array([loss]), grad=-grad if case["negated"] else grad, kl=np.array([kl_sum / total]),
                clipped=np.array([clipped / total]), count=None)


def _exact_head8(case, s):
    if case["M"] * case["V"] * case["D"] > 1e11:
        return None
    x = s["hidden"].float().cpu().numpy()
    q = np.zeros(x.shape)
    scale = np.zeros(x.shape[0])
    for i, row in enumerate(x):
        top = np.abs(row).max()
        if top >= TINY:
            q[i] = np.clip(np.rint(row * (np.float32(127) / top)), -127, 127)
            scale[i] = np.float32(top) / np.float32(127)
    y = (q @ s["q"].cpu().numpy().astype(np.float64).T) * scale[:, None] * _host(s["scales"])
    return y if s["bias"] is None else y + _host(s["bias"])


def exact(case, seed):
    s = prepare(case, seed)
    return dict(embed=_exact_embed, scatter=_exact_scatter, dropout=_exact_dropout, policy=_exact_policy,
                head8=_exact_head8)[case["op"]](case, s)
