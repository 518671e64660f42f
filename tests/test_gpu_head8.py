"""The head in 8-bit integers on the GPU: quantization bit by bit, products against whole numbers.

Tolerances: a product's sum is exact; it is rounded to fp32, multiplied by the product of the scales (two roundings) and added to
the bias in one operation: 3 * 2^-24 of the product and 2^-24 of the result, then rounded to the type (bf16 2^-8)."""

import ctypes

import pytest
import torch

from paper_2609_33645_b200 import binding, workloads as wl

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 2.0 ** -24
HALF = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8}
BF, FP = torch.bfloat16, torch.float32


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def quantized(x):
    """The definition: fp32 divisions by tensors (correctly rounded), products and roundings to even."""
    x = x.float()
    top = x.abs().amax(-1)
    most = torch.full_like(top, 127.0)
    inv = most / top
    q = torch.round(x * inv[:, None]).clamp(-127, 127)
    zero = top < 2.0 ** -100
    return torch.where(zero[:, None], 0.0, q).to(torch.int8), torch.where(zero, 0.0, top / most)


@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (1, 8), (37, 64), (9, 250), (5, 256), (4, 512), (3, 1000), (2, 1024), (3, 2048),
                                       (3, 2056), (2, 4096), (2, 5120), (2, 8192), (2, 8200), (2, 30_000), (3001, 72)])
@pytest.mark.parametrize("dtype", [BF, FP])
def test_quantization(rows, cols, dtype):
    x = (torch.randn(rows, cols, generator=gen(1), device=DEV) * torch.logspace(-6, 6, rows, device=DEV)[:, None]).to(dtype)
    q, s = binding.quantize_rows(x)
    wq, ws = quantized(x)
    assert torch.equal(q, wq) and torch.equal(s, ws) and int(q.abs().max()) == 127
    assert q.stride(0) % 16 == 0 and q.data_ptr() % 16 == 0
    buf = torch.randn(rows, cols + 5, generator=gen(2), device=DEV).to(dtype)
    for view in (buf[:, :cols], buf[:, 3:3 + cols]):                # other strides, other alignment
        q, s = binding.quantize_rows(view)
        wq, ws = quantized(view)
        assert torch.equal(q, wq) and torch.equal(s, ws)


@pytest.mark.parametrize("cols", [40, 33, 9000])
def test_rows_of_zeros_of_tiny_and_of_values_that_are_not_finite(cols):
    x = torch.randn(7, cols, generator=gen(1), device=DEV)
    x[1], x[2], x[3, 5], x[4, 7], x[5] = 0.0, 1e-38, float("nan"), float("-inf"), x[5] * 1e-30
    x[6, 0] = torch.finfo(FP).max
    q, s = binding.quantize_rows(x)
    assert not q[1:5].any() and s[1] == 0 and s[2] == 0 and bool(s[3].isnan()) and bool(s[4].isnan())
    wq, ws = quantized(x)
    for i in (0, 5, 6):
        assert torch.equal(q[i], wq[i]) and torch.equal(s[i], ws[i])


def pair(m, n, k, seed=1):
    out = []
    for i, r in enumerate((m, n)):
        q = torch.zeros(r, (k + 15) // 16 * 16, dtype=torch.int8, device=DEV)
        q[:] = 99                                                 # what lies behind a row's k values does not count
        q[:, :k] = torch.randint(-128, 128, (r, k), generator=gen(seed + i), device=DEV, dtype=torch.int32).to(torch.int8)
        out.append(binding.QuantizedHead(q[:, :k], torch.rand(r, generator=gen(seed + 2 + i), device=DEV) + 0.1))
    return out


def product(a, b, bias=None):
    part = (a.q.double() @ b.q.double().T) * a.scales.double()[:, None] * b.scales.double()
    return part, part if bias is None else part + bias.double()


def check(got, part, want):
    near = 3.01 * EPS * part.abs() + EPS * want.abs()
    assert bool(((got.double() - want).abs() <= near + HALF[got.dtype] * (want.abs() + near)).all())


@pytest.mark.parametrize("m", [1, 2, 15, 16, 17, 31, 32, 33, 64, 97, 127, 128, 129, 200, 256, 257, 513])
@pytest.mark.parametrize("n,k", [(1, 1), (31, 16), (127, 31), (128, 128), (129, 129), (255, 33), (257, 1000), (1000, 500), (2305, 256)])
def test_products(m, n, k):
    a, b = pair(m, n, k)
    for i, dtype in enumerate((FP, BF)):
        bias = None if (m + n + i) % 3 == 0 else torch.randn(n, generator=gen(9), device=DEV).to(BF if (m + i) % 2 else FP) * 100
        word = torch.zeros(1, dtype=torch.int32, device=DEV)
        got = binding.matmul_i8(a, b, bias=bias, dtype=dtype, status=word)
        assert got.shape == (m, n) and got.dtype == dtype and int(word) == 0
        check(got, *product(a, b, bias))


@pytest.mark.parametrize("m,n,k", [(4, 20_000, 1024), (700, 5000, 5120), (1500, 9000, 64)])
def test_products_of_many_tiles(m, n, k):
    a, b = pair(m, n, k, 5)
    for dtype in (FP, BF):
        check(binding.matmul_i8(a, b, dtype=dtype), *product(a, b))


def test_the_longest_sums_are_exact():
    k = 131_071
    for m in (3, 300):
        a = binding.QuantizedHead(torch.full((m, k + 1), -128, dtype=torch.int8, device=DEV)[:, :k], torch.ones(m, device=DEV))
        b = binding.QuantizedHead(torch.full((5, k + 1), -128, dtype=torch.int8, device=DEV)[:, :k], torch.ones(5, device=DEV))
        a.q[1], b.q[2, ::2] = 127, 127
        got = binding.matmul_i8(a, b)
        assert torch.equal(got, (a.q.double() @ b.q.double().T).float())


def test_rows_of_the_result_may_lie_apart():
    for m, n in ((5, 37), (130, 300)):
        a, b = pair(m, n, 96)
        for dtype, ld in ((FP, n + 5), (BF, n + 4), (BF, n + 5)):
            C = torch.full((m + 1, ld), 7.0, device=DEV, dtype=dtype)
            p = binding.I8Problem(m, n, 96, int(dtype == FP), a.q.stride(0), b.q.stride(0), ld, 0, 0)
            stream = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
            vp = lambda t: ctypes.c_void_p(t.data_ptr())         # noqa: E731
            assert binding.load().pctc_i8_matmul(ctypes.byref(p), vp(a.q), vp(a.scales), vp(b.q), vp(b.scales), None, vp(C), None, stream) == 0
            check(C[:m, :n], *product(a, b))
            assert bool((C[:, n:] == 7).all()) and bool((C[m] == 7).all())


@pytest.mark.parametrize("m", [1, 16, 17, 127, 128, 129, 130, 256, 257, 600, 768, 769, 8192])
@pytest.mark.parametrize("k", [1, 8, 10, 31, 63, 64])
def test_short_rows(m, k):
    """Few values, and yet more tokens than a tile of few tokens holds."""
    hidden = torch.randn(m, k, generator=gen(m), device=DEV)
    head = binding.quantize_rows(torch.randn(300, k, generator=gen(k), device=DEV))
    got = binding.quantized_logits(hidden, head)
    check(got, *product(binding.QuantizedHead(*quantized(hidden)), head))


def test_a_workspace_that_is_too_small_is_refused():
    head = binding.quantize_rows(torch.randn(300, 64, generator=gen(1), device=DEV))
    with pytest.raises(binding.PctcError) as e:
        binding.quantized_logits(torch.randn(200, 64, device=DEV), head, workspace=torch.empty(4096, dtype=torch.uint8, device=DEV))
    assert e.value.status == 2


def test_scales_that_are_not_finite_spoil_their_rows_and_channels_alone():
    x, W = torch.randn(6, 64, generator=gen(1), device=DEV), torch.randn(200, 64, generator=gen(2), device=DEV)
    x[2, 3], W[100, 5] = float("nan"), float("inf")
    y = binding.quantized_logits(x, binding.quantize_rows(W))
    bad = y.isnan()
    assert bool(bad[2].all()) and bool(bad[:, 100].all()) and int(bad.sum()) == 200 + 6 - 1


@pytest.mark.parametrize("shape,V,D", [((4,), 151936, 1024), ((2, 3), 999, 516), ((1, 1), 50_001, 64), ((3, 70), 3001, 333), ((0,), 100, 64)])
@pytest.mark.parametrize("dtype,out", [(BF, FP), (FP, BF), (BF, BF)])
def test_logits(shape, V, D, dtype, out):
    hidden = torch.randn(*shape, D, generator=gen(1), device=DEV).to(dtype)
    head = binding.quantize_rows(torch.randn(V, D, generator=gen(2), device=DEV) * D ** -0.5)
    bias = torch.randn(V, generator=gen(3), device=DEV).to(dtype)
    ws = torch.full((hidden.numel() * 2 + 8192,), 255, dtype=torch.uint8, device=DEV)
    got = binding.quantized_logits(hidden, head, bias=bias, dtype=out, workspace=ws)
    assert got.shape == (*shape, V) and got.dtype == out
    if hidden.numel():
        states = binding.QuantizedHead(*quantized(hidden.view(-1, D)))
        check(got.view(-1, V), *product(states, head, bias))
        assert binding.workspace_status(ws) == 0
        wide = torch.zeros(*shape, D + 7, device=DEV, dtype=dtype)
        wide[..., 4:4 + D] = hidden
        assert torch.equal(binding.quantized_logits(wide[..., 4:4 + D], head, bias=bias, dtype=out), got)


def test_results_and_heads_of_more_than_2_31_bytes():
    a, b = pair(16_000, 151_936, 32, 3)
    C = binding.matmul_i8(a, b, dtype=BF)
    assert C.numel() > 2 ** 31
    rows = torch.tensor([0, 8000, 14_135, 15_999], device=DEV)
    few = binding.QuantizedHead(a.q[rows], a.scales[rows])
    check(C[rows], *product(few, b))
    del C
    V, D = 140_000, 16_384
    head = binding.QuantizedHead(torch.randint(-127, 128, (V, D), device=DEV, dtype=torch.int8), torch.ones(V, device=DEV))
    x = torch.randint(-127, 128, (3, D), device=DEV, dtype=torch.int8)
    got = binding.matmul_i8(binding.QuantizedHead(x, torch.ones(3, device=DEV)), head)
    at = torch.tensor([0, 131_071, 131_073, V - 1], device=DEV)
    assert torch.equal(got[:, at], (x.double() @ head.q[at].double().T).float())


def test_captured_into_a_graph_and_on_another_stream():
    for m in (5, 300):
        hidden = torch.randn(m, 96, generator=gen(1), device=DEV)
        head = binding.quantize_rows(torch.randn(700, 96, generator=gen(2), device=DEV))
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            first = binding.quantized_logits(hidden, head)
        torch.cuda.synchronize()
        assert torch.equal(first, binding.quantized_logits(hidden, head))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y = binding.quantized_logits(hidden, head)
        for seed in (3, 4):
            hidden.copy_(torch.randn(m, 96, generator=gen(seed), device=DEV))
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(y, binding.quantized_logits(hidden, head))


@pytest.mark.parametrize("dtype,D,V,k,chunk", [(BF, 64, 3001, 8, 0), (FP, 50, 500, 4, 128), (BF, 200, 9000, 1, 4096), (FP, 128, 5, 8, 0)])
def test_best_classes_of_every_frame(dtype, D, V, k, chunk):
    N, T, lengths = 3, 50, [50, 1, 33]
    hidden = torch.randn(N, T, D, generator=gen(1), device=DEV).to(dtype)
    head = binding.quantize_rows(torch.randn(V, D, generator=gen(2), device=DEV) * 3 * D ** -0.5)
    bias = torch.randn(V, generator=gen(3), device=DEV).to(dtype)
    r = binding.topk_decode(hidden, head, bias, lengths, k, chunk=chunk)
    assert binding.workspace_status(r["workspace"]) == 0
    states = binding.QuantizedHead(*quantized(hidden.view(-1, D)))
    _, z = product(states, head, bias)
    z = z.view(N, T, V)
    lp = torch.log_softmax(z, -1)
    for n, t in enumerate(lengths):
        got, val = r["classes"][n, :t].long(), r["logprobs"][n, :t].double()
        kk = min(k, V)
        # fp32 logits may swap classes that are nearer than their rounding: compare values
        picked = lp[n, :t].gather(1, got[:, :kk])
        best = lp[n, :t].topk(kk, dim=1).values
        size = z[n, :t].abs().amax(1, keepdim=True)
        # a logit: 4 roundings; the log-sum-exp of fp32 exponentials and its subtraction: 1e-5 absolute is 80 roundings
        assert bool(((picked - best).abs() <= 8 * EPS * size).all())
        assert bool(((val[:, :kk] - picked).abs() <= 1e-5 + 16 * EPS * size).all())
        assert bool((got[:, kk:] == -1).all()) and bool((r["classes"][n, t:] == -1).all())


def test_prefix_search_with_the_head_in_8_bits():
    batch = wl.make_batch(wl.reduced(wl.CONFIGS["c2"], name="i8", V=2048, D=128, N=4, T_div=8, U_div=2), permute_ids=True)
    hidden = torch.from_numpy(batch.hidden).to(DEV).to(BF)
    head = binding.quantize_rows(torch.from_numpy(batch.W).to(DEV))
    r = binding.beam_decode(hidden, head, None, batch.input_lengths, batch.blank, 4)
    best = binding.topk_decode(hidden, head, None, batch.input_lengths, 8)
    want = binding.prefix_beam_decode(best["classes"], best["logprobs"], batch.input_lengths, batch.blank, 4)
    assert torch.equal(r["tokens"], want["tokens"]) and torch.equal(r["scores"], want["scores"])


def test_a_decoding_loop():
    """Lookup, states, the head in 8 bits, selection and reordering, a step at a time, against the same in 64 bits."""
    N, B, V, D = 3, 4, 4001, 64
    W = torch.randn(V, D, generator=gen(1), device=DEV) * D ** -0.5
    head = binding.quantize_rows(W)
    mix = torch.randn(D, D, generator=gen(2), device=DEV) * D ** -0.5
    state = torch.randn(N, B, D, generator=gen(3), device=DEV)
    scores = torch.full((N, B), float("-inf"), device=DEV)
    scores[:, 0] = 0.0
    tokens = torch.zeros(N, B, dtype=torch.int32, device=DEV)
    for _ in range(4):
        x = binding.embed(tokens, head, scale=D ** 0.5, dtype=FP)
        deq = torch.where((tokens >= 0)[..., None], head.q[tokens.clamp(min=0).long()].float() * head.scales[tokens.clamp(min=0).long()][..., None], 0.0)
        assert bool(((x - deq * D ** 0.5).abs() <= 4 * EPS * x.abs()).all())
        state = torch.tanh(state @ mix + x)
        logits = binding.quantized_logits(state, head, dtype=FP)
        states = binding.QuantizedHead(*quantized(state.view(-1, D)))
        check(logits.view(-1, V), *product(states, head))
        sel = binding.beam_select(logits, scores, B)
        cand = (scores.double()[..., None] + torch.log_softmax(logits.double(), -1)).view(N, -1).topk(B)
        assert torch.equal(sel["parents"].long(), cand.indices // V) and torch.equal(sel["tokens"].long(), cand.indices % V)
        binding.beam_reorder([state], sel["parents"])
        scores, tokens = sel["scores"], sel["tokens"]


def test_refusals():
    a, b = pair(3, 40, 64)
    x = torch.zeros(3, 64, device=DEV)
    H = binding.QuantizedHead
    for bad in (H(b.q.int(), b.scales), H(b.q, b.scales[:5]), H(b.q, b.scales.double()), H(b.q[:, :48], b.scales), H(b.q.cpu(), b.scales),
                H(b.q.t(), b.scales)):
        with pytest.raises(ValueError):
            binding.quantized_logits(x, bad)
        with pytest.raises(ValueError):
            binding.matmul_i8(a, bad)
    shifted = torch.zeros(40, 80, dtype=torch.int8, device=DEV)[:, 8:72]          # rows that do not start on 16 bytes
    tight = torch.zeros(40 * 65, dtype=torch.int8, device=DEV).view(40, 65)[:, :64]
    for q in (shifted, tight):
        with pytest.raises(binding.PctcError):
            binding.quantized_logits(x, H(q, b.scales))
    for kw in (dict(bias=torch.zeros(39, device=DEV)), dict(bias=torch.zeros(40, device=DEV).half()), dict(dtype=torch.float16)):
        with pytest.raises(ValueError):
            binding.quantized_logits(x, b, **kw)
    with pytest.raises(TypeError):
        binding.quantized_logits(x, b, dtype="bf16")


def test_a_wait_that_runs_out_is_reported_and_the_kernel_returns(lib):
    """In the test build whose waits give up after 3,000 cycles, a long contraction cannot finish its first tile in time."""
    from paper_2609_33645_b200 import build
    short = lib.load_variant(build.build_variant("shortwait"))
    vp = lambda t: ctypes.c_void_p(t.data_ptr())                  # noqa: E731
    for m in (16, 256):
        a, b = pair(m, 256, 32_768)
        C = torch.zeros(m, 256, device=DEV)
        word = torch.zeros(64, dtype=torch.int32, device=DEV)
        stream = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
        p = binding.I8Problem(m, 256, 32_768, 1, 32_768, 32_768, 256, 0, 0)
        assert short.pctc_i8_matmul(ctypes.byref(p), vp(a.q), vp(a.scales), vp(b.q), vp(b.scales), None, vp(C), vp(word), stream) == 0
        host = ctypes.c_int32(0)
        assert short.pctc_workspace_status(vp(word), stream, ctypes.byref(host)) == 6 and host.value in (1, 2, 3, 4)
        torch.cuda.synchronize()                                  # the kernel has returned and the context is intact
        check(binding.matmul_i8(a, b), *product(a, b))


def test_a_checked_product_is_the_product():
    x, head = torch.randn(3, 64, generator=gen(1), device=DEV), binding.quantize_rows(torch.randn(300, 64, generator=gen(2), device=DEV))
    for states in (x, x.repeat(100, 1), x[:0]):
        assert torch.equal(binding.quantized_logits(states, head, check_status=True), binding.quantized_logits(states, head))
    a, b = pair(30, 300, 64)
    word = torch.zeros(1, dtype=torch.int32, device=DEV)
    assert torch.equal(binding.matmul_i8(a, b, check_status=True), binding.matmul_i8(a, b))
    assert torch.equal(binding.matmul_i8(a, b, status=word, check_status=True), binding.matmul_i8(a, b))
    word.fill_(3)                                                 # as a wait that gave up leaves it
    with pytest.raises(binding.PctcError) as e:
        binding.matmul_i8(a, b, status=word, check_status=True)
    assert e.value.status == 6


@pytest.mark.parametrize("m,n,k,dtype", [
    (16, 256, 32_768, FP), (256, 256, 32_768, BF),                # behind their quantization, one CTA and a pair
    (1, 128, 6016, FP), (1, 128, 6016, BF)])                      # one CTA that quantizes its token itself
def test_logits_report_a_wait_that_runs_out_whatever_the_status_word_held(lib, m, n, k, dtype):
    """As above: 47 blocks of k take an SM some 12,000 cycles at 64 bytes a cycle, 256 take more, and the limit is 3,000."""
    from paper_2609_33645_b200 import build
    short = lib.load_variant(build.build_variant("shortwait"))
    vp = lambda t: ctypes.c_void_p(t.data_ptr())                  # noqa: E731
    x = torch.randn(m, k, generator=gen(1), device=DEV).to(dtype)
    head = binding.quantize_rows(torch.randn(n, k, generator=gen(2), device=DEV))
    C = torch.zeros(m, n, device=DEV)
    p = binding.I8Problem(m, n, k, 1, k, head.q.stride(0), n, 0, 0)
    stream = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    ws = torch.full((2 * m * (k + 128) + 8192,), 255, dtype=torch.uint8, device=DEV)
    for _ in range(5):
        assert short.pctc_i8_logits(ctypes.byref(p), vp(x), int(dtype == FP), vp(head.q), vp(head.scales), None, vp(C), vp(ws),
                                    ctypes.c_size_t(ws.numel()), stream) == 0
        host = ctypes.c_int32(0)
        assert short.pctc_workspace_status(vp(ws), stream, ctypes.byref(host)) == 6 and host.value in (1, 2, 3, 4)
        torch.cuda.synchronize()                                  # the kernel has returned and the context is intact
    check(binding.quantized_logits(x, head, dtype=FP, check_status=True), *product(binding.QuantizedHead(*quantized(x)), head))


@pytest.mark.parametrize("dtype,V,beams", [(FP, 1000, 4), (BF, 3001, 6)])
def test_recognition_in_8_bits_against_64_bits_and_the_oracles_search(dtype, V, beams):
    """The best classes of the product in 64 bits and a search on the host.  A log-probability is within 1e-5 + 16 EPS of the
    largest logit (as above), a score within that for each of its frames.  A frame's log-sum-exp shifts all its classes, and all
    hypotheses, alike; what may change an order are the logits' four roundings and that of the subtraction, on both sides: 10 EPS."""
    from oracle import pruned_ctc_oracle as O
    lengths, D, blank = [25, 9, 1], 64, 0
    hidden = torch.randn(3, 25, D, generator=gen(3), device=DEV).to(dtype)
    head = binding.quantize_rows((torch.randn(V, D, generator=gen(4), device=DEV) / 4).to(dtype))
    bias = torch.randn(V, generator=gen(5), device=DEV).to(dtype)
    bias[blank] += 6.0
    got = binding.beam_decode(hidden, head, bias, lengths, blank, beams, k=8)
    assert binding.workspace_status(got["workspace"]) == 0
    _, z = product(binding.QuantizedHead(*quantized(hidden.view(-1, D))), head, bias)
    best = torch.log_softmax(z, -1).view(3, 25, V).topk(9)
    near, apart = 1e-5 + 16 * EPS * float(z.abs().max()), 10 * EPS * float(z.abs().max())
    for n, T in enumerate(lengths):
        val = best.values[n, :T]
        assert bool((val[:, :-1] - val[:, 1:] > apart).all())     # the eight are in no doubt, nor is their order
        classes, logprobs = best.indices[n, :T, :8].int().cpu().numpy(), val[:, :8].float().cpu().numpy()
        want, bad = O.prefix_beam_search(classes, logprobs, T, blank, beams + 1)
        want = want[:beams + 1]
        assert not bad and len(want) > 1 and all(a[1] - b[1] > T * apart for a, b in zip(want, want[1:]))
        exact, _ = O.prefix_beam_search(classes, logprobs, T, blank, beams)
        for b in range(min(beams, len(exact))):
            labels, score = exact[b]
            assert got["tokens"][n, b, : len(labels)].tolist() == labels and int(got["token_lengths"][n, b]) == len(labels)
            assert abs(float(got["scores"][n, b]) - score) <= T * near + 2.0 ** -22 * abs(score)
