"""Beam selection on the GPU against the oracle in 64 bits on the same values.

Parents and tokens have to be equal wherever neighbouring candidates are further apart than the error of a score;
exact ties are ties on both sides.  That error: lse sums exponentials in fp32, each within about 2^-21 relative, and
a thread adds a few hundred of them (2^-24 each, partly cancelling): 1e-6 bounds it with room.  Scores come back rounded
to fp32: 2^-24 relative more."""

import math

import numpy as np
import pytest
import torch

from oracle import pruned_ctc_oracle as O
from paper_2609_33645_b200 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
LSE_TOL = 1e-6


def make(N, B, V, dtype, seed, scale=2.5, pad=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    full = (torch.randn(N, B, V + pad, generator=g, device=DEV) * scale).to(dtype)
    full[:, :, V:] = 1e4 if pad else 0                      # what lies behind a row may not be read as its part
    scores = -10 - 5 * torch.rand(N, B, generator=g, device=DEV)
    return full[:, :, :V], scores


def check(logits, scores, K, finished=None, eos=None):
    r = binding.beam_select(logits, scores, K, finished=finished, eos_id=eos)
    x, s = logits.float().cpu().numpy(), scores.cpu().numpy()
    f = None if finished is None else finished.cpu().numpy()
    out, parents, tokens, ended, flags = (r[q].cpu().numpy() for q in ("scores", "parents", "tokens", "finished", "flags"))
    skipped = 0
    for n in range(x.shape[0]):
        want, bad, near = O.beam_select(x[n], s[n], K, None if f is None else f[n], eos)
        assert flags[n] == (2 if bad else 0)
        for k in range(K):
            if k >= len(want):
                assert out[n, k] == -math.inf and parents[n, k] == -1 and tokens[n, k] == -1 and not ended[n, k]
                continue
            score, b, v = want[k]
            assert abs(float(out[n, k]) - score) <= LSE_TOL + 2.0 ** -23 * abs(score)
            if near > 2 * LSE_TOL:
                assert (parents[n, k], tokens[n, k]) == (b, v), (n, k)
            assert ended[n, k] == ((f is not None and f[n, parents[n, k]]) or (eos is not None and tokens[n, k] == eos))
        skipped += near <= 2 * LSE_TOL
    assert skipped <= max(1, x.shape[0] // 8)
    return r


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N,B,K,V,pad", [
    (1, 1, 1, 1, 0), (1, 1, 5, 1, 0), (2, 1, 4, 3, 0), (1, 4, 4, 255, 0), (3, 2, 7, 256, 0), (3, 4, 4, 257, 0),
    (2, 3, 3, 1000, 0), (2, 8, 8, 1000, 24), (1, 32, 32, 1000, 0), (5, 5, 10, 4099, 0), (2, 16, 16, 5000, 3),
    (1, 32, 32, 20001, 7), (9, 4, 4, 32768, 0), (1, 4, 4, 151936, 0), (4, 8, 8, 151936, 128), (2, 1, 32, 180000, 0),
    (20, 2, 2, 65537, 0), (1, 2, 2, 2 ** 21, 0), (1, 31, 32, 70000, 1),
])
def test_against_the_oracle(N, B, K, V, pad, dtype):
    logits, scores = make(N, B, V, dtype, V + B + K, pad=pad)
    check(logits, scores, K)


def test_the_widest_call():
    logits, scores = make(1, 32, 2 ** 21, torch.bfloat16, 1)
    r = binding.beam_select(logits, scores, 32)
    lse = torch.logsumexp(logits.double(), -1)
    cand = scores.double()[..., None] + (logits.double() - lse[..., None])
    want, _ = torch.sort(cand.reshape(1, -1), descending=True, stable=True)
    assert float((r["scores"].double() - want[:, :32]).abs().max()) <= LSE_TOL + 2.0 ** -23 * 40


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("scale", [0.0, 0.01, 30.0])
def test_ties_and_peaks(scale, dtype):
    """Rows of equal logits, rows that repeat, and rows with one token that has it all."""
    for B, K, V in [(4, 4, 1000), (3, 16, 3001), (8, 8, 40000), (32, 32, 9000)]:
        logits, scores = make(2, B, V, dtype, 7, scale)
        scores[:, 1:] = scores[:, :1]
        logits[:, 1::2] = logits[:, :1]
        check(logits, scores, K)


def test_more_ties_than_the_lists_hold():
    # blocks whose maxima all lie in one group of blocks: 33 blocks apart by 32, so that the candidates outgrow the lists
    logits = torch.full((1, 32, 256 * 64), -50.0, device=DEV)
    logits[:, :, 0:256] = 1.0
    logits[:, :, 32 * 256:33 * 256] = 1.0
    scores = torch.full((1, 32), -3.0, device=DEV)
    check(logits, scores, 32)
    scores = torch.arange(32, device=DEV).float()[None] * -1e-3
    check(logits, scores, 32)


@pytest.mark.parametrize("rise", [0.7, 3.9, 4.1, 7.3, 17.9, 39.37, 41.3, 95.1])
def test_late_peaks(rise):
    # a row's sum of exponentials is nearly all its last tokens, whose logits lie `rise` above those before them (so
    # many rows that a warp goes through several blocks of one)
    g = torch.Generator(device=DEV).manual_seed(5)
    logits = torch.randn(160, 4, 9000, generator=g, device=DEV) * 0.05 - rise
    logits[:, :, -3:] = torch.rand(160, 4, 3, generator=g, device=DEV) * 0.3
    check(logits, torch.rand(160, 4, generator=g, device=DEV) * 0.1, 4)
    check(logits.to(torch.bfloat16), torch.rand(160, 4, generator=g, device=DEV) * 0.1, 4)


@pytest.mark.parametrize("V", [151936, 150001])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_ties_all_over_a_wide_call(dtype, V):
    # equal rows of three levels: one token of the highest, a tenth of the middle one, all others of the lowest
    row = torch.zeros(V, device=DEV)
    row[torch.randperm(V, generator=torch.Generator().manual_seed(1))[:V // 10].to(DEV)] = 1.0
    row[V // 2] = 2.0
    mid = (row == 1.0).nonzero().flatten().cpu().numpy()
    for B, K in ((31, 32), (32, 32), (28, 30)):
        r = binding.beam_select(row.to(dtype).expand(2, B, V).contiguous(), torch.full((2, B), -3.0, device=DEV), K)
        want = [(b, V // 2) for b in range(B)] + [(0, int(v)) for v in mid]
        for n in range(2):
            assert list(zip(r["parents"][n].tolist(), r["tokens"][n].tolist())) == want[:K]
        flat = torch.zeros(2, B, V, device=DEV, dtype=dtype)
        r = binding.beam_select(flat, torch.zeros(2, B, device=DEV), K)
        assert r["parents"].eq(0).all() and r["tokens"].eq(torch.arange(K, device=DEV)).all()


def test_dead_ended_and_masked():
    logits, scores = make(8, 4, 3000, torch.float32, 5)
    finished = torch.zeros(8, 4, dtype=torch.bool, device=DEV)
    scores[0, 1:] = -math.inf                               # a first step
    scores[1] = -math.inf                                   # nothing is left
    finished[2] = True                                      # all have ended
    finished[3, 1] = True
    scores[3, 1] = 0.0
    finished[4, 0] = True
    scores[4, 0] = -math.inf
    logits[5, :, 5:] = -math.inf                            # few tokens allowed
    logits[6] = -math.inf                                   # none
    logits[6, 2, 77] = -3.0                                 # one
    logits[7, 0] = -math.inf
    for K in (1, 4, 16):
        check(logits, scores, K, finished, 2)
        check(logits.to(torch.bfloat16), scores, K, finished, 2999)
    keep = logits[0, 1:].clone()
    logits[0, 1:] = math.nan                                # a dead beam's logits do not count
    logits[2] = math.nan                                    # nor an ended one's
    check(logits, scores, 4, finished, 0)
    logits[0, 1:] = keep


@pytest.mark.parametrize("value", [math.nan, math.inf])
def test_rows_that_are_not_finite_are_flagged(value):
    logits, scores = make(3, 4, 30000, torch.bfloat16, 6)
    logits[0, 2, 12345] = value
    logits[1, 0, 29999] = value
    logits[1, 1, 0] = value
    scores[2, 3] = value
    r = check(logits, scores, 4)
    assert r["flags"].tolist() == [2, 2, 2] and not (r["parents"][0] == 2).any()
    row = torch.full((1, 1, 600), -math.inf, device=DEV)
    row[0, 0, 300] = value
    check(row, torch.zeros(1, 1, device=DEV), 3)


def test_lowest_value_masks():
    """Masks of the type's lowest value instead of -inf."""
    for dtype in (torch.float32, torch.bfloat16):
        logits, scores = make(2, 4, 5000, dtype, 8)
        logits[:, :, 100:] = torch.finfo(dtype).min
        check(logits, scores, 4)
        logits[1] = torch.finfo(dtype).min
        check(logits, scores, 4)


def test_strides():
    logits, scores = make(3, 4, 1111, torch.bfloat16, 9, pad=9)
    base = check(logits, scores, 4)
    swapped = logits.transpose(0, 1).contiguous().transpose(0, 1)
    a = binding.beam_select(swapped, scores, 4)
    shared = logits[:1].expand(3, 4, 1111)                  # one utterance's logits for all: stride 0
    b = binding.beam_select(shared, scores[:1].expand(3, 4).contiguous(), 4)
    for q in ("parents", "tokens"):
        assert torch.equal(a[q], base[q])
        assert torch.equal(b[q], base[q][:1].expand(3, 4))
    with pytest.raises(ValueError, match="contiguous rows"):
        binding.beam_select(logits.transpose(1, 2), scores, 4)
    with pytest.raises(ValueError, match="overlap"):
        binding.beam_select(logits[:, :1].expand(3, 4, 1111), scores, 4)
    with pytest.raises(ValueError, match="scores"):
        binding.beam_select(logits, scores.double(), 4)
    with pytest.raises(ValueError, match="finished"):
        binding.beam_select(logits, scores, 4, finished=scores > 0)
    with pytest.raises(ValueError, match="eos_id"):
        binding.beam_select(logits, scores, 4, eos_id=1111)
    with pytest.raises(binding.PctcError):
        binding.beam_select(logits, scores, 33)


def test_captured_into_a_graph_and_on_another_stream():
    logits, scores = make(4, 4, 20000, torch.bfloat16, 10)
    want = binding.beam_select(logits, scores, 4)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = binding.beam_select(logits, scores, 4)
    torch.cuda.current_stream().wait_stream(side)
    x = torch.zeros_like(logits)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = binding.beam_select(x, scores, 4)
    x.copy_(logits)
    graph.replay()
    for q in ("scores", "parents", "tokens", "flags"):
        assert torch.equal(r[q], want[q]) and torch.equal(other[q], want[q])


def test_scores_may_be_written_over():
    import ctypes
    logits, scores = make(3, 4, 20000, torch.bfloat16, 12)
    want = binding.beam_select(logits, scores, 4, finished=torch.zeros(3, 4, dtype=torch.bool, device=DEV), eos_id=0)
    done = torch.zeros(3, 4, dtype=torch.bool, device=DEV)
    p = binding.BeamProblem(3, 4, 4, 20000, logits.stride(0), logits.stride(1), 0, 0)
    o = [torch.empty(3, 4, dtype=torch.int32, device=DEV) for _ in range(2)]
    need = ctypes.c_size_t(0)
    assert binding.load().pctc_beam_workspace_bytes(ctypes.byref(p), ctypes.byref(need)) == 0
    ws = torch.empty(need.value, dtype=torch.uint8, device=DEV)
    st = binding.load().pctc_beam_select(ctypes.byref(p), logits.data_ptr(), scores.data_ptr(), done.data_ptr(),
                                         scores.data_ptr(), o[0].data_ptr(), o[1].data_ptr(), done.data_ptr(), None,
                                         ws.data_ptr(), need.value, torch.cuda.current_stream().cuda_stream)
    assert st == 0 and torch.equal(scores, want["scores"]) and torch.equal(o[0], want["parents"])
    assert torch.equal(o[1], want["tokens"]) and torch.equal(done, want["finished"])


@pytest.mark.parametrize("seed", range(40))
def test_random_calls(seed):
    """Sizes, types, alignment, dead, ended and masked beams in any mixture."""
    rng = np.random.default_rng(seed)
    N, B = int(rng.integers(1, 7)), int(rng.choice([1, 2, 3, 4, 7, 8, 16, 32]))
    V = int(np.exp(rng.uniform(np.log(2), np.log(60000))))
    K = int(rng.choice([1, B, 4, 32]))
    dtype = torch.bfloat16 if rng.random() < 0.5 else torch.float32
    logits, scores = make(N, B, V, dtype, seed, scale=float(rng.choice([0.5, 2.5, 8.0])), pad=int(rng.choice([0, 0, 1, 8, 64])))
    if rng.random() < 0.3:                                  # a base address that is not a multiple of 16 bytes
        buf = torch.zeros(N * B * V + 8, device=DEV, dtype=dtype)
        shifted = buf[1:1 + N * B * V].view(N, B, V)
        shifted.copy_(logits)
        logits = shifted
    g = torch.Generator(device=DEV).manual_seed(seed)
    if rng.random() < 0.4:
        scores[torch.rand(N, B, generator=g, device=DEV) < 0.3] = -math.inf
    finished = torch.rand(N, B, generator=g, device=DEV) < 0.25 if rng.random() < 0.5 else None
    if rng.random() < 0.3:
        logits.masked_fill_(torch.rand(V, generator=g, device=DEV) < rng.choice([0.1, 0.9, 0.999]), -math.inf)
    if rng.random() < 0.15:
        logits[N - 1, B - 1, V // 2] = math.nan
    check(logits, scores, K, finished, int(rng.integers(0, V)) if finished is not None or rng.random() < 0.5 else None)


def test_many_utterances():
    logits, scores = make(700, 2, 1500, torch.bfloat16, 3)
    check(logits, scores, 3)


def test_equal_rows_tie():
    """Rows with the same logits and score tie candidate by candidate, wherever their sums were computed."""
    for dtype, V, pad in [(torch.float32, 100_003, 0), (torch.bfloat16, 151_936, 0), (torch.bfloat16, 30_001, 7)]:
        logits, scores = make(2, 8, V, dtype, 11, pad=pad)
        logits[:, 1:] = logits[:, :1]
        scores[:, 1:] = scores[:, :1]
        r = binding.beam_select(logits, scores, 8)
        for n in range(2):
            x = logits[n, 0].float().cpu().numpy()
            best = np.argsort(-x, kind="stable")[:8]        # a row may hold its largest logit more than once
            want = sorted(((-x[v], b, int(v)) for b in range(8) for v in best))[:8]
            assert list(zip(r["parents"][n].tolist(), r["tokens"][n].tolist())) == [(b, v) for _, b, v in want]


def test_outputs_in_the_padding_of_the_logits():
    """What is written may lie between the rows (nothing there is read), but not on them."""
    import ctypes
    logits, scores = make(2, 4, 1000, torch.float32, 3, pad=24)
    want = binding.beam_select(logits.clone(), scores, 4)
    p = binding.BeamProblem(2, 4, 4, 1000, logits.stride(0), logits.stride(1), 1, -1)
    ws = torch.empty(1 << 16, dtype=torch.uint8, device=DEV)
    stream = torch.cuda.current_stream().cuda_stream

    def call(first):
        out = [logits.data_ptr() + 4 * (b * logits.stride(1) + first) for b in range(3)]
        return binding.load().pctc_beam_select(ctypes.byref(p), logits.data_ptr(), scores.data_ptr(), None, *out, None, None,
                                               ws.data_ptr(), ws.numel(), stream)

    assert call(999) == 1 and call(1017) == 1               # the last token of a row, and the first one of the next
    assert call(1000) == 0
    rows = logits.as_strided((3, 8), (logits.stride(1), 1), logits.storage_offset() + 1000)
    for x, row in zip(("scores", "parents", "tokens"), rows):
        assert torch.equal(row.contiguous().view(want[x].dtype), want[x].flatten())


@pytest.mark.parametrize("rise", [0.5, 1.5, 2.5, 3.5, 3.9])
@pytest.mark.parametrize("low", [-20.0, -14.0])
def test_a_peak_a_little_above_the_blocks_before_it(rise, low):
    """Rows of one token at 0, a few blocks behind two at about -rise and all else at `low`.

    The largest logit counts exactly 1; an exponential d below it is off by (2^-22 + 1.4e-7 |d|) of its share of
    the row, a lane's sum of 16 takes five roundings, and the score one more."""
    V, R = 32768, 512
    g = torch.Generator(device=DEV).manual_seed(1)
    x = torch.full((R, 8, V), low, device=DEV)
    x[:, :, 0] = -rise * (1 - 1e-3 * torch.rand(R, 8, generator=g, device=DEV))
    x[:, :, 4000] = x[:, :, 0]
    x[:, :, 600] = 0
    scores = -torch.rand(R, 8, generator=g, device=DEV)
    r = binding.beam_select(x.view(R * 8, 1, V), scores.view(-1, 1), 1)
    got = r["scores"].view(R, 8).double()
    want = scores.double() - torch.logsumexp(x.double(), -1)
    rest = 1 - torch.exp(-torch.logsumexp(x.double(), -1))
    tol = 5 * 2.0 ** -24 + rest * (2.0 ** -22 + 1.4e-7 * -low) + 2.0 ** -24 * want.abs()
    assert r["tokens"].eq(600).all() and bool(((got - want).abs() <= tol).all())
    assert bool((r["scores"].view(R, 8) <= scores).all())


def test_no_candidate_scores_above_its_parent():
    for dtype in (torch.float32, torch.bfloat16):
        for gap in (15.0, 17.0, 20.0, 90.0):                # what is not the best adds up to about nothing
            logits, _ = make(40, 4, 20011, dtype, 3, 0.5)
            logits[:, :, 7777] = logits.float().amax(-1).to(dtype) + gap
            scores = torch.tensor([0.0, -1e-7, -1e-3, -2.0], device=DEV).expand(40, 4).contiguous()
            r = binding.beam_select(logits, scores, 4)
            assert bool((r["scores"] <= scores.gather(1, r["parents"].long())).all()) and r["tokens"].eq(7777).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,blocks,pad", [(8, 128, 5), (8, 128, 3), (32, 512, 3)])
def test_ties_beyond_the_lists_among_other_beams(B, blocks, pad, dtype):
    """More candidates than the lists hold, beside ended, dead, masked and not finite beams.

    Blocks are 512 logits and the threshold is the K-th best of the maxima of 32 groups of blocks (by block number
    modulo 32), so the six groups that reach 0.5 only put it there; all other blocks hold 40 logits of 1.0 and give K
    candidates each: 104 blocks in a row of 128, so more than 2,048 candidates in one row.  (More than 2 K blocks a row:
    the threshold is not raised.)"""
    V = 512 * blocks - 3
    g = torch.Generator(device=DEV).manual_seed(B)
    full = torch.full((1, B, V + pad), -50.0, device=DEV)
    full[:, :, V:] = 1e4
    x = full[:, :, :V]
    at = torch.stack([torch.randperm(508, generator=torch.Generator().manual_seed(i))[:40] + 512 * i for i in range(blocks)])
    low = torch.arange(blocks) % 32 >= 26
    x[:, :, at[~low].flatten().to(DEV)] = 1.0
    x[:, :, at[low, 0].to(DEV)] = 0.5
    x[0, :, [512 * 5 + 100, 512 * 33, 7]] = 1.25            # three winners a row, in blocks that reach 1.0 anyway
    x = full.to(dtype)[:, :, :V]
    scores = torch.full((1, B), -3.0, device=DEV)           # beams 0 and 2 tie candidate by candidate
    scores[0, 1], scores[0, 3] = -3.01, -3.2
    finished = torch.zeros(1, B, dtype=torch.bool, device=DEV)
    finished[0, 4] = True
    scores[0, 4] = -3.0 - float(torch.logsumexp(x[0, 0].double(), 0)) + 1.1      # between the winners and the ties
    scores[0, 5] = -math.inf
    x[0, 6, 1000] = math.nan
    x[0, 7] = -math.inf
    for b in range(8, B):
        scores[0, b] = -4.0 - b / 64
    for K in (32, 27):
        r = check(x, scores, K, finished, 9)
        assert r["flags"].item() == 2
        # 1.25 from beams 0 and 2, 1.24, the ended one at 1.1, 1.25 - 0.2, then the ties at 1.0 of beam 0
        assert r["parents"][0].tolist() == [0] * 3 + [2] * 3 + [1] * 3 + [4] + [3] * 3 + [0] * (K - 13)
