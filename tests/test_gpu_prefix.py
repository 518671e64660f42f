"""CTC prefix beam search on the GPU against the oracle on the same inputs.

Labels, lengths and flags have to be equal: both sides do the same IEEE operations on the same 24-bit
probabilities.  A score is a 64-bit logarithm rounded once to fp32 (2^-24 relative); 2^-22 leaves room for the
order of the sum of the frames' shifts."""

import math

import numpy as np
import pytest
import torch

from oracle import pruned_ctc_oracle as O
from paper_2609_33645_b200 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def make(N, T, k, V, seed, sharp=1.5, hold=6, blank=0.8):
    rng = np.random.default_rng(seed)
    classes = np.zeros((N, T, k), dtype=np.int32)
    for n in range(N):
        for t0 in range(0, T, hold):
            c = rng.choice(V - 1, size=k, replace=False) + 1
            if rng.random() < blank:
                c[0] = 0
            classes[n, t0:t0 + hold] = c
    z = rng.normal(size=(N, T, k)) * sharp
    z = (z - np.log(np.exp(z).sum(-1, keepdims=True) * 1.01)).astype(np.float32)
    order = np.argsort(-z, axis=-1, kind="stable")
    return np.take_along_axis(classes, order, -1), np.take_along_axis(z, order, -1)


def check(res, classes, logprobs, lengths, blank, beams):
    tokens, sizes, scores, flags = (res[x].cpu().numpy() for x in ("tokens", "token_lengths", "scores", "flags"))
    for n in range(classes.shape[0]):
        want, bad = O.prefix_beam_search(classes[n], logprobs[n], lengths[n], blank, beams)
        assert flags[n] == (2 if bad else 0) | (0 if want else 1)
        for b in range(beams):
            if b >= len(want):
                assert sizes[n, b] == 0 and scores[n, b] == -math.inf and (tokens[n, b] == -1).all()
                continue
            labels, score = want[b]
            assert sizes[n, b] == len(labels), (n, b)
            assert tokens[n, b, : len(labels)].tolist() == labels and (tokens[n, b, len(labels):] == -1).all()
            assert abs(float(scores[n, b]) - score) <= 2.0 ** -22 * abs(score) + 1e-6


def run(classes, logprobs, lengths, blank, beams):
    return binding.prefix_beam_decode(torch.from_numpy(classes).to(DEV), torch.from_numpy(logprobs).to(DEV), lengths, blank, beams)


@pytest.mark.parametrize("N,T,k,V,beams", [
    (1, 1, 1, 5, 1), (1, 1, 8, 50, 4), (2, 40, 1, 9, 4), (3, 40, 2, 4, 3), (2, 33, 8, 9, 1), (4, 65, 8, 12, 4),
    (2, 100, 8, 40, 16), (2, 50, 32, 40, 32), (1, 64, 5, 1000, 32), (2, 31, 7, 151936, 10), (1, 200, 4, 6, 8),
    (2, 48, 32, 33, 2), (1, 60, 3, 4, 31), (2, 40, 12, 30, 16), (1, 40, 9, 20, 9), (2, 64, 8, 9, 8), (1, 33, 8, 30, 17),
])
@pytest.mark.parametrize("sharp", [0.3, 3.0, 12.0])
def test_against_the_oracle(N, T, k, V, beams, sharp):
    classes, logprobs = make(N, T, k, V, N * 1000 + T + k, sharp)
    lengths = [T] + [max(1, T - 7 * i - 1) for i in range(1, N)]
    check(run(classes, logprobs, lengths, 0, beams), classes, logprobs, lengths, 0, beams)


def test_a_long_utterance_is_rescaled():
    classes, logprobs = make(2, 3000, 8, 5000, 3, 1.0)
    check(run(classes, logprobs, [3000, 1777], 0, 16), classes, logprobs, [3000, 1777], 0, 16)
    low = (logprobs - 300.0).astype(np.float32)
    check(run(classes[:1, :500], low[:1, :500], [500], 0, 4), classes[:1, :500], low[:1, :500], [500], 0, 4)


@pytest.mark.parametrize("blank", [0, 3])
def test_ties(blank):
    """Equal probabilities everywhere, and frames that repeat: order alone decides."""
    classes = np.tile(np.arange(5, dtype=np.int32), (2, 20, 1))
    classes[1, 10:] = classes[1, 10:, ::-1]
    logprobs = np.full((2, 20, 5), np.float32(math.log(0.2)))
    for beams in (3, 8, 32):
        check(run(classes, logprobs, [20, 20], blank, beams), classes, logprobs, [20, 20], blank, beams)
    classes, logprobs = make(1, 1, 6, 7, 1)
    classes, logprobs = np.repeat(classes, 30, 1), np.repeat(logprobs, 30, 1)
    for beams in (2, 16):
        check(run(classes, logprobs, [30], blank, beams), classes, logprobs, [30], blank, beams)


def test_masked_entries():
    classes, logprobs = make(6, 30, 6, 12, 8)
    classes[0, ::3, 2:] = -1
    logprobs[1, ::2, 3] = -np.inf
    logprobs[2, 7, 0] = np.nan
    logprobs[2, 9, 1] = np.inf
    classes[3, :, 4] = classes[3, :, 1]                    # a class given twice
    classes[3, 5, 5] = classes[3, 5, 0]
    logprobs[4, ::4, 2:] = -800.0                          # beyond exp(-700) of the best
    logprobs[4, 1::4, 1] = -650.0
    logprobs[5] += 90.0                                    # not normalised
    classes[1, 4] = -1                                     # nothing is possible from here on
    for beams in (1, 4, 16):
        res = run(classes, logprobs, [30] * 6, 0, beams)
        check(res, classes, logprobs, [30] * 6, 0, beams)
        assert res["flags"].tolist() == [0, 1, 2, 0, 0, 0]


def test_only_blank_and_only_one_class():
    classes = np.zeros((2, 12, 1), dtype=np.int32)
    classes[1] = 4
    logprobs = np.full((2, 12, 1), -0.25, dtype=np.float32)
    res = run(classes, logprobs, [12, 12], 0, 4)
    check(res, classes, logprobs, [12, 12], 0, 4)
    assert res["token_lengths"].tolist() == [[0, 0, 0, 0], [1, 0, 0, 0]]


def test_padded_frames_are_not_read():
    classes, logprobs = make(3, 40, 4, 9, 2)
    a = run(classes, logprobs, [40, 11, 1], 0, 4)
    logprobs[1, 11:], logprobs[2, 1:], classes[1, 11:], classes[2, 1:] = np.nan, np.nan, 2 ** 31 - 1, 1
    b = run(classes, logprobs, [40, 11, 1], 0, 4)
    for x in ("tokens", "token_lengths", "scores", "flags"):
        assert torch.equal(a[x], b[x])


@pytest.mark.parametrize("cuts", [[1] * 70, [69, 1], [32, 32, 6], [5, 0, 17, 48]])
def test_portions_make_the_whole(cuts):
    classes, logprobs = make(3, 70, 8, 30, 4)
    lengths = [70, 41, 3]
    whole = run(classes, logprobs, lengths, 0, 8)
    s = binding.PrefixBeam(3, 8, 80, 0, DEV)
    at = 0
    for c in cuts:
        if c == 0:
            s.advance(torch.zeros(3, 1, 8, dtype=torch.int32, device=DEV), torch.zeros(3, 1, 8, device=DEV), [0, 0, 0])
            continue
        s.advance(torch.from_numpy(classes[:, at:at + c].copy()).to(DEV), torch.from_numpy(logprobs[:, at:at + c].copy()).to(DEV),
                  [min(c, max(0, l - at)) for l in lengths])
        at += c
    got = s.read()
    for x in ("token_lengths", "scores", "flags"):
        assert torch.equal(got[x], whole[x])
    assert torch.equal(got["tokens"], whole["tokens"])
    again = s.read(max_tokens=5)                            # reading changes nothing; labels beyond the row are left out
    assert torch.equal(again["tokens"], got["tokens"][:, :, :5]) and torch.equal(again["token_lengths"], got["token_lengths"])


def test_a_finished_search_goes_on():
    """The search that prefix_beam_decode returns reads the same hypotheses, and its state is full."""
    classes, logprobs = make(2, 40, 8, 30, 4)
    r = run(classes, logprobs, [40, 17], 0, 8)
    again = r["search"].read()
    for x in ("tokens", "token_lengths", "scores", "flags"):
        assert torch.equal(again[x], r[x])
    c, l = torch.from_numpy(classes[:, :23].copy()).to(DEV), torch.from_numpy(logprobs[:, :23].copy()).to(DEV)
    with pytest.raises(ValueError, match="room"):
        r["search"].advance(c, l)
    r["search"].advance(c, l, [0, 23])
    two = [np.concatenate([x[1:, :17], x[1:, :23]], 1) for x in (classes, logprobs)]
    got = r["search"].read()
    check({x: got[x][1:] for x in ("tokens", "token_lengths", "scores", "flags")}, *two, [40], 0, 8)


def test_more_utterances_than_one_launch_takes():
    classes, logprobs = make(1030, 3, 2, 4, 6)
    lengths = [1 + i % 3 for i in range(1030)]
    check(run(classes, logprobs, lengths, 0, 2), classes, logprobs, lengths, 0, 2)


def test_a_state_that_does_not_fit_takes_nothing():
    import ctypes
    lib = binding.load()
    classes, logprobs = make(2, 6, 4, 9, 1)
    c, l = torch.from_numpy(classes).to(DEV), torch.from_numpy(logprobs).to(DEV)
    s = binding.PrefixBeam(2, 4, 8, 0, DEV)
    s.advance(c, l)
    before = s.read(max_tokens=8)
    ln = (ctypes.c_int32 * 2)(6, 2)                         # 12 of 8 frames, and 8 of 8
    p = binding.PrefixProblem(2, 6, 4, 4, 0, 8)
    stream = torch.cuda.current_stream().cuda_stream
    assert lib.pctc_prefix_advance(ctypes.byref(p), c.data_ptr(), l.data_ptr(), ln, 0, s.state.data_ptr(), s.state.numel(), stream) == 0
    after = s.read(max_tokens=8)
    assert after["flags"].tolist() == [binding.UTT_STATE_FULL, 0]
    assert torch.equal(after["tokens"][0], before["tokens"][0]) and torch.equal(after["scores"][0], before["scores"][0])
    two = [np.concatenate([x[1:], x[1:, :2]], 1) for x in (classes, logprobs)]
    check({x: after[x][1:] for x in ("tokens", "token_lengths", "scores", "flags")}, *two, [8], 0, 4)
    # never started: nothing is read, nothing taken
    s = binding.PrefixBeam(2, 4, 8, 0, DEV)
    s.state.zero_()
    assert lib.pctc_prefix_advance(ctypes.byref(p), c.data_ptr(), l.data_ptr(), ln, 0, s.state.data_ptr(), s.state.numel(), stream) == 0
    s.started = True
    r = s.read(max_tokens=4)
    assert r["flags"].tolist() == [binding.UTT_STATE_FULL] * 2 and (r["tokens"] == -1).all() and (r["scores"] == -math.inf).all()


def test_captured_into_a_graph_and_on_another_stream():
    classes, logprobs = make(2, 50, 8, 20, 9)
    c, l = torch.from_numpy(classes).to(DEV), torch.from_numpy(logprobs).to(DEV)
    want = binding.prefix_beam_decode(c, l, [50, 20], 0, 4)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = binding.prefix_beam_decode(c, l, [50, 20], 0, 4)
    torch.cuda.current_stream().wait_stream(side)
    cc, ll = torch.zeros_like(c), torch.zeros_like(l)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        res = binding.prefix_beam_decode(cc, ll, [50, 20], 0, 4)
    cc.copy_(c)
    ll.copy_(l)
    graph.replay()
    graph.replay()
    for x in ("tokens", "token_lengths", "scores", "flags"):
        assert torch.equal(res[x], want[x]) and torch.equal(other[x], want[x])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_with_the_head(dtype):
    """Recognition as it is used: hidden states, the k best classes of every frame, the search."""
    g = torch.Generator(device=DEV).manual_seed(3)
    hidden = torch.randn(3, 25, 64, device=DEV, generator=g).to(dtype)
    W = (torch.randn(1000, 64, device=DEV, generator=g) / 4).to(dtype)
    lengths = [25, 9, 1]
    best = binding.topk_decode(hidden, W, None, lengths, 8)
    res = binding.beam_decode(hidden, W, None, lengths, 0, 4, k=8)
    check(res, best["classes"].cpu().numpy(), best["logprobs"].cpu().numpy(), lengths, 0, 4)
    one = binding.beam_decode(hidden, W, None, lengths, 0, 1, k=1)
    greedy = binding.greedy_decode(hidden, W, None, lengths, 0)
    assert torch.equal(one["tokens"][:, 0], greedy["tokens"]) and torch.equal(one["token_lengths"][:, 0], greedy["token_lengths"])


@pytest.mark.parametrize("seed", range(30))
def test_random_calls(seed):
    """Sizes, confusable classes, absent and repeated entries and equal probabilities in any mixture."""
    rng = np.random.default_rng(1000 + seed)
    N, T = int(rng.integers(1, 4)), int(rng.integers(1, 90))
    k, beams = int(rng.choice([1, 2, 3, 5, 8, 8, 13, 32])), int(rng.choice([1, 2, 4, 5, 8, 9, 16, 20, 32]))
    V = k + int(rng.choice([1, 2, 5, 200]))
    classes, logprobs = make(N, T, k, V, seed, float(rng.choice([0.2, 1.0, 4.0, 15.0])), int(rng.choice([1, 3, 9])))
    if rng.random() < 0.4:
        logprobs = np.round(logprobs * 2) / np.float32(2)   # many equal ones
    if rng.random() < 0.4:
        classes[rng.random(classes.shape) < 0.2] = -1
    if rng.random() < 0.3:
        classes[rng.random(classes.shape) < 0.2] = 1        # given twice
    if rng.random() < 0.2:
        logprobs[rng.random(logprobs.shape) < 0.02] = np.nan
    lengths = [int(rng.integers(1, T + 1)) for _ in range(N)]
    blank = int(rng.integers(0, 3))
    check(run(classes, logprobs, lengths, blank, beams), classes, logprobs, lengths, blank, beams)


def test_refusals_on_the_device():
    c, l = torch.zeros(2, 5, 4, dtype=torch.int32, device=DEV), torch.zeros(2, 5, 4, device=DEV)
    for kw, error in [(dict(lengths=[5, 6]), ValueError), (dict(lengths=[5, -1]), binding.PctcError),
                      (dict(lengths=[5]), ValueError), (dict(beams=0), binding.PctcError), (dict(beams=33), binding.PctcError),
                      (dict(blank=-1), binding.PctcError)]:
        a = dict(lengths=[5, 5], beams=4, blank=0)
        a.update(kw)
        with pytest.raises(error):
            binding.prefix_beam_decode(c, l, a["lengths"], a["blank"], a["beams"])
    with pytest.raises(binding.PctcError):
        binding.prefix_beam_decode(torch.zeros(1, 5, 33, dtype=torch.int32, device=DEV), torch.zeros(1, 5, 33, device=DEV), [5], 0, 4)
    s = binding.PrefixBeam(2, 4, 9, 0, DEV)
    with pytest.raises(ValueError, match="device"):
        s.advance(c.cpu(), l.cpu())
    s.advance(c, l)
    with pytest.raises(ValueError, match="room"):
        s.advance(c, l)
    with pytest.raises(ValueError, match="max_tokens"):
        s.read(max_tokens=0)


# Label sequences whose 64-bit hashes are equal (found by solving for them; labels of a vocabulary of 2^18 and 2^21, and,
# of different lengths, of any 32-bit labels).
TWINS = [((141360, 45075), (158416, 213418)), ((1580687, 180223), (1368230, 1849779)), ((837479, 2220), (1184745, 1717519)),
         ((336947217,), (59540, 1632145480)), ((59540, 1632145480), (336947217,)), ((474014802,), (126093, 18546947))]


@pytest.mark.parametrize("beams", [16, 32])
@pytest.mark.parametrize("first,second", TWINS)
def test_prefixes_with_equal_hashes_are_kept_apart(first, second, beams):
    """The first prefix is grown by c and leaves the beam, the second comes up later, and then c is its best extension:
    it may not be taken for the parent of the first one's child."""
    c, quiet = 7, -1
    a, p = first[0], second[0]
    frames = [[(a, 0.5), (p, 0.5)] if len(second) > 1 else [(a, 0.5), (99, 0.5)]]
    keep = p if len(second) > 1 else 99                     # what the second prefix will be grown from, or next to
    if len(first) > 1:
        frames.append([(first[1], 0.9), (keep, 0.5)])
    frames.append([(c, 0.9), (keep, 0.5)])
    if len(second) > 1:
        frames.append([(second[1], 0.9), (c, 0.5)])
    else:                                                   # a single label grows only from the empty prefix: keep that by blanks
        frames = [[(0, 0.5)] + f for f in frames] + [[(second[0], 0.9), (c, 0.5)]]
    frames += [[(c, 1.0)], [(c, 0.6), (0, 0.4)], [(c, 0.5), (a, 0.5)]]
    k = max(len(f) for f in frames)
    classes = np.array([[[x for x, _ in f] + [quiet] * (k - len(f)) for f in frames]], dtype=np.int32)
    logprobs = np.log(np.array([[[x for _, x in f] + [1.0] * (k - len(f)) for f in frames]])).astype(np.float32)
    T = len(frames)
    check(run(classes, logprobs, [T], 0, beams), classes, logprobs, [T], 0, beams)
    s = binding.PrefixBeam(1, beams, T, 0, DEV)             # the same, a frame at a time
    for t in range(T):
        s.advance(torch.from_numpy(classes[:, t:t + 1].copy()).to(DEV), torch.from_numpy(logprobs[:, t:t + 1].copy()).to(DEV))
        got = s.read()
        check(got, classes, logprobs, [t + 1], 0, beams)


def test_portions_without_frames():
    """A recogniser's empty portions, at the start, in between and as the whole utterance."""
    classes, logprobs = make(2, 20, 8, 30, 4)
    c, l = torch.from_numpy(classes).to(DEV), torch.from_numpy(logprobs).to(DEV)
    none = c[:, :0].contiguous(), l[:, :0].contiguous()
    s = binding.PrefixBeam(2, 8, 20, 0, DEV)
    s.advance(*none)
    r = s.read()
    assert r["token_lengths"].eq(0).all() and r["scores"][:, 0].eq(0).all() and r["scores"][:, 1:].eq(-math.inf).all()
    s.advance(c[:, :7].contiguous(), l[:, :7].contiguous())
    s.advance(*none, [0, 0])
    s.advance(c[:, 7:].contiguous(), l[:, 7:].contiguous())
    s.advance(*none)
    check(s.read(), classes, logprobs, [20, 20], 0, 8)
    whole = binding.prefix_beam_decode(*none, [0, 0], 0, 4)
    again = whole["search"].read()
    for r in (whole, again):
        assert r["token_lengths"].eq(0).all() and r["tokens"].eq(-1).all() and r["flags"].eq(0).all()
        assert r["scores"].tolist() == [[0.0] + [-math.inf] * 3] * 2
    with pytest.raises(ValueError):
        binding.prefix_beam_decode(*none, [1, 0], 0, 4)
    with pytest.raises(binding.PctcError):
        s.advance(*none, [-1, 0])
    with pytest.raises((binding.PctcError, ValueError)):
        binding.PrefixBeam(2, 8, 20, 0, DEV).advance(*none, [1, 0])


@pytest.mark.parametrize("N,beams,max_frames", [(1, 4, 12), (2, 4, 12), (4, 4, 12), (9, 4, 12), (3, 5, 12), (3, 4, 11)])
def test_a_state_of_other_sizes_is_left_as_it_is(N, beams, max_frames):
    import ctypes
    lib = binding.load()
    classes, logprobs = make(9, 6, 4, 9, 1)
    c, l = torch.from_numpy(classes).to(DEV), torch.from_numpy(logprobs).to(DEV)
    s = binding.PrefixBeam(3, 4, 12, 0, DEV)
    s.state = torch.zeros(1 << 16, dtype=torch.uint8, device=DEV)          # room for every size that is tried
    s.advance(c[:3].contiguous(), l[:3].contiguous())
    before, state = s.read(max_tokens=12), s.state.clone()
    p = binding.PrefixProblem(N, 3, 4, beams, 0, max_frames)
    need = ctypes.c_size_t(0)
    assert lib.pctc_prefix_state_bytes(ctypes.byref(p), ctypes.byref(need)) == 0 and need.value <= s.state.numel()
    ln, stream = (ctypes.c_int32 * N)(*[3] * N), torch.cuda.current_stream().cuda_stream
    assert lib.pctc_prefix_advance(ctypes.byref(p), c.data_ptr(), l.data_ptr(), ln, 0, s.state.data_ptr(), s.state.numel(), stream) == 0
    out = [torch.empty(n, dtype=torch.int32, device=DEV) for n in (N * beams * 12, N * beams, N * beams, N)]
    assert lib.pctc_prefix_read(ctypes.byref(p), s.state.data_ptr(), s.state.numel(), out[0].data_ptr(), 12, out[1].data_ptr(),
                                out[2].data_ptr(), out[3].data_ptr(), stream) == 0
    assert out[3].eq(binding.UTT_STATE_FULL).all() and out[1].eq(0).all() and out[0].eq(-1).all()
    after = s.read(max_tokens=12)
    for x in ("tokens", "token_lengths", "scores"):
        assert torch.equal(after[x], before[x])
    assert after["flags"].tolist() == [binding.UTT_STATE_FULL if n < N else 0 for n in range(3)]
    assert int((s.state != state).sum()) == min(N, 3)       # a flag each
    c2, l2 = (x[:3, :6].contiguous() for x in (c, l))
    s.advance(c2, l2)                                       # and goes on as if nothing had been
    two = [np.concatenate([x[:3], x[:3]], 1) for x in (classes, logprobs)]
    got = s.read(max_tokens=12)
    got["flags"] = got["flags"] & ~binding.UTT_STATE_FULL
    check(got, *two, [12] * 3, 0, 4)
