"""CTC prefix beam search, without a GPU: the oracle against sums over all alignments, and the refusals."""

import ctypes
import itertools

import numpy as np
import pytest
import torch

from oracle import pruned_ctc_oracle as O
from paper_2609_33645_b200 import binding


def all_sequences(classes, logprobs, T, blank):
    """Probability of every label sequence: the sum over all alignments, one by one."""
    total = {}
    k = classes.shape[1]
    for path in itertools.product(range(k), repeat=T):
        lp = sum(float(logprobs[t, j]) for t, j in enumerate(path))
        seq = tuple(O.collapse([classes[t, j] for t, j in enumerate(path)], blank))
        total[seq] = total.get(seq, 0.0) + np.exp(lp)
    return sorted(total.items(), key=lambda e: -e[1])


@pytest.mark.parametrize("seed", range(8))
def test_oracle_with_room_for_all_prefixes_sums_all_alignments(seed):
    rng = np.random.default_rng(seed)
    T, k, V = 6, 3, 4
    classes = np.stack([rng.permutation(V)[:k] for _ in range(T)])
    logprobs = np.log(rng.dirichlet(np.ones(k), size=T))
    want = all_sequences(classes, logprobs, T, 0)
    got, bad = O.prefix_beam_search(classes, logprobs, T, 0, 10 ** 6)
    assert not bad and len(got) == len(want)
    assert [tuple(l) for l, _ in got][:10] == [s for s, _ in want][:10]
    for (_, g), (_, w) in zip(got, want):
        # T probabilities rounded to 24 bits
        assert g == pytest.approx(np.log(w), abs=2 * T * 2.0 ** -24)


def test_oracle_keeps_a_prefix_that_was_dropped_and_came_back():
    """A grown prefix finds the slot that holds it also when its parent left the beam in between."""
    rng = np.random.default_rng(5)
    for _ in range(50):
        classes = np.tile(np.arange(4), (12, 1))
        logprobs = np.log(rng.dirichlet(np.ones(4) * 0.3, size=12))
        got, _ = O.prefix_beam_search(classes, logprobs, 12, 0, 3)
        assert len({tuple(l) for l, _ in got}) == len(got)


def test_oracle_probabilities():
    pairs, shift, bad = O.frame_probabilities([3, 3, -1, 5, 7, 9], [-1.0, -0.5, 0.0, -np.inf, -900.0, -2.0])
    assert shift == -1.0 and not bad                     # the second 3 and the -1 do not count
    assert [c for c, _ in pairs] == [3, -2, -2, -2, -2, 9]
    assert pairs[0][1] == 1.0 and pairs[5][1] == pytest.approx(np.exp(-1.0), rel=2.0 ** -24)
    assert O.frame_probabilities([1, 2], [np.nan, np.inf])[2]


def _problem(**kw):
    d = dict(N=2, T=5, k=4, beams=4, blank_id=0, max_frames=9)
    d.update(kw)
    return binding.PrefixProblem(*[d[f] for f, _ in binding.PrefixProblem._fields_])


@pytest.mark.parametrize("kw,want", [
    (dict(N=0), 1), (dict(T=0), 1), (dict(k=0), 1), (dict(k=33), 3), (dict(beams=0), 1), (dict(beams=33), 3),
    (dict(blank_id=-1), 1), (dict(max_frames=0), 1), (dict(max_frames=2 ** 30), 3),
])
def test_bad_problems_are_refused(lib, kw, want):
    out = ctypes.c_size_t(0)
    assert lib.load().pctc_prefix_state_bytes(ctypes.byref(_problem(**kw)), ctypes.byref(out)) == want


def test_bad_calls_are_refused_before_any_launch(lib):
    cdll = lib.load()
    out = ctypes.c_size_t(0)
    p = _problem()
    assert cdll.pctc_prefix_state_bytes(ctypes.byref(p), ctypes.byref(out)) == 0
    assert cdll.pctc_prefix_state_bytes(ctypes.byref(p), None) == 1
    need, at = out.value, 1 << 20

    def advance(lengths=(5, 0), cls=at, lp=at, fresh=1, state=at, size=need):
        ln = (ctypes.c_int32 * 2)(*lengths)
        return cdll.pctc_prefix_advance(ctypes.byref(p), cls, lp, ln, fresh, state, size, None)

    assert advance(lengths=(6, 0)) == 1 and advance(lengths=(-1, 0)) == 1
    assert advance(cls=None) == 1 and advance(lp=None) == 1 and advance(state=None) == 1
    assert advance(state=at + 8) == 1 and advance(cls=at + 2) == 1 and advance(fresh=2) == 1
    assert advance(size=need - 1) == 2
    read = lambda tokens=at, stride=9, ln=at, sc=at, size=need: cdll.pctc_prefix_read(
        ctypes.byref(p), at, size, tokens, stride, ln, sc, None, None)
    assert read(tokens=None) == 1 and read(stride=0) == 1 and read(ln=None) == 1 and read(sc=None) == 1
    assert read(size=need - 1) == 2

    def decode(lengths=(5, 0), cls=at, state=at, size=need, tokens=at, stride=9, sizes=at, scores=at):
        ln = (ctypes.c_int32 * 2)(*lengths)
        return cdll.pctc_prefix_decode(ctypes.byref(p), cls, at, ln, state, size, tokens, stride, sizes, scores, None, None)

    assert decode(lengths=(6, 0)) == 1 and decode(cls=None) == 1 and decode(state=None) == 1 and decode(size=need - 1) == 2
    assert decode(tokens=None) == 1 and decode(stride=0) == 1 and decode(sizes=None) == 1 and decode(scores=None) == 1


def test_more_hypotheses_than_32_bits_count_are_refused(lib):
    out = ctypes.c_size_t(0)
    for N, beams, want in ((2 ** 26, 32, 3), (2 ** 26 - 1, 32, 0), (2 ** 31 - 1, 2, 3), (2 ** 31 - 1, 1, 0)):
        p = _problem(N=N, beams=beams)
        assert lib.load().pctc_prefix_state_bytes(ctypes.byref(p), ctypes.byref(out)) == want
        if want:
            args = [ctypes.byref(p), 1 << 20, 2 ** 62, (1 << 20) * 2, 9, (1 << 20) * 3, (1 << 20) * 4, None, None]
            assert lib.load().pctc_prefix_read(*args) == want


@pytest.mark.parametrize("which", ["tokens", "sizes", "scores", "flags"])
def test_misaligned_outputs_are_refused(lib, which):
    cdll, p, at = lib.load(), _problem(), 1 << 20
    out = ctypes.c_size_t(0)
    assert cdll.pctc_prefix_state_bytes(ctypes.byref(p), ctypes.byref(out)) == 0
    ln = (ctypes.c_int32 * 2)(5, 0)
    for off in (1, 2, 3):
        o = dict(tokens=at * 4, sizes=at * 5, scores=at * 6, flags=at * 7)
        o[which] += off
        assert cdll.pctc_prefix_read(ctypes.byref(p), at, out.value, o["tokens"], 9, o["sizes"], o["scores"], o["flags"], None) == 1
        assert cdll.pctc_prefix_decode(ctypes.byref(p), at * 2, at * 3, ln, at, out.value, o["tokens"], 9, o["sizes"], o["scores"],
                                       o["flags"], None) == 1


@pytest.mark.parametrize("a,b,off", [
    ("state", "classes", 159), ("state", "logprobs", 0), ("classes", "state", 0), ("tokens", "state", 0), ("flags", "state", 4),
    ("sizes", "tokens", 284), ("scores", "tokens", 0), ("flags", "scores", 28), ("scores", "sizes", 28), ("tokens", "classes", 156),
    ("flags", "logprobs", 156),
])
def test_what_a_search_writes_lies_apart(lib, a, b, off):
    """2 utterances of 5 frames of 4 classes (160 bytes), 4 beams of 9 labels (288 bytes)."""
    cdll, p = lib.load(), _problem()
    out = ctypes.c_size_t(0)
    assert cdll.pctc_prefix_state_bytes(ctypes.byref(p), ctypes.byref(out)) == 0
    at = {x: (1 << 20) * (i + 1) for i, x in enumerate(("classes", "logprobs", "state", "tokens", "sizes", "scores", "flags"))}
    at[a] = at[b] + off
    if a == "state":
        at[a] = at[b] - at[b] % 256
        at[b] = at[a] + out.value - 4                       # on the state's last bytes
    ln = (ctypes.c_int32 * 2)(5, 0)
    args = [at[x] for x in ("classes", "logprobs")]
    outs = [at["tokens"], 9, at["sizes"], at["scores"], at["flags"]]
    if a not in ("tokens", "sizes", "scores", "flags"):
        assert cdll.pctc_prefix_advance(ctypes.byref(p), *args, ln, 1, at["state"], out.value, None) == 1
    elif b not in ("classes", "logprobs"):
        assert cdll.pctc_prefix_read(ctypes.byref(p), at["state"], out.value, *outs, None) == 1
    for k in (4, 9):                                        # in one launch, and in two
        assert cdll.pctc_prefix_decode(ctypes.byref(_problem(k=k)), *args, ln, at["state"], out.value, *outs, None) == 1


def test_binding_refuses_before_it_calls(lib):
    s = binding.PrefixBeam.__new__(binding.PrefixBeam)
    s.N, s.beams, s.max_frames, s.blank_id, s.started = 2, 4, 9, 0, False
    s.device = torch.device("cpu")
    s.frames = np.zeros(2, dtype=np.int64)
    c, l = torch.zeros(2, 5, 4, dtype=torch.int32), torch.zeros(2, 5, 4)
    for bad in [(c.long(), l), (c, l.double()), (c[:1], l[:1]), (c, l[:, :4]), (c[0], l[0]), (c.transpose(1, 2), l.transpose(1, 2))]:
        with pytest.raises(ValueError):
            s.advance(*bad)
    with pytest.raises(ValueError, match="one length"):
        s.advance(c, l, [5])
    s.frames[1] = 5
    with pytest.raises(ValueError, match="room"):
        s.advance(c, l)
    with pytest.raises(ValueError, match="no frames"):
        s.read()
    with pytest.raises(ValueError, match="CUDA device"):
        binding.PrefixBeam(2, 4, 9, 0, "cpu")
    with pytest.raises(ValueError, match="CUDA device"):
        binding.prefix_beam_decode(c, l, [5, 5], 0, 4)
