"""Beam selection and reordering, without a GPU: the oracle on planted answers, and the refusals."""

import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import pruned_ctc_oracle as O
from paper_2609_33645_b200 import binding

AT = 1 << 20            # a made-up address: these calls return before they touch a device


def test_oracle_selection():
    x = np.log(np.array([[0.5, 0.25, 0.25], [0.1, 0.8, 0.1]]))
    got, bad, _ = O.beam_select(x + 7.0, [-1.0, -1.0], 3)
    assert not bad and [(b, v) for _, b, v in got] == [(1, 1), (0, 0), (0, 1)]
    assert got[0][0] == pytest.approx(-1.0 + math.log(0.8))
    got, _, _ = O.beam_select(x, [-1.0, -np.inf], 9)
    assert [(b, v) for _, b, v in got] == [(0, 0), (0, 1), (0, 2)]
    got, _, _ = O.beam_select(x, [-1.0, -1.1], 2, finished=[False, True], eos=2)
    assert [(s, b, v) for s, b, v in got] == [(-1.1, 1, 2), (pytest.approx(-1 + math.log(0.5)), 0, 0)]
    x[0, 1] = np.nan
    assert O.beam_select(x, [-1.0, -1.0], 2)[1]


def _problem(**kw):
    d = dict(N=2, B=4, K=4, V=100, stride_n=400, stride_b=100, dtype=0, eos_id=-1)
    d.update(kw)
    return binding.BeamProblem(*[d[f] for f, _ in binding.BeamProblem._fields_])


@pytest.mark.parametrize("kw,want", [
    (dict(N=0), 1), (dict(B=0), 1), (dict(K=0), 1), (dict(V=0), 1), (dict(B=33), 3), (dict(K=33), 3),
    (dict(V=2 ** 21 + 1, stride_b=2 ** 22), 3), (dict(dtype=2), 3), (dict(eos_id=100), 1), (dict(eos_id=-2), 1),
    (dict(stride_b=99), 1), (dict(stride_n=-1), 1), (dict(N=2 ** 30), 3),
])
def test_bad_selections_are_refused_before_any_launch(lib, kw, want):
    p = _problem(**kw)
    assert lib.load().pctc_beam_select(ctypes.byref(p), AT, AT, None, AT, AT, AT, None, None, AT, 1 << 20, None) == want


def test_bad_pointers_are_refused_before_any_launch(lib):
    p, f = _problem(), lib.load().pctc_beam_select
    good = [AT, AT, None, AT, AT, AT, None, None, AT, 1 << 20, None]
    for i in (0, 1, 3, 4, 5):
        args = list(good)
        args[i] = None
        assert f(ctypes.byref(p), *args) == 1
        args[i] = AT + 1
        assert f(ctypes.byref(p), *args) == 1
    args = list(good)
    args[2] = AT                                            # ended beams without a token that ends
    assert f(ctypes.byref(p), *args) == 1
    assert f(None, *good) == 1
    out = ctypes.c_size_t(1)
    assert lib.load().pctc_beam_workspace_bytes(ctypes.byref(p), ctypes.byref(out)) == 0 and 0 < out.value < 1 << 20
    assert lib.load().pctc_beam_workspace_bytes(ctypes.byref(p), None) == 1
    p = _problem(N=64, B=8, V=151936, stride_n=8 * 151936, stride_b=151936)
    assert lib.load().pctc_beam_workspace_bytes(ctypes.byref(p), ctypes.byref(out)) == 0 and out.value > 0
    need = out.value
    assert need < 64 * 8 * 151936 / 50                      # maxima and sums, not logits
    assert f(ctypes.byref(p), *good[:8], None, need, None) == 1
    assert f(ctypes.byref(p), *good[:8], AT + 8, need, None) == 1
    assert f(ctypes.byref(p), *good[:8], AT, need - 1, None) == 2


def test_binding_refuses_what_it_cannot_hand_on(lib):
    x, s = torch.zeros(2, 4, 10), torch.zeros(2, 4)
    with pytest.raises(ValueError, match="CUDA"):
        binding.beam_select(x, s, 4)
    with pytest.raises(ValueError, match="bf16 or fp32"):
        binding.beam_select(x.double(), s, 4)
    with pytest.raises(ValueError, match="bf16 or fp32"):
        binding.beam_select(x[0], s, 4)


def _state(**kw):
    d = dict(src=AT, dst=AT, src_stride_n=400, src_stride_b=100, dst_stride_n=400, dst_stride_b=100, segments=1,
             segment_stride=0, units=25, unit_bytes=4, timed=0, reserved=0)
    d.update(kw)
    return binding.BeamState(*[d[f] for f, _ in binding.BeamState._fields_])


def _reorder(lib, states, N=2, B=4, K=4, parents=AT, lengths=None, n=None):
    table = (binding.BeamState * max(1, len(states)))(*states)
    return lib.load().pctc_beam_reorder(len(states) if n is None else n, table, N, B, K, parents, lengths, None)


FAR = AT * 16


@pytest.mark.parametrize("states,kw,want", [
    ([_state(src=None)], {}, 1), ([_state(dst=None)], {}, 1), ([_state(segments=0)], {}, 1), ([_state(units=-1)], {}, 1),
    ([_state(unit_bytes=0)], {}, 1), ([_state(timed=2)], {}, 1), ([_state(timed=1)], {}, 1),
    ([_state(unit_bytes=2 ** 50)], {}, 3),
    ([_state(segments=2, segment_stride=99)], {}, 1),                       # segments into each other
    ([_state(dst=FAR, dst_stride_b=99)], {}, 1),                            # written rows into each other
    ([_state(dst=FAR, dst_stride_n=399)], {}, 1), ([_state(dst=FAR, dst_stride_n=0)], {}, 1),
    ([_state(dst=FAR, src_stride_b=-100)], {}, 1),
    ([_state(dst_stride_b=104, dst_stride_n=416)], {}, 1),                  # in place with other strides
    ([_state()], dict(K=3), 1),                                             # in place with fewer beams
    ([_state(dst=AT + 100)], {}, 1), ([_state(dst=AT - 96)], {}, 1),        # rows into each other
    ([_state(), _state()], {}, 1),                                          # the same state twice
    ([_state(), _state(dst=FAR, src=AT + 50)], {}, 1),                      # what one writes another reads
    ([_state(dst=FAR), _state(src=FAR * 2, dst=FAR + 300)], {}, 1),
    ([_state(src_stride_b=200, dst_stride_b=200, src_stride_n=800, dst_stride_n=800),
      _state(src=AT + 99, dst=AT + 99, src_stride_b=200, dst_stride_b=200, src_stride_n=800, dst_stride_n=800)], {}, 1),
    ([_state()], dict(N=0), 1), ([_state()], dict(B=0), 1), ([_state()], dict(B=33, K=33), 3), ([_state()], dict(n=-1), 1),
    ([_state()], dict(parents=None), 1), ([_state()], dict(parents=AT + 2), 1),
    ([_state(timed=1)], dict(lengths=AT + 1), 1),
])
def test_bad_states_are_refused_before_any_launch(lib, states, kw, want):
    assert _reorder(lib, states, **kw) == want


@pytest.mark.parametrize("states,kw,want", [
    ([_state()], dict(parents=AT + 300), 1),                                # the parents are among what is written
    ([_state(dst=FAR)], dict(parents=FAR + 800 - 4), 1),                   # their first value is the last one written
    ([_state(dst=FAR)], dict(parents=FAR - 28), 1),                         # their last value the first
    ([_state(timed=1)], dict(parents=FAR, lengths=AT + 796), 1),
    ([_state(dst=FAR, src_stride_n=2 ** 46)], {}, 3), ([_state(dst=FAR, dst_stride_n=2 ** 46)], {}, 3),
    ([_state(dst=FAR)], dict(N=2 ** 26), 3),
])
def test_states_that_clash_with_the_rest_of_the_call_are_refused(lib, states, kw, want):
    assert _reorder(lib, states, **kw) == want


@pytest.mark.parametrize("alias", ["scores", "finished"])
def test_selection_in_place_needs_as_many_beams(lib, alias):
    p = _problem(K=3, eos_id=0)
    out, done = (FAR, FAR * 4) if alias == "scores" else (FAR * 2, FAR * 3)
    assert lib.load().pctc_beam_select(ctypes.byref(p), AT, FAR, FAR * 3, out, FAR * 5, FAR * 6, done, None, FAR * 7,
                                       1 << 20, None) == 1


def test_misaligned_flags_are_refused(lib):
    p = _problem()
    for off in (1, 2, 3):
        assert lib.load().pctc_beam_select(ctypes.byref(p), AT, AT * 2, None, AT * 3, AT * 4, AT * 5, None, AT * 6 + off, AT * 7,
                                           1 << 20, None) == 1


@pytest.mark.parametrize("name,at", [
    ("scores_out", "scores+4"), ("scores_out", "parents"), ("parents", "scores+28"), ("tokens", "parents+28"), ("flags", "tokens"),
    ("finished_out", "finished+7"), ("finished_out", "scores_out+31"), ("tokens", "finished+4"), ("finished", "tokens+8"),
    ("workspace", "scores-256"), ("workspace", "logits+256"), ("parents", "workspace+256"), ("flags", "workspace+0"),
    ("scores_out", "logits+1596"), ("tokens", "logits-28"), ("flags", "logits+196"), ("finished_out", "logits+1599"),
    ("finished_out", "logits-7"),
])
def test_outputs_of_a_selection_lie_apart(lib, name, at):
    """Logits of 2 x 4 rows of 200 bytes, 400 apart; 8 scores in and out."""
    p = _problem(stride_n=800, stride_b=200, eos_id=0)
    a = {x: FAR * (i + 1) for i, x in enumerate(("logits", "scores", "finished", "scores_out", "parents", "tokens", "finished_out",
                                                 "flags", "workspace"))}
    base = at.split("+")[0].split("-")[0]
    a[name] = a[base] + int(at[len(base):] or 0)
    assert lib.load().pctc_beam_select(ctypes.byref(p), *list(a.values()), 1 << 20, None) == 1


def test_nothing_to_move_is_no_error(lib):
    assert _reorder(lib, []) == 0
    assert _reorder(lib, [_state(units=0)]) == 0


def test_reorder_binding_refuses_what_it_cannot_hand_on(lib):
    p = torch.zeros(2, 4, dtype=torch.int32)
    with pytest.raises(ValueError, match="at least one"):
        binding.beam_reorder([], p)
    with pytest.raises(ValueError, match="CUDA"):
        binding.beam_reorder([torch.zeros(2, 4, 5)], p)


def test_lazily_conjugated_and_negated_views_are_refused(lib):
    """Their memory holds other values than they do."""
    p = torch.zeros(2, 4, dtype=torch.int32)
    z = torch.zeros(2, 4, 5, dtype=torch.complex64)
    for bad in (z.conj(), torch._neg_view(z.real.contiguous())):
        with pytest.raises(ValueError, match="resolve_conj"):
            binding.beam_reorder([bad], p)
        with pytest.raises(ValueError, match="resolve_conj"):
            binding.clip_grad_norm([bad], 1.0)
    with pytest.raises(ValueError, match="resolve_conj"):
        binding.beam_select(torch._neg_view(torch.zeros(2, 4, 10)), torch.zeros(2, 4), 4)
