"""Reordering of beam states on the GPU: copies, so that every byte has to be equal."""

import numpy as np
import pytest
import torch

from paper_2609_33645_b200 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def plain(x, o, parents, lengths, axis):
    """o after the call, by indexing."""
    want = o.clone()
    for n in range(parents.shape[0]):
        for k in range(parents.shape[1]):
            p = int(parents[n, k])
            if not 0 <= p < x.shape[1]:
                continue
            if axis is None:
                want[n, k] = x[n, p]
            else:
                m = min(max(int(lengths[n]), 0), x.shape[axis])
                want[n, k].narrow(axis - 2, 0, m).copy_(x[n, p].narrow(axis - 2, 0, m))
    return want


def states_of(N, B, L, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)

    def r(*shape, dtype=torch.float32):
        x = torch.randn(N, B, *shape, generator=g, device=DEV) * 100
        return x.to(dtype) if dtype != torch.bool else x > 0

    return [(r(L, dtype=torch.int32), 2), (r(3, L, 8, dtype=torch.bfloat16), 3), (r(L, 5), 2), (r(7), None),
            (r(2, L, 3, dtype=torch.uint8), 3), (r(L, 1, 65, dtype=torch.bfloat16), 2), (r(2, L, dtype=torch.float64), 3),
            (r(513, dtype=torch.bfloat16), None), (r(dtype=torch.int64), None), (r(L, dtype=torch.bool), 2),
            (r(4, 2, L, 64, dtype=torch.bfloat16), 4)]


@pytest.mark.parametrize("N,B,K,L", [(1, 1, 1, 1), (1, 4, 4, 3), (3, 4, 4, 33), (2, 3, 5, 40), (2, 8, 8, 17), (2, 1, 6, 9),
                                     (1, 32, 32, 21), (5, 16, 16, 7), (2, 32, 1, 12), (1, 9, 9, 700)])
def test_into_other_buffers_and_in_place(N, B, K, L):
    g = torch.Generator(device=DEV).manual_seed(N + B + K + L)
    parents = torch.randint(-1, B + 1, (N, K), generator=g, device=DEV, dtype=torch.int32)     # -1 and B: no parent
    lengths = torch.randint(0, L + 1, (N,), generator=g, device=DEV, dtype=torch.int32)
    lengths[0] = L + 5                                     # cut to the axis
    if N > 1:
        lengths[1] = -3
    both = states_of(N, B, L, 1)
    xs, axes = [x for x, _ in both], [a for _, a in both]
    keep = [x.clone() for x in xs]
    outs = [torch.full(x.shape[:1] + (K,) + x.shape[2:], 1, dtype=x.dtype, device=DEV) for x in xs]
    want = [plain(x, o, parents, lengths, a) for x, o, a in zip(xs, outs, axes)]
    got = binding.beam_reorder(xs, parents, lengths=lengths, time_axes=axes, out=outs)
    for o, w, x, c in zip(got, want, xs, keep):
        assert torch.equal(o, w) and torch.equal(x, c)
    if K == B:
        want = [plain(x, x, parents, lengths, a) for x, a in zip(xs, axes)]
        got = binding.beam_reorder(xs, parents, lengths=lengths, time_axes=axes)
        for x, o, w in zip(xs, got, want):
            assert o is x and torch.equal(x, w)


@pytest.mark.parametrize("offset", range(1, 17, 3))
def test_odd_addresses_and_neighbours(offset):
    buf = torch.arange(2 * 4 * 101 + 64, device=DEV, dtype=torch.int32).to(torch.uint8)
    x = buf[offset:offset + 2 * 4 * 101].view(2, 4, 101)
    keep = buf.clone()
    parents = torch.tensor([[3, 2, 1, 0], [1, 1, 1, 2]], dtype=torch.int32, device=DEV)
    want = plain(x.clone(), x, parents, None, None)
    binding.beam_reorder([x], parents)
    assert torch.equal(x, want)
    assert torch.equal(buf[:offset], keep[:offset]) and torch.equal(buf[offset + 808:], keep[offset + 808:])


def test_a_cycle_in_place_and_back():
    x = torch.randn(3, 32, 5000, device=DEV)
    keep = x.clone()
    ring = (torch.arange(32, device=DEV, dtype=torch.int32) + 1) % 32
    parents = ring.expand(3, 32).contiguous()
    for _ in range(31):
        binding.beam_reorder([x], parents)
    assert torch.equal(x, keep.roll(-31, 1))
    binding.beam_reorder([x], parents)
    assert torch.equal(x, keep)


def test_interleaved_views_of_one_buffer():
    kv = torch.randn(2, 4, 2, 6, 16, device=DEV)
    keep = kv.clone()
    parents = torch.tensor([[1, 0, 0, 3], [2, 2, 3, 0]], dtype=torch.int32, device=DEV)
    lengths = torch.tensor([6, 2], dtype=torch.int32, device=DEV)
    k, v = kv[:, :, 0], kv[:, :, 1]
    binding.beam_reorder([k, v], parents, lengths=lengths, time_axes=[2, 2])
    for i, x in enumerate((k, v)):
        assert torch.equal(x, plain(keep[:, :, i], keep[:, :, i], parents, lengths, 2))
    with pytest.raises(binding.PctcError):
        binding.beam_reorder([k, k], parents)
    with pytest.raises(binding.PctcError):
        binding.beam_reorder([kv[:, :, 0], kv], parents)


def test_beam_major_states_and_shared_parents():
    g = torch.Generator(device=DEV).manual_seed(0)
    x = torch.randn(4, 3, 40, generator=g, device=DEV).transpose(0, 1)          # [N=3, B=4, 40], stored beam by beam
    parents = torch.randint(0, 4, (3, 4), generator=g, device=DEV, dtype=torch.int32)
    want = plain(x.clone(), x, parents, None, None)
    binding.beam_reorder([x], parents)
    assert torch.equal(x, want)
    one = torch.randn(3, 1, 40, generator=g, device=DEV)                        # one row for all beams of a first step
    out = torch.zeros(3, 4, 40, device=DEV)
    binding.beam_reorder([one], torch.zeros(3, 4, dtype=torch.int32, device=DEV), out=[out])
    assert torch.equal(out, one.expand(3, 4, 40))
    out.zero_()
    binding.beam_reorder([one.expand(3, 4, 40)], parents, out=[out])            # the same as a broadcast view
    assert torch.equal(out, one.expand(3, 4, 40))


def test_many_states_take_more_than_one_launch():
    xs = [torch.randn(1, 2, 3 + i % 5, device=DEV) for i in range(300)]
    parents = torch.tensor([[1, 0]], dtype=torch.int32, device=DEV)
    want = [x[:, [1, 0]] for x in xs]
    binding.beam_reorder(xs, parents)
    assert all(torch.equal(x, w) for x, w in zip(xs, want))


def test_offsets_beyond_32_bits():
    x = torch.empty(2, 3, 3, 300_000_000, dtype=torch.uint8, device=DEV)        # 5.4 GB, rows of 900 MB
    marks = [0, 1 << 28, 300_000_000 - 1]
    for n in range(2):
        for b in range(3):
            for m in marks:
                x[n, b, 2, m] = n * 100 + b * 10 + marks.index(m)
    parents = torch.tensor([[2, 0, 1], [1, 2, 0]], dtype=torch.int32, device=DEV)
    binding.beam_reorder([x], parents)
    for n in range(2):
        for b in range(3):
            assert [int(x[n, b, 2, m]) for m in marks] == [n * 100 + int(parents[n, b]) * 10 + i for i in range(3)]


def test_refusals():
    x = torch.zeros(2, 4, 6, 8, device=DEV)
    p = torch.zeros(2, 4, dtype=torch.int32, device=DEV)
    lengths = torch.zeros(2, dtype=torch.int32, device=DEV)
    for kw, match in [(dict(time_axes=[2]), "lengths"), (dict(time_axes=[1], lengths=lengths), "time axis"),
                      (dict(time_axes=[2, 2], lengths=lengths), "one entry"), (dict(out=[]), "one entry"),
                      (dict(out=[x[:, :3]]), "out must"), (dict(lengths=lengths.long()), "lengths"),
                      (dict(out=[torch.zeros(2, 4, 6, 8, device=DEV, dtype=torch.bfloat16)]), "out must")]:
        with pytest.raises(ValueError, match=match):
            binding.beam_reorder([x], p, **kw)
    with pytest.raises(ValueError, match="contiguous behind"):
        binding.beam_reorder([x.transpose(2, 3)], p)
    with pytest.raises(ValueError, match="parents"):
        binding.beam_reorder([x], p.long())
    with pytest.raises(ValueError, match="as many columns"):
        binding.beam_reorder([x], p[:, :3].contiguous())
    with pytest.raises(binding.PctcError):
        binding.beam_reorder([x], p, out=[torch.as_strided(x, (2, 4, 6, 8), (0, 48, 8, 1))])


def test_captured_into_a_graph():
    x = torch.randn(2, 4, 100, device=DEV)
    out = torch.zeros_like(x)
    parents = torch.zeros(2, 4, dtype=torch.int32, device=DEV)
    binding.beam_reorder([x], parents, out=[out])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.beam_reorder([x], parents, out=[out])
    parents.copy_(torch.tensor([[3, 1, 2, 0], [0, 0, 1, 1]], dtype=torch.int32))
    graph.replay()
    assert torch.equal(out, plain(x, out, parents, None, None))


def test_a_decoding_loop():
    """Selection and reordering as a decoder uses them: the histories that come out are those of a search by
    enumeration with the same step function."""
    N, B, V, steps, eos = 2, 4, 50, 6, 1
    g = torch.Generator(device=DEV).manual_seed(4)
    emb = torch.randn(V, 16, generator=g, device=DEV)
    head = torch.randn(V, 16, generator=g, device=DEV) * 0.7
    start = torch.randn(N, 16, generator=g, device=DEV)

    def logits_of(state):
        return state @ head.T

    state = start[:, None].repeat(1, B, 1)
    tokens = torch.full((N, B, steps), -1, dtype=torch.int32, device=DEV)
    scores = torch.full((N, B), -float("inf"), device=DEV)
    scores[:, 0] = 0.0
    finished = torch.zeros(N, B, dtype=torch.bool, device=DEV)
    # the same search on the host, hypothesis by hypothesis
    hyps = [[(0.0, [], start[n].double().cpu(), False)] for n in range(N)]
    e, h = emb.double().cpu(), head.double().cpu()
    for t in range(steps):
        r = binding.beam_select(logits_of(state), scores, B, finished=finished, eos_id=eos)
        binding.beam_reorder([state, tokens], r["parents"])
        scores, finished = r["scores"], r["finished"]
        tokens[:, :, t] = r["tokens"]
        state = torch.tanh(state + emb[r["tokens"].clamp(min=0).long()])
        for n in range(N):
            cand = []
            for b, (s, seq, st, done) in enumerate(hyps[n]):
                if done:
                    cand.append((s, b, eos))
                    continue
                lp = torch.log_softmax(st @ h.T, 0)
                cand += [(s + float(lp[v]), b, v) for v in range(V)]
            cand.sort(key=lambda c: (-c[0], c[1], c[2]))
            hyps[n] = [(s, hyps[n][b][1] + [v], torch.tanh(hyps[n][b][2] + e[v]), hyps[n][b][3] or v == eos) for s, b, v in cand[:B]]
    for n in range(N):
        for b in range(B):
            assert tokens[n, b].tolist() == hyps[n][b][1]
            # steps of fp32 products of 16 terms of size up to 4: within 1e-4
            assert abs(float(scores[n, b]) - hyps[n][b][0]) < 1e-4
            assert bool(finished[n, b]) == hyps[n][b][3]


@pytest.mark.parametrize("N,B", [(1, 4), (2, 4), (3, 1), (4, 32)])
@pytest.mark.parametrize("parts", [2, 5])
def test_views_that_interleave_by_utterance(N, B, parts):
    """Keys and values, or layers, of one batch-first buffer [N, parts, B, ...]."""
    g = torch.Generator(device=DEV).manual_seed(N * B + parts)
    packed = torch.randn(N, parts, B, 6, 16, generator=g, device=DEV)
    keep = packed.clone()
    parents = torch.randint(0, B, (N, B), generator=g, device=DEV, dtype=torch.int32)
    lengths = torch.randint(0, 7, (N,), generator=g, device=DEV, dtype=torch.int32)
    views = [packed[:, i] for i in range(parts)]
    binding.beam_reorder(views, parents, lengths=lengths, time_axes=[2] * parts)
    for i, x in enumerate(views):
        assert torch.equal(x, plain(keep[:, i], keep[:, i], parents, lengths, 2))
    keep.copy_(packed)
    binding.beam_reorder([views[0]], parents, out=[views[1]])                # from one part into another
    assert torch.equal(packed[:, 1], plain(keep[:, 0], keep[:, 1], parents, None, None))
    for bad in ([views[0], packed[:, 0, :, 2:]], [views[1], views[1]], [packed.flatten(0, 1)[:N], views[0]]):
        with pytest.raises(binding.PctcError):
            binding.beam_reorder(bad, parents)


def shared_bytes(N, B, D, sn, sb, first, second):
    at = torch.arange(200)
    x, y = (set(at.as_strided((N, B, D), (sn, sb, 1), o).flatten().tolist()) for o in (first, second))
    return bool(x & y)


@pytest.mark.parametrize("seed", range(60))
def test_random_views_of_one_buffer(seed):
    """Views with the strides of one layout, anywhere in one buffer: those that share a byte are refused, all others move."""
    rng = np.random.default_rng(seed)
    N, B, D = int(rng.integers(1, 4)), int(rng.integers(1, 4)), int(rng.integers(1, 5))
    if rng.random() < 0.5:                                                   # beams inside utterances, or the other way
        sb = D + int(rng.integers(0, 6))
        sn = B * sb + int(rng.integers(0, 25))
    else:
        sn = D + int(rng.integers(0, 6))
        sb = N * sn + int(rng.integers(0, 25))
    first, second = 4, 4 + int(rng.integers(0, 40))
    buf = torch.arange(200, device=DEV).to(torch.uint8)
    x, y = (buf.as_strided((N, B, D), (sn, sb, 1), at) for at in (first, second))
    parents = torch.from_numpy(rng.integers(0, B, (N, B)).astype(np.int32)).to(DEV)
    if shared_bytes(N, B, D, sn, sb, first, second):
        with pytest.raises(binding.PctcError):
            binding.beam_reorder([x, y], parents)
        return
    want = buf.clone()
    for at in (first, second):
        v = want.as_strided((N, B, D), (sn, sb, 1), at)
        v.copy_(plain(v.clone(), v, parents, None, None))
    binding.beam_reorder([x, y], parents)
    assert torch.equal(buf, want)


def test_conjugated_states_are_moved_when_resolved():
    z = torch.randn(2, 3, 7, device=DEV, dtype=torch.complex64)
    parents = torch.tensor([[2, 0, 0], [1, 1, 2]], dtype=torch.int32, device=DEV)
    out = torch.zeros_like(z)
    for args, kw in [(([z.conj()], parents), dict(out=[out])), (([z], parents), dict(out=[out.conj()])), (([z.conj()], parents), {})]:
        with pytest.raises(ValueError, match="resolve_conj"):
            binding.beam_reorder(*args, **kw)
    assert not out.any()
    binding.beam_reorder([z.conj().resolve_conj()], parents, out=[out])
    assert torch.equal(out, plain(z.conj().resolve_conj(), out, parents, None, None))


def test_saved_states_are_not_overwritten_unnoticed():
    parents = torch.tensor([[1, 0]], dtype=torch.int32, device=DEV)
    for into in (False, True):
        x = torch.randn(1, 2, 5, device=DEV, requires_grad=True)
        y, other = x * 2, torch.randn(1, 2, 5, device=DEV)
        loss = (y * y).sum()                                # saves y
        if into:
            binding.beam_reorder([other], parents, out=[y.detach()])
        else:
            binding.beam_reorder([y.detach()], parents)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.backward()
        assert other._version == 0                          # read only
    with torch.inference_mode():
        z = torch.randn(1, 2, 5, device=DEV)
    want = z[:, [1, 0]].clone()
    binding.beam_reorder([z], parents)                      # has no version to count
    assert torch.equal(z, want)
