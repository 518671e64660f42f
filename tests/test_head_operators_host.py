"""Lookup and its gradient, dropout, policy loss and the 8-bit head, without a GPU: argument checks of the C entry points and
of the binding, workspace sizes, and the generator's published test vectors."""

import ctypes

import pytest
import torch

from paper_2609_33645_b200 import binding
from tests.philox import philox

BASE = 1 << 20          # made-up addresses: these calls return before they touch a device
A = [BASE << i for i in range(4, 20)]        # far enough apart for everything here
INVALID, SMALL, UNSUPPORTED = 1, 2, 3


def embed(lib, p=None, tokens=A[0], W=A[1], scales=None, out=A[2], **kw):
    v = dict(M=10, V=100, D=16, ld_w=16, ld_x=16, dtype_w=0, dtype_x=0, scale=1.0, accumulate=0)
    v.update(kw)
    return lib.load().pctc_embed(ctypes.byref(binding.EmbedProblem(**v)) if p is None else None, tokens, W, scales, out, None)


def embed_grad(lib, tokens=A[0], grad=A[2], dW=A[1], ws=A[5], ws_bytes=1 << 20, **kw):
    v = dict(M=10, V=100, D=16, ld_w=16, ld_x=16, dtype_w=0, dtype_x=0, scale=1.0, accumulate=0)
    v.update(kw)
    return lib.load().pctc_embed_grad(ctypes.byref(binding.EmbedProblem(**v)), tokens, grad, dW, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,want", [
    (dict(M=-1), INVALID), (dict(V=0), INVALID), (dict(D=0), INVALID), (dict(ld_w=15), INVALID), (dict(ld_x=15), INVALID),
    (dict(scale=float("nan")), INVALID), (dict(scale=float("inf")), INVALID),
    (dict(M=1 << 31), UNSUPPORTED), (dict(M=(1 << 31) - 4096), UNSUPPORTED), (dict(V=1 << 31), UNSUPPORTED), (dict(D=(1 << 24) + 1, ld_w=1 << 25, ld_x=1 << 25), UNSUPPORTED),
    (dict(ld_x=1 << 40), UNSUPPORTED), (dict(ld_w=1 << 40), UNSUPPORTED),
    (dict(dtype_w=3), UNSUPPORTED), (dict(dtype_x=2), UNSUPPORTED),
    (dict(dtype_w=2), INVALID),                                # 8 bits need scales ...
    (dict(scales=A[6]), INVALID),                              # ... and only they do
    (dict(dtype_w=2, scales=A[6] + 2), INVALID),
    (dict(tokens=None), INVALID), (dict(tokens=A[0] + 2), INVALID), (dict(W=None), INVALID), (dict(W=A[1] + 1), INVALID),
    (dict(out=None), INVALID), (dict(out=A[2] + 1), INVALID), (dict(out=A[2] + 2, dtype_x=1), INVALID),
    (dict(out=A[1] + 3198), INVALID),                          # on the matrix' last value
    (dict(out=A[0] + 36), INVALID),                            # on the last token
    (dict(dtype_w=2, scales=A[6], out=A[6] + 396), INVALID),   # on the last scale
    (dict(p=0), INVALID),
    (dict(M=0, tokens=None, W=None, out=None), 0),
])
def test_lookups_are_refused_before_any_launch(lib, kw, want):
    assert embed(lib, **kw) == want


@pytest.mark.parametrize("kw,want", [
    (dict(M=-1), INVALID), (dict(dtype_w=2), UNSUPPORTED), (dict(dtype_x=2), UNSUPPORTED),
    (dict(tokens=None), INVALID), (dict(grad=None), INVALID), (dict(grad=A[2] + 1), INVALID), (dict(dW=None), INVALID),
    (dict(dW=A[1] + 2, dtype_w=1), INVALID), (dict(ws=None), INVALID), (dict(ws=A[5] + 16), INVALID), (dict(ws_bytes=64), SMALL),
    (dict(dW=A[2] + 318), INVALID), (dict(dW=A[0] + 36), INVALID),
    (dict(ws=A[1], dW=A[1] + 512), INVALID), (dict(grad=A[5] + 256), INVALID), (dict(tokens=A[5] + 256), INVALID),
    (dict(M=0, accumulate=1, tokens=None, grad=None, dW=None, ws=None), 0),
])
def test_gradients_are_refused_before_any_launch(lib, kw, want):
    assert embed_grad(lib, **kw) == want


def test_workspace_of_the_gradient_holds_no_vocabulary_by_width_array(lib):
    def need(**kw):
        v = dict(M=1000, V=100, D=64, ld_w=1 << 14, ld_x=1 << 14, dtype_w=0, dtype_x=0, scale=1.0, accumulate=0)
        v.update(kw)
        out = ctypes.c_size_t(0)
        assert lib.load().pctc_embed_grad_workspace_bytes(ctypes.byref(binding.EmbedProblem(**v)), ctypes.byref(out)) == 0
        return out.value
    assert need(V=200_000) - need(V=100_000) <= 4 * 100_000 + 512
    assert need(V=200_000, D=8192) - need(V=100_000, D=8192) <= 4 * 100_000 + 512


def dropout(lib, x=A[0], residual=None, step=None, out=A[1], **kw):
    v = dict(rows=4, cols=32, ld_x=32, ld_res=32, ld_out=32, dtype=0, reserved=0, p=0.1, seed=1, offset=0)
    v.update(kw)
    return lib.load().pctc_dropout(ctypes.byref(binding.DropoutProblem(**v)), x, residual, step, out, None)


@pytest.mark.parametrize("kw,want", [
    (dict(rows=-1), INVALID), (dict(cols=-1), INVALID), (dict(p=-0.01), INVALID), (dict(p=1.01), INVALID), (dict(p=float("nan")), INVALID),
    (dict(dtype=2), UNSUPPORTED), (dict(x=None), INVALID), (dict(out=None), INVALID), (dict(ld_x=31), INVALID),
    (dict(ld_out=31), INVALID), (dict(residual=A[2], ld_res=31), INVALID),
    (dict(x=A[0] + 1), INVALID), (dict(out=A[1] + 1), INVALID), (dict(residual=A[2] + 1), INVALID), (dict(x=A[0] + 2, dtype=1), INVALID),
    (dict(step=A[3] + 4), INVALID), (dict(step=A[1] + 248), INVALID),
    (dict(rows=1 << 30, cols=1 << 12, ld_x=1 << 12, ld_out=1 << 12), UNSUPPORTED),
    (dict(out=A[0] + 2), INVALID), (dict(out=A[0], ld_out=64), INVALID),          # into itself, shifted or spread
    (dict(residual=A[1] + 16), INVALID), (dict(residual=A[1], ld_res=64), INVALID),
    (dict(out=A[0] + 62, ld_x=64, ld_out=64), INVALID),                           # one value shared, a row
    (dict(rows=0, x=None, out=None), 0), (dict(cols=0, x=None, out=None), 0),
])
def test_dropouts_are_refused_before_any_launch(lib, kw, want):
    assert dropout(lib, **kw) == want


def policy(lib, logp=A[0], old=A[1], ref=None, adv=A[3], mask=None, lengths=None, grad=A[6], stats=A[7], count=A[8], ws=A[9],
           ws_bytes=1 << 20, **kw):
    v = dict(N=4, T=8, ld_logp=8, ld_old=8, ld_ref=8, ld_adv=0, ld_mask=8, ld_grad=8, clip_low=0.2, clip_high=0.2, kl_weight=0.1,
             reduction=0, negated=0)
    v.update(kw)
    return lib.load().pctc_policy_loss(ctypes.byref(binding.PolicyProblem(**v)), logp, old, ref, adv, mask, lengths, grad, stats,
                                       count, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,want", [
    (dict(N=0), INVALID), (dict(T=0), INVALID), (dict(N=1 << 20, T=1 << 11), UNSUPPORTED),
    (dict(clip_low=-0.1), INVALID), (dict(clip_low=1.1), INVALID), (dict(clip_high=-0.1), INVALID), (dict(clip_high=float("nan")), INVALID),
    (dict(kl_weight=float("inf")), INVALID), (dict(kl_weight=1e39), INVALID), (dict(reduction=3), INVALID), (dict(reduction=-1), INVALID),
    (dict(logp=None), INVALID), (dict(old=None), INVALID), (dict(adv=None), INVALID), (dict(stats=None), INVALID),
    (dict(count=None), INVALID), (dict(ws=None), INVALID), (dict(ws=A[9] + 8), INVALID), (dict(ws_bytes=8), SMALL),
    (dict(logp=A[0] + 2), INVALID), (dict(grad=A[6] + 1), INVALID), (dict(lengths=A[5] + 2), INVALID),
    (dict(ld_logp=7), INVALID), (dict(ld_old=7), INVALID), (dict(ref=A[2], ld_ref=7), INVALID), (dict(ld_adv=7), INVALID),
    (dict(mask=A[4], ld_mask=7), INVALID), (dict(ld_grad=7), INVALID),
    (dict(grad=A[0]), INVALID), (dict(stats=A[6] + 124), INVALID), (dict(count=A[7] + 8), INVALID), (dict(stats=A[1]), INVALID),
    (dict(mask=A[6] + 64), INVALID), (dict(lengths=A[8]), INVALID), (dict(ws=A[3], adv=A[3] + 256), INVALID),
    (dict(count=A[3] + 12), INVALID),
])
def test_policy_losses_are_refused_before_any_launch(lib, kw, want):
    assert policy(lib, **kw) == want


def matmul(lib, a=A[0], sa=A[1], b=A[2], sb=A[3], bias=None, c=A[4], status=None, **kw):
    v = dict(m=4, n=32, k=48, out_dtype=1, lda=48, ldb=48, ldc=32, bias_dtype=0, reserved=0)
    v.update(kw)
    return lib.load().pctc_i8_matmul(ctypes.byref(binding.I8Problem(**v)), a, sa, b, sb, bias, c, status, None)


def logits(lib, x=A[0], x_dtype=0, b=A[2], sb=A[3], bias=None, c=A[4], ws=A[6], ws_bytes=1 << 20, **kw):
    v = dict(m=4, n=32, k=48, out_dtype=1, lda=48, ldb=48, ldc=32, bias_dtype=0, reserved=0)
    v.update(kw)
    return lib.load().pctc_i8_logits(ctypes.byref(binding.I8Problem(**v)), x, x_dtype, b, sb, bias, c, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,want", [
    (dict(m=-1), INVALID), (dict(n=0), INVALID), (dict(k=0), INVALID), (dict(k=131072, lda=131072, ldb=131072), UNSUPPORTED),
    (dict(out_dtype=2), UNSUPPORTED), (dict(ldc=31), INVALID), (dict(ldc=1 << 40), UNSUPPORTED),
    (dict(bias=A[5], bias_dtype=2), UNSUPPORTED), (dict(bias=A[5] + 1), INVALID), (dict(bias=A[5] + 2, bias_dtype=1), INVALID),
    (dict(b=None), INVALID), (dict(b=A[2] + 8), INVALID), (dict(ldb=47), INVALID), (dict(ldb=56), INVALID), (dict(sb=None), INVALID),
    (dict(sb=A[3] + 2), INVALID), (dict(c=None), INVALID), (dict(c=A[4] + 2), INVALID), (dict(c=A[2] + 16), INVALID),
    (dict(c=A[3] + 124), INVALID), (dict(bias=A[4] + 8), INVALID), (dict(m=0, b=None, c=None), 0),
])
@pytest.mark.parametrize("call", [matmul, logits])
def test_products_are_refused_before_any_launch(lib, call, kw, want):
    assert call(lib, **kw) == want


def test_products_refuse_their_own_operands(lib):
    for kw in (dict(a=None), dict(a=A[0] + 8), dict(lda=47), dict(lda=56), dict(sa=None), dict(sa=A[1] + 1), dict(c=A[0] + 160),
               dict(c=A[1] + 12), dict(status=A[4] + 8), dict(status=A[4] + 2), dict(status=A[1] + 4)):
        assert matmul(lib, **kw) == INVALID, kw
    for kw in (dict(x=None), dict(x=A[0] + 1), dict(lda=47), dict(ws=None), dict(ws=A[6] + 8), dict(c=A[0] + 128),
               dict(ws=A[4]), dict(ws=A[2] - 256), dict(bias=A[6] + 256)):
        assert logits(lib, **kw) == INVALID, kw
    assert logits(lib, ws_bytes=128) == SMALL
    assert logits(lib, x_dtype=2) == UNSUPPORTED


@pytest.mark.parametrize("kw,want", [
    (dict(rows=-1), INVALID), (dict(cols=0), INVALID), (dict(ld_x=47), INVALID), (dict(ld_q=47), INVALID), (dict(dtype=2), UNSUPPORTED),
    (dict(x=None), INVALID), (dict(x=A[0] + 1), INVALID), (dict(q=None), INVALID), (dict(scales=None), INVALID),
    (dict(scales=A[2] + 2), INVALID), (dict(q=A[0] + 8), INVALID), (dict(scales=A[1]), INVALID), (dict(scales=A[0]), INVALID),
    (dict(rows=1 << 31), UNSUPPORTED), (dict(rows=0, x=None), 0),
])
def test_quantizations_are_refused_before_any_launch(lib, kw, want):
    v = dict(rows=4, cols=48, dtype=0, x=A[0], ld_x=48, q=A[1], ld_q=48, scales=A[2])
    v.update(kw)
    assert lib.load().pctc_i8_quantize(*v.values(), None) == want


def test_topk_with_the_head_in_8_bits_is_refused_before_any_launch(lib):
    f = lib.load()
    p = lib.make_problem(2, 10, 48, 100, 0, 0)
    n = (ctypes.c_int32 * 2)(10, 5)

    def call(ld=48, scales=A[2], ws=A[5], ws_bytes=1 << 30, k=4, W=A[1], prob=p):
        return f.pctc_i8_topk_decode(ctypes.byref(prob), A[0], W, ld, scales, None, n, k, A[3], A[4], ws, ws_bytes, None)
    for kw in (dict(ld=47), dict(ld=56), dict(scales=None), dict(scales=A[2] + 2), dict(ws=None), dict(ws=A[5] + 8), dict(k=3),
               dict(W=None), dict(W=A[1] + 8)):
        assert call(**kw) == INVALID, kw
    assert call(ws_bytes=1024) == SMALL
    assert call(prob=lib.make_problem(2, 10, 131072, 100, 0, 0), ld=131072) == UNSUPPORTED
    a, b = ctypes.c_size_t(0), ctypes.c_size_t(0)
    assert f.pctc_topk_workspace_bytes(ctypes.byref(p), n, 4, ctypes.byref(a)) == 0
    assert f.pctc_i8_topk_workspace_bytes(ctypes.byref(p), n, 4, ctypes.byref(b)) == 0
    assert a.value < b.value <= a.value + 15 * 128 + 15 * 4 + 512


def test_binding_refuses_what_it_cannot_hand_on(lib):
    ids, x, v = torch.zeros(3, dtype=torch.int32), torch.zeros(3, 16), torch.zeros(3)
    head = binding.QuantizedHead(torch.zeros(5, 16, dtype=torch.int8), torch.ones(5))
    with pytest.raises(ValueError, match="CUDA"):
        binding.embed(ids, x)
    with pytest.raises(ValueError, match="CUDA"):
        binding.embed_grad(ids, x, 5)
    with pytest.raises(ValueError, match="CUDA"):
        binding.dropout(x, 0.1, 1)
    with pytest.raises(ValueError, match="CUDA"):
        binding.policy_loss(v, v, v)
    with pytest.raises(ValueError, match="reduction"):
        binding.policy_loss(v, v, v, reduction="mean")
    with pytest.raises(ValueError, match="CUDA"):
        binding.quantize_rows(x)
    with pytest.raises(ValueError, match="CUDA"):
        binding.matmul_i8(head, head)
    with pytest.raises(ValueError, match="CUDA"):
        binding.quantized_logits(x, head)
    with pytest.raises(ValueError, match="CUDA"):
        binding.topk_decode(x[None], head, None, [3], 4)
    with pytest.raises(TypeError, match="tensor"):
        binding.embed([1, 2], x)
    with pytest.raises(ValueError, match="utt_weights"):
        binding.ctc_policy_fwd_bwd(None, None, None, None, None, None, 0, None, None, forward_only=True)


@pytest.mark.parametrize("counter,key,words", [
    # the test vectors that are published with the generator (Philox-4x32, ten rounds)
    ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0), (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1)),
])
def test_the_tests_own_generator_gives_the_published_words(counter, key, words):
    block, offset = counter[0] | counter[1] << 32, counter[2] | counter[3] << 32
    assert philox(block, offset, key[0] | key[1] << 32) == words


def test_a_policy_step_takes_the_defaults_of_the_calls_it_is_made_of(monkeypatch):
    import inspect

    calls = []

    def both(*args, forward_only=False, utt_weights=None, **kw):
        calls.append((forward_only, utt_weights is None))
        return dict(loss=torch.ones(2), flags=torch.zeros(2, dtype=torch.int32))
    defaults = {k: p.default for k, p in inspect.signature(binding.pruned_ctc_fwd_bwd).parameters.items() if p.kind is p.KEYWORD_ONLY}
    monkeypatch.setattr(binding, "pruned_ctc_fwd_bwd", both)
    monkeypatch.setattr(binding, "policy_loss", lambda *args, **kw: dict(grad=torch.ones(2)))
    assert defaults["forward_only"] is False and "utt_weights" in defaults
    res = binding.ctc_policy_fwd_bwd(None, None, None, None, None, None, 0, None, None, **defaults)
    assert calls == [(True, True), (False, False)] and "policy" in res


def test_products_report_a_wait_that_gave_up_if_they_are_asked(monkeypatch):
    class Native:
        def quantized_logits(self, x, q, scales, bias, dtype, workspace):
            return torch.zeros(x.shape[0], 5), "the workspace" if workspace is None else workspace

        def matmul_i8(self, a, sa, b, sb, bias, dtype, status):
            words.append(status)
            return torch.zeros(a.shape[0], 5)
    read, words, code = [], [], [0]
    monkeypatch.setattr(binding, "_native", Native)
    monkeypatch.setattr(binding, "workspace_status", lambda w: (read.append(w), code[0])[1])
    head = binding.QuantizedHead(torch.zeros(5, 16, dtype=torch.int8), torch.ones(5))
    x = torch.zeros(3, 16)
    binding.quantized_logits(x, head)
    binding.matmul_i8(head, head)
    assert read == [] and words == [None]
    for code[0] in (0, 3):
        for call, what in ((lambda **kw: binding.quantized_logits(x, head, **kw), "the workspace"),
                           (lambda **kw: binding.quantized_logits(x, head, workspace="mine", **kw), "mine"),
                           (lambda **kw: binding.matmul_i8(head, head, status="my word", **kw), "my word")):
            if code[0]:
                with pytest.raises(binding.PctcError) as e:
                    call(check_status=True)
                assert e.value.status == 6
            else:
                assert call(check_status=True).shape[1] == 5
            assert read.pop() == what
    with pytest.raises(binding.PctcError):                          # a word of its own where none is given
        binding.matmul_i8(head, head, check_status=True)
    assert words[-1].dtype == torch.int32 and int(words[-1].sum()) == 0
    read.clear()
    assert binding.quantized_logits(x[:0], head, check_status=True).shape == (0, 5) and read == []    # nothing ran, nothing was written
