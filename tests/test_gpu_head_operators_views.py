"""Views with several row dimensions, on the GPU: the operators around the head's matrix give what they give for a contiguous
copy, or refuse them before anything is launched."""

import pytest
import torch

from paper_2609_33645_b200 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def views():
    """[3, 5, 16] views whose rows lie one stride apart."""
    x = torch.randn(3, 5, 24, generator=gen(1), device=DEV)
    yield x[:, :, 4:20]
    yield x[:, :, 8:].clone()
    yield torch.randn(3, 1, 5, 40, generator=gen(2), device=DEV)[:, 0, :, :16]
    yield torch.randn(1, 15, 40, generator=gen(3), device=DEV)[0, :, 3:19].unflatten(0, (3, 5))


def test_rows_one_stride_apart():
    t = torch.randint(-1, 40, (3, 5), generator=gen(4), device=DEV, dtype=torch.int32)
    W = torch.randn(40, 16, generator=gen(5), device=DEV)
    head = binding.quantize_rows(W)
    for v in views():
        dense = v.clone(memory_format=torch.contiguous_format)
        assert v.shape == (3, 5, 16)
        assert torch.equal(binding.dropout(v, 0.3, 1), binding.dropout(dense, 0.3, 1))
        assert torch.equal(binding.dropout(dense, 0.3, 1, residual=v), binding.dropout(dense, 0.3, 1, residual=dense))
        assert torch.equal(binding.embed_grad(t, v, 40)["dW"], binding.embed_grad(t, dense, 40)["dW"])
        assert torch.equal(binding.quantized_logits(v, head), binding.quantized_logits(dense, head))
        binding.embed(t, W, out=v)
        assert torch.equal(v, binding.embed(t, W))
        binding.dropout(dense, 0.3, 1, out=v)
        assert torch.equal(v, binding.dropout(dense, 0.3, 1))


def test_dimensions_of_size_one_may_have_any_stride():
    row = torch.randn(16, generator=gen(1), device=DEV)
    for v in (row.expand(1, 1, 16), row[None, None], torch.randn(4, 16, generator=gen(2), device=DEV)[:, None].expand(4, 1, 16)):
        assert torch.equal(binding.dropout(v, 0.3, 1), binding.dropout(v.contiguous(), 0.3, 1))
        t = torch.full(v.shape[:-1], 3, dtype=torch.int32, device=DEV)
        assert torch.equal(binding.embed_grad(t, v, 5)["dW"], binding.embed_grad(t, v.contiguous(), 5)["dW"])


def test_expanded_rows_are_refused_and_leave_everything_as_it_was():
    t, dW = torch.zeros(3, 5, dtype=torch.int32, device=DEV), torch.full((4, 16), 7.0, device=DEV)
    whole = torch.full((200, 16), 7.0, device=DEV)
    x = torch.ones(3, 5, 16, device=DEV)
    for shape in ((3, 1, 16), (1, 5, 16), (1, 1, 16)):
        v = whole[:shape[0] * shape[1]].view(shape).expand(3, 5, 16)
        for call in (lambda: binding.embed(t, dW, out=v), lambda: binding.embed_grad(t, v, dW=dW), lambda: binding.dropout(v, 0.1, 1),
                     lambda: binding.dropout(x, 0.1, 1, residual=v), lambda: binding.dropout(x, 0.1, 1, out=v),
                     lambda: binding.quantized_logits(v, binding.quantize_rows(dW))):
            with pytest.raises(ValueError, match="one stride apart|overlap"):
                call()
    assert bool((whole == 7).all()) and bool((dW == 7).all())
