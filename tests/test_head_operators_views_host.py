"""Views that the binding of the operators around the head's matrix must not hand on, without a GPU: tensors that have a
device, a shape and strides, but no memory."""

import pytest
import torch
from torch._subclasses import FakeTensorMode

from paper_2609_33645_b200 import binding


def empty(*shape, dtype=torch.float32):
    with FakeTensorMode():
        return torch.empty(shape, dtype=dtype, device="cuda")


HEAD = (40, 16)
VIEWS = [
    ((3, 1, 16), (3, 5, 16)),            # a middle dimension: what the gradient of x.sum(1) looks like
    ((1, 5, 16), (3, 5, 16)),            # the outermost one
    ((1, 1, 16), (3, 5, 16)),            # both
    ((2, 1, 4, 16), (2, 3, 4, 16)),
    ((2, 3, 1, 16), (2, 3, 4, 16)),
    ((3, 1, 1), (3, 5, 1)),              # rows of one value
]
CALLS = dict(
    embed_out=lambda v: binding.embed(empty(*v.shape[:-1], dtype=torch.int32), empty(40, v.shape[-1]), out=v),
    embed_grad=lambda v: binding.embed_grad(empty(*v.shape[:-1], dtype=torch.int32), v, 40),
    dropout=lambda v: binding.dropout(v, 0.1, 1),
    dropout_residual=lambda v: binding.dropout(empty(*v.shape), 0.1, 1, residual=v),
    dropout_out=lambda v: binding.dropout(empty(*v.shape), 0.1, 1, out=v),
    quantized_logits=lambda v: binding.quantized_logits(v, binding.QuantizedHead(empty(40, v.shape[-1], dtype=torch.int8), empty(40))),
)


@pytest.mark.parametrize("first,shape", VIEWS)
@pytest.mark.parametrize("name", CALLS)
def test_expanded_views_are_refused(lib, name, first, shape):
    with pytest.raises(ValueError, match="one stride apart|overlap"):
        CALLS[name](empty(*first).expand(shape))


def test_expanded_matrices_are_refused(lib):
    tokens, row = empty(3, dtype=torch.int32), empty(1, 16).expand(HEAD)
    for call in (lambda: binding.embed(tokens, row), lambda: binding.embed_grad(tokens, empty(3, 16), dW=row), lambda: binding.quantize_rows(row)):
        with pytest.raises(ValueError, match="overlap"):
            call()


@pytest.mark.parametrize("bias", [
    lambda: empty(40),                                             # another type than that of the states
    lambda: empty(40, dtype=torch.float16),
    lambda: empty(39, dtype=torch.bfloat16),
    lambda: empty(40, 1, dtype=torch.bfloat16),
    lambda: empty(80, dtype=torch.bfloat16)[::2],
    lambda: empty(1, dtype=torch.bfloat16).expand(40),
    lambda: torch.zeros(40, dtype=torch.bfloat16),                 # not on the device
])
def test_recognition_with_the_head_in_8_bits_checks_its_bias(lib, bias):
    hidden = empty(2, 3, 16, dtype=torch.bfloat16)
    head = binding.QuantizedHead(empty(40, 16, dtype=torch.int8), empty(40))
    for decode in (lambda b: binding.topk_decode(hidden, head, b, [3, 2], 4), lambda b: binding.beam_decode(hidden, head, b, [3, 2], 0, 4)):
        with pytest.raises(ValueError, match="bias"):
            decode(bias())


def test_recognition_with_the_head_in_8_bits_checks_its_bias_beside_fp32_states(lib):
    head = binding.QuantizedHead(empty(40, 16, dtype=torch.int8), empty(40))
    with pytest.raises(ValueError, match="bias"):
        binding.topk_decode(empty(2, 3, 16), head, empty(40, dtype=torch.bfloat16), [3, 2], 4)


def test_calls_that_need_the_whole_matrix_refuse_one_in_8_bits(lib):
    hidden, targets = empty(2, 3, 16), empty(2, 4, dtype=torch.int32)
    head = binding.QuantizedHead(empty(40, 16, dtype=torch.int8), empty(40))
    with pytest.raises(TypeError, match="topk_decode"):
        binding.greedy_decode(hidden, head, None, [3, 2], 0)
    with pytest.raises(TypeError, match="QuantizedHead"):
        binding.pruned_ctc_fwd_bwd(hidden, head, None, targets, [3, 2], [1, 1], 0)
    with pytest.raises(TypeError, match="QuantizedHead"):
        binding.ctc_policy_fwd_bwd(hidden, head, None, targets, [3, 2], [1, 1], 0, empty(2), empty(2))


def test_recognition_checks_the_types_of_the_head(lib):
    half = dict(dtype=torch.bfloat16)
    for hidden, W, bias in ((empty(2, 3, 16, **half), empty(40, 16), None), (empty(2, 3, 16), empty(40, 16, **half), None),
                            (empty(2, 3, 16, **half), empty(40, 16, **half), empty(40)), (empty(2, 3, 16), empty(40, 16), empty(40, **half)),
                            (empty(2, 3, 16, dtype=torch.float16), empty(40, 16, dtype=torch.float16), None)):
        for call in (lambda: binding.topk_decode(hidden, W, bias, [3, 2], 4), lambda: binding.greedy_decode(hidden, W, bias, [3, 2], 0),
                     lambda: binding.beam_decode(hidden, W, bias, [3, 2], 0, 4)):
            with pytest.raises(ValueError, match="one type"):
                call()
