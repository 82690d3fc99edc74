"""What the examples hand to the library, on the CPU with stand-ins for the calls: the description says the types of the tensors that it gets."""
import importlib.util
import os

import pytest
import torch

from paper_1810_10962_amd import bns

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
TYPES = {bns.BNS_F32: torch.float32, bns.BNS_BF16: torch.bfloat16}


def _load(name):
    spec = importlib.util.spec_from_file_location(name + "_for_types", os.path.join(ROOT, "examples", name + ".py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.fixture
def calls(monkeypatch):
    """Stand-ins that keep the names of the calls made, with their tensors' types compared with the description's; outputs get ones."""
    made = []

    def stand_in(name, types):
        def call(spec, *args):
            made.append(name)
            for a, want in zip(args, types):
                want = TYPES[spec.dtype] if want == "same" else TYPES[spec.weight_dtype] if want == "weight" else want
                assert a is None or a.dtype == want and a.is_contiguous() or want == "any", (name, a.dtype, want)
            for a, want in zip(args, types):
                if want == torch.float32 and a is not None:
                    a.fill_(1)
        monkeypatch.setattr(bns, "bns_" + name, call)

    stand_in("rms_forward", ["same", "same", "weight", "same", "same", "any", torch.float32])
    stand_in("rms_backward", ["same", "weight", torch.float32, "same", "same", "same", torch.float32])
    stand_in("qk_forward", ["any", "any", "weight", "weight", torch.int64, torch.float64])
    stand_in("qk_backward", ["any", "any", "weight", "weight", torch.int64, torch.float64, "same", "same", "any", "any", torch.float32, torch.float32])
    stand_in("logprob_forward", ["same", torch.int64, torch.float32, torch.float32, torch.float32])
    stand_in("logprob_backward", ["same", torch.int64, torch.float32, torch.float32, torch.float32, torch.float32, "same"])
    stand_in("head_forward", ["same", "same", torch.int64, torch.float32, torch.float32])
    stand_in("head_backward", ["same", "same", torch.int64, torch.float32, torch.float32, "same", "same"])
    stand_in("distill_forward", ["same", torch.int64, torch.float32, torch.float32, torch.float32, torch.float32, "same"])
    return made


@pytest.mark.parametrize("weights", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_weights_of_either_type(calls, dtype, weights):
    """Norms' weights as a model has them that was converted as a whole, too."""
    example = _load("policy_gradient")
    delta, stream, w = torch.randn(5, 64, dtype=dtype), torch.randn(5, 64, dtype=dtype), torch.ones(64, dtype=weights, requires_grad=True)
    total, y = example.AddNorm.apply(delta.requires_grad_(), stream, w)
    (total.sum() + y.sum()).backward()
    assert w.grad.dtype == weights and bool((w.grad == 1).all())
    packed, turns = torch.randn(5, 6 * 16, dtype=dtype, requires_grad=True), torch.rand(8, dtype=torch.float64)
    wq, wk = (torch.ones(16, dtype=weights, requires_grad=True) for _ in "qk")
    q, k, v = example.QueriesKeys.apply(packed, wq, wk, torch.arange(5), turns, 4, 1)
    (q.sum() + k.sum() + v.sum()).backward()
    assert wq.grad.dtype == wk.grad.dtype == weights and bool((wq.grad == 1).all()) and bool((wk.grad == 1).all())
    assert calls == ["rms_forward", "rms_backward", "qk_forward", "qk_backward"]


def test_weights_of_two_types_are_refused(calls):
    example = _load("policy_gradient")
    with pytest.raises(TypeError):
        example.QueriesKeys.apply(torch.randn(5, 6 * 16), torch.ones(16), torch.ones(16).bfloat16(), torch.arange(5), torch.rand(8, dtype=torch.float64), 4, 1)
    assert calls == []


def test_operands_of_two_types_are_refused(calls):
    """As a product under autocast leaves them beside a residual stream in 32 bits: the library has one type for both."""
    example = _load("language_model")
    with pytest.raises(TypeError):
        example.AddNorm.apply(torch.randn(5, 64).bfloat16(), torch.randn(5, 64), torch.ones(64))
    with pytest.raises(TypeError):
        example.HeadLoss.apply(torch.randn(5, 64).bfloat16(), torch.randn(30, 64), torch.arange(5))
    assert calls == []


@pytest.mark.parametrize("whole", [torch.int32, torch.int64])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_whole_numbers_of_either_size(calls, dtype, whole):
    """Targets, ids and positions as a data loader has them, in 32 bits too; a teacher in the student's type."""
    example, language_model = _load("policy_gradient"), _load("language_model")
    logits, targets = torch.randn(5, 30, dtype=dtype, requires_grad=True), torch.arange(10, dtype=whole)[::2]
    logp, entropy = example.LogProb.apply(logits, targets, 1.0)
    (logp.sum() + entropy.sum()).backward()
    example.QueriesKeys.apply(torch.randn(5, 6 * 16, dtype=dtype), torch.ones(16), torch.ones(16), torch.arange(10, dtype=whole)[::2], torch.rand(8), 4, 1)
    hidden, weight = torch.randn(5, 64, dtype=dtype, requires_grad=True), torch.randn(30, 64, dtype=dtype)
    language_model.HeadLoss.apply(hidden, weight, targets).backward()
    language_model.DistillLoss.apply(torch.randn(5, 30, dtype=dtype), torch.zeros(5, 3, dtype=whole), torch.randn(5, 3, dtype=dtype), 2.0)
    assert calls == ["logprob_forward", "logprob_backward", "qk_forward", "head_forward", "head_backward", "distill_forward"]
