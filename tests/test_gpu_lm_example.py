"""The example model: norms, loss without logits, distillation and 8-bit serving together, learning something."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("language_model_example", os.path.join(ROOT, "examples", "language_model.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_the_model_learns_is_distilled_and_served(example):
    print("[gpu-case] example model", flush=True)
    losses, distilled, same = example.main(steps=40, say=lambda text: print(text, flush=True))
    # 1000 words: chance is log(1000) = 6.9; the chain's own entropy is 0.91
    assert losses[0] > 6.0 and losses[-1] < 3.0
    assert distilled[-1] < 0.5 * distilled[0]
    assert same >= 0.9


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_its_gradients_are_those_of_the_same_model_in_torch(example, dtype):
    """Every parameter's gradient against torch's autograd through elementary operations in 64 bits.  In 32 bits the chain of products keeps six digits; in bf16
    each of the dozen roundings on the way costs 2^-8, independently."""
    print(f"[gpu-case] example gradients {dtype}", flush=True)
    model = example.Model(300, 64, 2, dtype, seed=3)
    now, then = example.chain(300, 257, 5)
    example.HeadLoss.apply(model.hidden(now), model.head, then).backward()
    wide = {n: p.detach().double().cpu().requires_grad_() for n, p in model.named_parameters()}
    norm = lambda s, w: w * s / torch.sqrt(s.pow(2).mean(1, keepdim=True) + example.EPS)  # noqa: E731
    stream = wide["embedding"][now.cpu()]
    delta = torch.zeros_like(stream)
    for i in range(2):
        stream = stream + delta
        delta = torch.nn.functional.gelu(norm(stream, wide[f"norms.{i}"]) @ wide[f"up.{i}"]) @ wide[f"down.{i}"]
    z = norm(stream + delta, wide["norms.2"]) @ wide["head"].T
    torch.nn.functional.cross_entropy(z, then.cpu(), ignore_index=-100).backward()
    for name, p in model.named_parameters():
        got, want = p.grad.double().cpu(), wide[name].grad
        assert float((got - want).norm() / want.norm()) < (1e-5 if dtype == torch.float32 else 12 * 2.0 ** -8), name
