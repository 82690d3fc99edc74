"""The autograd functions of the example model with tensors that are not dense, as slices and transposes hand them over, and a second derivative."""
import pytest
import torch

from test_gpu_lm_example import example  # noqa: F401

pytestmark = pytest.mark.gpu


def rnd(*shape, seed=0):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).cuda()


def arguments(name):
    """Dense ones, and the same values laid out otherwise."""
    targets = torch.randint(0, 200, (40,), generator=torch.Generator().manual_seed(1)).cuda()
    if name == "AddNorm":
        dense = [rnd(40, 64), rnd(40, 64, seed=1), rnd(64, seed=2)]
    elif name == "HeadLoss":
        dense = [rnd(40, 64), rnd(200, 64, seed=1), targets]
    else:
        top = torch.topk(rnd(40, 200, seed=3), 8)
        dense = [rnd(40, 200), top.indices, top.values]
    apart = [torch.stack([t, t], -1)[..., 0] if t.dim() == 1 else t.T.contiguous().T for t in dense]
    assert not any(t.is_contiguous() for t in apart) and all(torch.equal(a, b) for a, b in zip(dense, apart))
    return dense, apart


@pytest.mark.parametrize("name", ["AddNorm", "HeadLoss", "DistillLoss"])
def test_any_layout_gives_the_same_result(name, example):  # noqa: F811
    print(f"[gpu-case] example layouts {name}", flush=True)
    results = []
    for given in arguments(name):
        given = [t.detach().requires_grad_() if t.is_floating_point() and not (name == "DistillLoss" and i == 2) else t for i, t in enumerate(given)]
        out = getattr(example, name).apply(*given, *([2.0] if name == "DistillLoss" else []))
        out = out if isinstance(out, tuple) else (out,)
        sum((o * o).sum() for o in out).backward()
        results.append([o.detach() for o in out] + [t.grad for t in given if t.requires_grad])
    assert len(results[0]) > 1 and all(torch.equal(a, b) for a, b in zip(*results))


@pytest.mark.parametrize("name", ["AddNorm", "HeadLoss", "DistillLoss"])
def test_a_second_derivative_is_refused(name, example):  # noqa: F811
    print(f"[gpu-case] example second derivative {name}", flush=True)
    dense, _ = arguments(name)
    x = dense[0].requires_grad_()
    out = getattr(example, name).apply(x, *dense[1:], *([2.0] if name == "DistillLoss" else []))
    value = (out[1] if isinstance(out, tuple) else out).square().sum()
    (slope,) = torch.autograd.grad(value, x, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        slope.sum().backward()
