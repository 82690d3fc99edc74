"""Distillation on the GPU: NaN and +infinity among the teacher's and the student's logits make their row NaN, loss and all of its gradient, and leave the
other rows the bits that they have without."""
import pytest
import torch

from lm_reference import TYPES
from paper_1810_10962_amd import bns
from test_gpu_distill import make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [5, 1001, 70001, 140001])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_nan_and_infinity_make_their_row_nan(value, vocab, dtype):
    tokens, k, tau = 7, 70, 2.0
    logits, ids, teacher, dloss = make(tokens, vocab, k, dtype, seed=8, missing=0.1)
    ids[:, 0], ids[:, 65] = 1, 3
    ids[4] = -1                                             # no entry: zero, whatever its teacher's logits are
    spec = bns.make_distill(tokens, vocab, k, dtype, temperature=tau)
    ids, dloss = ids.cuda(), dloss.cuda()
    loss, lse, out = torch.empty(tokens, device="cuda"), torch.empty(tokens, device="cuda"), torch.empty(tokens, vocab, dtype=TYPES[dtype], device="cuda")
    back = torch.empty_like(out)
    print(f"[gpu-case] distill {value} {vocab} {dtype}", flush=True)

    def call(z, u):
        bns.bns_distill_forward(spec, z, ids, u, dloss, loss, lse, out)
        bns.bns_distill_backward(spec, z, ids, u, lse, dloss, back)
        return [t.clone().cpu() for t in (loss, out, back)]

    clean = call(logits.cuda(), teacher.cuda())
    assert all(bool(torch.isfinite(t).all()) for t in clean)
    teacher[1, 0] = teacher[2, 65] = teacher[4, 3] = value
    logits[5, vocab - 1] = logits[6, 0] = value
    for got, want in zip(call(logits.cuda(), teacher.cuda()), clean):
        for row in range(tokens):
            if row in (1, 2, 5, 6):
                assert bool(torch.isnan(got[row]).all()), row
            else:
                assert torch.equal(got[row], want[row]), row
