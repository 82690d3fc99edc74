"""Distillation from a teacher's top logits on the GPU against its definition in 64 bits (lm_reference).

Tolerances, with Z = max |z / tau| of a row.  The exponents are formed in fp32 in powers of two: z log2(e) / tau - maximum has an error of a few units
of 2^-24 of Z + 1, which is the relative error of a probability; the sum has at most 128 terms per thread in turn and some 30 above, (160)
2^-24 relative.  So p is off by at most P = (4 (Z + 1) + 160) 2^-24 of itself, and lse by as much in absolute terms; the teacher's side adds as
much with its own largest logit.  A gradient in 16 bits is rounded once, 2^-8."""
import pytest
import torch

import lm_reference as ref
from lm_reference import HALF_ULP, TYPES, Rows, vector, written
from paper_1810_10962_amd import bns

pytestmark = pytest.mark.gpu


def make(tokens, vocab, k, dtype, seed=0, missing=0.2):
    g = torch.Generator().manual_seed(seed * 7919 + tokens * 31 + vocab)
    logits = (2.5 * torch.randn(tokens, vocab, generator=g)).to(TYPES[dtype])
    ids = torch.randint(0, vocab, (tokens, k), generator=g)             # (an id may come twice)
    ids = torch.where(torch.rand(tokens, k, generator=g) < missing, torch.tensor([-1, vocab, -100, 2 ** 40])[torch.randint(0, 4, (tokens, k), generator=g)], ids)
    teacher = 10 * torch.rand(tokens, k, generator=g) - 3
    return logits, ids, teacher, 0.5 + torch.rand(tokens, generator=g)


def bounds(logits, teacher, tau):
    z = logits.double().abs().where(logits.double().abs() < torch.inf, torch.zeros(()).double()).amax(1) / tau
    u = teacher.double().abs().where(teacher.double().abs() < torch.inf, torch.zeros(()).double()).amax(1) / tau
    return (4 * (z + 1) + 160) * 2.0 ** -24, (8 * (u + 1) + 40) * 2.0 ** -24


def check(got_loss, got_lse, got_dz, logits, ids, teacher, tau, dloss, dtype):
    loss, lse, dz = ref.distill(logits.double(), ids, teacher.double(), tau, dloss.double())
    p_off, q_off = bounds(logits, teacher, tau)
    if got_lse is not None:
        assert bool(((got_lse.double().cpu() - lse).abs() <= p_off * (1 + lse.abs())).all())
        size = tau * tau * (lse.abs() + logits.double().abs().amax(1) / tau + 10)
        assert bool(((got_loss.double().cpu() - loss).abs() <= (p_off + 2 * q_off) * size).all())
    if got_dz is not None:
        c = (tau * dloss.double())[:, None]
        p = torch.exp(logits.double() / tau - lse[:, None])
        terms = c * (p * p_off[:, None] + (dz / c - p).abs() * q_off[:, None])
        off = (got_dz.double().cpu() - dz).abs() - (HALF_ULP[dtype] * dz.abs() + 2 * terms + 1e-37)
        assert bool((off <= 0).all()), f"worst excess {off.max().item():.3e}"


SHAPES = [(1, 1, 1), (2, 3, 5), (3, 8, 1), (5, 1000, 7), (4, 1001, 64), (2, 4096, 100), (3, 8191, 20), (2, 16385, 33), (3, 32003, 130), (2, 50257, 64), (2, 65536, 1000),
          (3, 100003, 50), (2, 131072, 64), (1, 131073, 3), (2, 262151, 1024)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens,vocab,k", SHAPES)
def test_forward_and_backward(tokens, vocab, k, dtype):
    for tau, pad in [(1.0, 0), (2.5, 3)]:
        logits, ids, teacher, dloss = make(tokens, vocab, k, dtype)
        stride = vocab + pad if pad else 0
        spec = bns.make_distill(tokens, vocab, k, dtype, temperature=tau, logits_stride=stride, dlogits_stride=stride + 1 if pad else 0)
        print(f"[gpu-case] distill {tokens}x{vocab} k={k} {dtype} tau={tau} pad={pad}", flush=True)
        z, out = Rows(logits, stride), Rows(torch.zeros(tokens, vocab), stride + 1 if pad else 0, TYPES[dtype], written=True)
        loss, lse = written(tokens), written(tokens)
        bns.bns_distill_forward(spec, z, ids.cuda(), teacher.cuda(), vector(dloss), loss, lse, out)
        check(loss.check()[0], lse.check()[0], out.check(), logits, ids, teacher, tau, dloss, dtype)
        # the loss alone has the same bits; the gradient alone, from that lse
        loss2, lse2 = torch.empty(tokens, device="cuda"), torch.empty(tokens, device="cuda")
        bns.bns_distill_forward(spec, z, ids.cuda(), teacher.cuda(), None, loss2, lse2, None)
        assert torch.equal(loss2, loss.t[0]) and torch.equal(lse2, lse.t[0])
        again = Rows(torch.zeros(tokens, vocab), stride + 1 if pad else 0, TYPES[dtype], written=True)
        bns.bns_distill_backward(spec, z, ids.cuda(), teacher.cuda(), lse2, vector(dloss), again)
        check(None, None, again.check(), logits, ids, teacher, tau, dloss, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens,vocab", [(700, 5000), (2500, 300), (3, 70001)])
def test_in_place_and_many_rows(tokens, vocab, dtype):
    logits, ids, teacher, dloss = make(tokens, vocab, 16, dtype, seed=1)
    spec = bns.make_distill(tokens, vocab, 16, dtype, temperature=2.0)
    print(f"[gpu-case] distill in place {tokens}x{vocab} {dtype}", flush=True)
    z, i, u, d = logits.cuda(), ids.cuda(), teacher.cuda(), dloss.cuda()
    loss, lse, out = torch.empty(tokens, device="cuda"), torch.empty(tokens, device="cuda"), torch.empty_like(z)
    bns.bns_distill_forward(spec, z, i, u, d, loss, lse, out)
    check(loss, lse, out, logits, ids, teacher, 2.0, dloss, dtype)
    z2, z3, out3 = z.clone(), z.clone(), torch.empty_like(z)
    bns.bns_distill_forward(spec, z2, i, u, d, loss, lse, z2)
    assert torch.equal(z2, out)
    bns.bns_distill_backward(spec, z3, i, u, lse, d, out3)
    bns.bns_distill_backward(spec, z3, i, u, lse, d, z3)
    assert torch.equal(z3, out3)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [40, 5000, 140001])
def test_rows_without_entries_and_masked_logits(vocab, dtype):
    tokens, k = 6, 8
    logits, ids, teacher, dloss = make(tokens, vocab, k, dtype, seed=2, missing=0.0)
    ids[:, :] = torch.arange(k) + 1
    ids[0] = -1                                             # no entry
    logits[0, 3] = float("nan")                             # (and nothing of the row reaches the gradient)
    ids[1], teacher[1] = 5, -float("inf")                   # entries, but the teacher gives them nothing
    logits[2, vocab // 2:] = -float("inf")                  # a vocabulary that is padded
    logits[3, 20:] = torch.finfo(TYPES[dtype]).min          # ... with the type's lowest value
    teacher[4, 1:] = -float("inf")                          # a single entry
    teacher[5] *= 30                                        # a teacher that is sure
    spec = bns.make_distill(tokens, vocab, k, dtype, temperature=1.0)
    print(f"[gpu-case] distill masks {vocab} {dtype}", flush=True)
    z, out = logits.cuda(), torch.empty(tokens, vocab, dtype=TYPES[dtype], device="cuda")
    loss, lse = torch.empty(tokens, device="cuda"), torch.empty(tokens, device="cuda")
    bns.bns_distill_forward(spec, z, ids.cuda(), teacher.cuda(), dloss.cuda(), loss, lse, out)
    back = torch.empty_like(out)
    bns.bns_distill_backward(spec, z, ids.cuda(), teacher.cuda(), lse, dloss.cuda(), back)
    for o in (out, back):
        assert bool((o[:2] == 0).all()) and bool((loss[:2] == 0).all())
        rest = slice(2, tokens)
        clean = torch.where(logits == torch.finfo(TYPES[dtype]).min, torch.tensor(-float("inf"), dtype=TYPES[dtype]), logits)
        # (bounds() goes by the logits that are not masked)
        check(loss[rest], lse[rest], o[rest], clean[rest], ids[rest], teacher[rest], 1.0, dloss[rest], dtype)


def test_gradient_against_differences():
    """The loss's own change along a direction, central difference with step 2^-5: third order h^2 / 6 = 2e-4, rounding 1e-6 / h = 3e-5."""
    tokens, vocab, k, tau, h = 20, 3000, 30, 2.0, 2.0 ** -5
    logits, ids, teacher, dloss = make(tokens, vocab, k, "f32", seed=3)
    spec = bns.make_distill(tokens, vocab, k, "f32", temperature=tau)
    d = torch.randn(tokens, vocab, generator=torch.Generator().manual_seed(5))
    loss, lse, out = torch.empty(tokens, device="cuda"), torch.empty(tokens, device="cuda"), torch.empty(tokens, vocab, device="cuda")
    print("[gpu-case] distill gradient against differences", flush=True)

    def value(step):
        bns.bns_distill_forward(spec, (logits + step * d).cuda(), ids.cuda(), teacher.cuda(), dloss.cuda(), loss, lse, out)
        return float((loss.double().cpu() * dloss.double()).sum())

    measured = (value(h) - value(-h)) / (2 * h)
    value(0.0)
    slope = float((out.double().cpu() * d.double()).sum())
    assert abs(slope - measured) < 2e-3 * float(out.double().cpu().norm() * d.double().norm()) / vocab ** 0.5


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [5, 1001, 8192, 70001, 140001])
def test_rows_of_the_lowest_value(vocab, dtype):
    """A mask of the type's lowest value that leaves nothing: all logits are alike, and so are the probabilities.  As a softmax does not change when a
    constant is taken off, the definition is evaluated on the differences to the row's maximum."""
    tokens, k, tau = 4, 5, 1.0
    logits, ids, teacher, dloss = make(tokens, vocab, k, dtype, seed=4, missing=0.0)
    ids[:, :] = torch.arange(k)
    lowest = torch.finfo(TYPES[dtype]).min
    logits[:2] = lowest
    teacher[1] = teacher[3] = torch.finfo(torch.float32).min
    logits[2] = 1e30                                        # alike, and far from zero
    spec = bns.make_distill(tokens, vocab, k, dtype, temperature=tau)
    print(f"[gpu-case] distill lowest value {vocab} {dtype}", flush=True)
    z, out = logits.cuda(), torch.empty(tokens, vocab, dtype=TYPES[dtype], device="cuda")
    loss, lse = torch.empty(tokens, device="cuda"), torch.empty(tokens, device="cuda")
    bns.bns_distill_forward(spec, z, ids.cuda(), teacher.cuda(), dloss.cuda(), loss, lse, out)
    apart = logits.double() - logits.double().amax(1, keepdim=True)
    want_loss, _, want = ref.distill(apart, ids, (teacher - teacher.amax(1, keepdim=True)).double(), tau, dloss.double())
    p_off, q_off = bounds(apart, teacher - teacher.amax(1, keepdim=True), tau)
    assert bool(((loss.double().cpu() - want_loss).abs() <= (p_off + 2 * q_off) * (apart.abs().amax(1) + 30)).all())
    assert bool(((lse.double().cpu() - logits.double().amax(1)).abs() <= 12 + 2.0 ** -22 * logits.double().abs().amax(1)).all())    # (ln 140001 < 12)
    p = torch.softmax(apart, 1)
    terms = dloss.double()[:, None] * (p * p_off[:, None] + (want / dloss.double()[:, None] - p).abs() * q_off[:, None])
    assert bool(((out.double().cpu() - want).abs() <= HALF_ULP[dtype] * want.abs() + 2 * terms + 1e-37).all())
    back = torch.empty_like(out)
    bns.bns_distill_backward(spec, z, ids.cuda(), teacher.cuda(), lse, dloss.cuda(), back)
    assert bool(torch.isfinite(back).all())                 # (its probabilities are as good as an lse of 2^-24 of its size, which is no good here)
