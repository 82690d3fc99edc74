"""Log probabilities, entropy, alternatives and their gradient on the GPU against the definition in 64 bits (answers_reference).

Tolerances, with u = 2^-24, z = (logit - largest) / tau and Z the largest |z| of a row that counts (terms beyond 104 are below what 32 bits hold).  The exponent of a term is
formed with three roundings (3 u |z|) and the power costs 2 u; a thread adds 32 terms in turn for each of its steps, and 30 additions join threads and segments: the sum is off by
P = (3 Z + 100 + steps) u of itself, and s by that and 2 u |s| of the logarithm.  log p: P + 4 u (|z| + |s|).  entropy = s + sum p |z|: (1 + entropy) 2 P.  Gradients: log p
from the given stats (6 |log p| + 6) u, and p as much relative; results rounded once."""
import math

import pytest
import torch

import answers_reference as ref
from answers_reference import HALF_ULP, TYPES, U, tail_is_whole, written
from paper_1810_10962_amd import bns

pytestmark = pytest.mark.gpu


def make(tokens, vocab, dtype, seed=0, left_out=0.2):
    g = torch.Generator().manual_seed(seed * 7919 + tokens * 31 + vocab)
    logits = (2.5 * torch.randn(tokens, vocab, generator=g)).to(TYPES[dtype])
    targets = torch.randint(0, vocab, (tokens,), generator=g)
    outside = torch.tensor([-1, vocab, -100, 2 ** 40])[torch.randint(0, 4, (tokens,), generator=g)]
    targets = torch.where(torch.rand(tokens, generator=g) < left_out, outside, targets)
    return logits, targets, torch.randn(tokens, generator=g), torch.randn(tokens, generator=g)


def bound(logits, tau):
    z = (logits - logits.amax(1, keepdim=True)) / tau
    z = torch.where(z.isnan() | (z < -104), 0.0, z).abs().amax(1)
    return (3 * z + 100 + logits.shape[1] / 4096) * U, z


def run_forward(logits, targets, top, tau, dtype, stride=0):
    tokens, vocab = logits.shape
    spec = bns.make_logprob(tokens, vocab, dtype, top=top, temperature=tau, logits_stride=stride)
    x = torch.full((1 + tokens * (stride or vocab),), float("nan"), dtype=TYPES[dtype])      # (from its second element on)
    x[1:].view(tokens, -1)[:, :vocab] = logits
    x = x.cuda()[1:]
    outs = {"logp": written(tokens), "entropy": written(tokens), "stats": written(tokens, 2)}
    if top:
        outs.update(top_ids=written(tokens, top, dtype=torch.int64), top_logp=written(tokens, top))
    room = bns.bns_logprob_workspace_bytes(spec)
    workspace, space = written(room, dtype=torch.uint8)
    o = {n: outs[n][1] if n in outs else None for n in ("logp", "entropy", "stats", "top_ids", "top_logp")}
    bns.bns_logprob_forward(spec, x, targets.cuda(), o["logp"], o["entropy"], o["stats"], o["top_ids"], o["top_logp"], space)
    for whole, part in outs.values():
        tail_is_whole(whole, part.numel())
    tail_is_whole(workspace, room)
    return {n: None if v is None else v.cpu() for n, v in o.items()}


def check_forward(got, logits, targets, top, tau):
    x = logits.double()
    m, s, logp, given, entropy = ref.logprob(x, targets, tau)
    off, z = bound(x, tau)
    assert torch.equal(got["stats"][:, 0].double(), m)
    assert bool(((got["stats"][:, 1].double() - s).abs() <= off + 2 * U * s.abs()).all())
    same = given == got["logp"].double()             # (-infinity among them)
    assert bool((same | ((got["logp"].double() - given).abs() <= off + 4 * U * (given.abs() + 2 * s.abs()))).all())
    assert bool(((got["entropy"].double() - entropy).abs() <= 2 * off * (1 + entropy)).all())
    if top:
        ids = ref.top(logits, top)
        assert torch.equal(got["top_ids"], ids)
        want = logp.gather(1, ids)
        same = want == got["top_logp"].double()
        assert bool((same | ((got["top_logp"].double() - want).abs() <= off[:, None] + 4 * U * (want.abs() + 2 * s.abs()[:, None]))).all())


SHAPES = [(1, 1, 1), (2, 3, 3), (3, 8, 2), (5, 9, 9), (2, 130, 128), (7, 1000, 5), (4, 1001, 20), (3, 4096, 64), (2, 8191, 1), (2, 16385, 33), (9, 32003, 128), (2, 50257, 5),
          (1, 65536, 20), (3, 100003, 50), (1, 131072, 20), (2, 131073, 128), (1, 262151, 7), (1500, 257, 4), (1100, 9001, 6), (140, 80001, 6),
          (1200, 16001, 20), (150, 40000, 128), (600, 1023, 128), (64, 70000, 33)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens,vocab,top", SHAPES)
def test_forward(tokens, vocab, top, dtype):
    for tau, pad, k in [(1.0, 0, top), (0.6, 3, 0)] + ([(2.5, 5, top)] if tokens < 100 else []):
        logits, targets, _, _ = make(tokens, vocab, dtype)
        print(f"[gpu-case] logprob {tokens}x{vocab} top={k} {dtype} tau={tau} pad={pad}", flush=True)
        check_forward(run_forward(logits, targets, k, tau, dtype, vocab + pad if pad else 0), logits, targets, k, tau)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens,vocab,top", SHAPES)
def test_backward(tokens, vocab, top, dtype):
    logits, targets, dlogp, dentropy = make(tokens, vocab, dtype, seed=1)
    tau, pad = (1.0, 0) if top % 2 else (0.8, 3)
    print(f"[gpu-case] logprob backward {tokens}x{vocab} {dtype} tau={tau} pad={pad}", flush=True)
    m, s, _, _, entropy = ref.logprob(logits.double(), targets, tau)
    stats, entropy = torch.stack([m, s], 1).float(), entropy.float()
    stride = vocab + pad
    x = torch.full((tokens, stride), float("nan"), dtype=TYPES[dtype])
    x[:, :vocab] = logits
    x = x.cuda()
    spec = bns.make_logprob(tokens, vocab, dtype, temperature=tau, logits_stride=stride if pad else 0, dlogits_stride=stride + 1 if pad else 0)
    for g, h in [(dlogp, dentropy), (dlogp, None), (None, dentropy)]:
        whole = torch.full((tokens * (stride + 1) + 64,), 7.0, device="cuda").to(TYPES[dtype])
        out = whole[:tokens * (stride + 1)].view(tokens, stride + 1)[:, :vocab] if pad else whole[:tokens * vocab].view(tokens, vocab)
        bns.bns_logprob_backward(spec, x, None if g is None else targets.cuda(), stats.cuda(), entropy.cuda(), None if g is None else g.cuda(),
                                 None if h is None else h.cuda(), out)
        gg, hh = (torch.zeros(tokens) if v is None else v for v in (g, h))
        want, logp, p = ref.logprob_backward(logits.double(), targets, stats.double(), entropy.double(), gg.double(), hh.double(), tau)
        kept = (targets >= 0) & (targets < vocab)
        ga = torch.where(kept, gg, 0.0).double().abs()[:, None]
        ha, each = hh.double().abs()[:, None], (6 * logp.abs() + 6) * U
        size = ga + ha * (logp.abs() + entropy.double().abs()[:, None])
        off = p * (each * size + ha * each + 5 * U * size) / tau + 1e-36
        at = torch.zeros_like(p)
        at.scatter_(1, torch.where(kept, targets, 0)[:, None], 2 * U * ga / tau)
        worst = ((out.double().cpu() - want).abs() - (off + at + (HALF_ULP[dtype] + U) * want.abs())).max().item()
        assert worst <= 0, f"worst excess {worst:.3e}"
        if pad:
            assert bool((whole[:tokens * (stride + 1)].view(tokens, stride + 1)[:, vocab:] == 7).all())
        assert bool((whole[tokens * (stride + 1) if pad else tokens * vocab:] == 7).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_backward_in_place(dtype):
    for tokens, vocab in [(3, 70001), (700, 3000)]:
        logits, targets, dlogp, dentropy = make(tokens, vocab, dtype, seed=2)
        print(f"[gpu-case] logprob backward in place {tokens}x{vocab} {dtype}", flush=True)
        got = run_forward(logits, targets, 0, 1.0, dtype)
        spec = bns.make_logprob(tokens, vocab, dtype)
        args = [targets.cuda(), got["stats"].cuda(), got["entropy"].cuda(), dlogp.cuda(), dentropy.cuda()]
        x, out = logits.cuda(), torch.empty(tokens, vocab, dtype=TYPES[dtype], device="cuda")
        bns.bns_logprob_backward(spec, x, *args, out)
        bns.bns_logprob_backward(spec, x, *args, x)
        assert torch.equal(x, out)


ORDERS = ["equal", "rising", "falling", "two values", "few above many equal", "one above", "masked but three", "masked but one", "all masked", "lowest everywhere",
          "lowest but some", "zeros of both signs", "nan and others", "infinite", "rising then equal"]


def order(kind, vocab, dtype):
    t = TYPES[dtype]
    x = torch.zeros(vocab)
    i = torch.arange(vocab)
    if kind == "rising":
        x = (i.float() / vocab * 30).sort().values
    elif kind == "falling":
        x = -(i.float() / vocab * 30)
    elif kind == "two values":
        x = (i % 7 == 3).float()
    elif kind == "few above many equal":
        x[vocab // 2:vocab // 2 + 3] = torch.tensor([2.0, 5.0, 2.0])[:len(x[vocab // 2:vocab // 2 + 3])]
    elif kind == "one above":
        x[vocab - 1] = 1.0
    elif kind == "masked but three":
        x = torch.full((vocab,), -math.inf)
        x[[0, vocab // 2, vocab - 1]] = torch.tensor([1.0, 3.0, 2.0])
    elif kind == "masked but one":
        x = torch.full((vocab,), -math.inf)
        x[vocab // 3] = -5.0
    elif kind == "all masked":
        x = torch.full((vocab,), -math.inf)
    elif kind == "lowest everywhere":
        return torch.full((vocab,), torch.finfo(t).min, dtype=t)
    elif kind == "lowest but some":
        x = torch.full((vocab,), torch.finfo(t).min, dtype=torch.float32)
        x[vocab // 2] = 3.0
        x[vocab // 3] = 3.5
    elif kind == "zeros of both signs":
        x = torch.where(i % 2 == 0, -0.0, 0.0)
    elif kind == "nan and others":
        x = torch.randn(vocab, generator=torch.Generator().manual_seed(vocab))
        x[vocab // 2] = float("nan")
    elif kind == "infinite":
        x = torch.randn(vocab, generator=torch.Generator().manual_seed(vocab))
        x[vocab // 2] = math.inf
    elif kind == "rising then equal":
        x = torch.minimum(i.float() / vocab * 60, torch.tensor(30.0))
    return x.to(t)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [5, 1001, 20000, 70001])
@pytest.mark.parametrize("tokens", [1, 150, 1030])
def test_orders_and_masks(tokens, vocab, dtype):
    """Rows whose alternatives are hard to find, whose masks leave little or nothing, and special values, on one block a row and on several."""
    if tokens > 150 and vocab > 20000:
        vocab = 30001
    kinds = [ORDERS[i % len(ORDERS)] for i in range(tokens)] if tokens > 1 else ORDERS
    top = min(vocab, 20)
    for rows in [list(range(tokens))] if tokens > 1 else [[i] for i in range(len(ORDERS))]:
        made = {k: order(k, vocab, dtype) for k in {kinds[r] for r in rows}}
        logits = torch.stack([made[kinds[r]] for r in rows])
        targets = torch.tensor([(r * 7) % vocab for r in rows])
        print(f"[gpu-case] logprob orders {len(rows)}x{vocab} {dtype} {[kinds[r] for r in rows][:15]}", flush=True)
        got = run_forward(logits, targets, top, 1.0, dtype)
        bad = torch.tensor([kinds[r] in ("nan and others", "infinite") for r in rows])
        fine = ~bad
        if bool(fine.any()):
            check_forward({n: v[fine] for n, v in got.items()}, logits[fine], targets[fine], top, 1.0)
        assert torch.equal(got["top_ids"], ref.top(logits, top))
        for n in ("logp", "entropy", "top_logp"):
            assert bool(got[n][bad].isnan().all()), n
        assert bool(got["stats"][bad][:, 1].isnan().all())
        empty = torch.tensor([kinds[r] == "all masked" for r in rows])
        assert bool((got["entropy"][empty] == 0).all()) and bool((got["logp"][empty] == -math.inf).all()) and bool((got["stats"][empty][:, 1] == 0).all())
        # gradients: nothing for rows that are empty, NaN for bad ones, finite and right elsewhere
        spec = bns.make_logprob(len(rows), vocab, dtype)
        out = torch.empty(len(rows), vocab, dtype=TYPES[dtype], device="cuda")
        g, h = torch.full((len(rows),), 0.5), torch.full((len(rows),), -0.25)
        bns.bns_logprob_backward(spec, logits.cuda(), targets.cuda(), got["stats"].cuda(), got["entropy"].cuda(), g.cuda(), h.cuda(), out)
        out = out.cpu()
        assert bool((out[empty] == 0).all()) and bool(out[bad].isnan().all())
        use = fine & ~empty
        if bool(use.any()):
            want, logp, p = ref.logprob_backward(logits[use].double(), targets[use], got["stats"][use].double(), got["entropy"][use].double(), g[use].double(), h[use].double(), 1.0)
            reach = torch.where(p == 0, 0.0, logp.abs())
            off = p * (12 * reach + 12) * U * (1 + reach) + 2 * U + (HALF_ULP[dtype] + U) * want.abs() + 1e-36
            assert bool(((out[use].double() - want).abs() <= off).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens,vocab", [(1, 5), (3, 1000), (2, 20000), (1, 131072), (300, 20001)])
def test_zeros_of_both_signs_in_words_of_their_own_tie(tokens, vocab, dtype):
    """Negative zeros in words that hold nothing as large, and positive ones in others, behind them and before them; the rest is negative.  A wave for a row, four, and several blocks."""
    print(f"[gpu-case] logprob zeros apart {tokens}x{vocab} {dtype}", flush=True)
    e = 4 if dtype == "f32" else 8
    i = torch.arange(vocab)
    lane, third = i // e % 64, i % e == min(3, vocab - 1)
    x = -1.0 - i.float() / vocab
    x = torch.where(third & (lane < 10), 0.0, x)
    logits = torch.stack([torch.where((x == 0) & ((lane % 9 == 0) == (row % 2 == 0)), -0.0, x) for row in range(tokens)]).to(TYPES[dtype])
    targets = torch.zeros(tokens, dtype=torch.int64)
    for top in (1, 2, 5, 20):
        if top <= vocab:
            check_forward(run_forward(logits, targets, top, 1.0, dtype), logits, targets, top, 1.0)


def test_rows_without_gradient_are_zero_whatever_they_hold():
    vocab, tokens = 3000, 4
    print("[gpu-case] logprob rows without gradient", flush=True)
    logits, _, _, _ = make(tokens, vocab, "f32", seed=3)
    logits[0, 5], logits[1, 6] = float("nan"), math.inf
    targets = torch.tensor([5, -100, 7, vocab])
    dlogp, dentropy = torch.tensor([0.0, float("nan"), 0.0, 3.0]), torch.zeros(tokens)
    got = run_forward(logits, targets, 0, 1.0, "f32")
    out = torch.empty(tokens, vocab, device="cuda")
    bns.bns_logprob_backward(bns.make_logprob(tokens, vocab, "f32"), logits.cuda(), targets.cuda(), got["stats"].cuda(), got["entropy"].cuda(), dlogp.cuda(), dentropy.cuda(), out)
    assert bool((out == 0).all())


def test_gradient_against_differences():
    """The change of sum(dlogp logp + dentropy entropy) along a direction, central difference with step 2^-5: third order h^2 / 6 = 2e-4, rounding 1e-6 / h = 3e-5."""
    tokens, vocab, tau, h = 20, 3000, 1.3, 2.0 ** -5
    logits, targets, dlogp, dentropy = make(tokens, vocab, "f32", seed=4)
    d = torch.randn(tokens, vocab, generator=torch.Generator().manual_seed(5))
    print("[gpu-case] logprob gradient against differences", flush=True)

    def value(step):
        got = run_forward(logits + step * d, targets, 0, tau, "f32")
        return float((got["logp"].double() * dlogp.double() + got["entropy"].double() * dentropy.double()).sum()), got

    measured = (value(h)[0] - value(-h)[0]) / (2 * h)
    got = value(0.0)[1]
    out = torch.empty(tokens, vocab, device="cuda")
    bns.bns_logprob_backward(bns.make_logprob(tokens, vocab, "f32", temperature=tau), logits.cuda(), targets.cuda(), got["stats"].cuda(), got["entropy"].cuda(), dlogp.cuda(),
                             dentropy.cuda(), out)
    slope = float((out.double().cpu() * d.double()).sum())
    assert abs(slope - measured) < 2e-3 * float(out.double().cpu().norm() * d.double().norm()) / vocab ** 0.5


@pytest.mark.parametrize("tokens", [1, 300])
def test_what_is_not_asked_for(tokens):
    """Entropy, stats, targets left out: the rest has the same bits."""
    logits, targets, _, _ = make(tokens, 50257, "bf16", seed=6)
    print(f"[gpu-case] logprob without {tokens}", flush=True)
    spec, x = bns.make_logprob(tokens, 50257, "bf16", top=3), logits.cuda()
    space = torch.empty(bns.bns_logprob_workspace_bytes(spec), dtype=torch.uint8, device="cuda")
    want = run_forward(logits, targets, 3, 1.0, "bf16")
    logp, ids, top = torch.empty(tokens, device="cuda"), torch.empty(tokens, 3, dtype=torch.int64, device="cuda"), torch.empty(tokens, 3, device="cuda")
    bns.bns_logprob_forward(spec, x, targets.cuda(), logp, None, None, ids, top, space)
    assert torch.equal(logp.cpu(), want["logp"]) and torch.equal(ids.cpu(), want["top_ids"]) and torch.equal(top.cpu(), want["top_logp"])
    bns.bns_logprob_forward(spec, x, None, None, None, None, ids.zero_(), top.zero_(), space)
    assert torch.equal(ids.cpu(), want["top_ids"]) and torch.equal(top.cpu(), want["top_logp"])


def test_captured_and_replayed_beside_other_streams():
    """Forward and backward in a graph, replayed on new logits with eager work between, and on a stream of their own with another workspace."""
    tokens, vocab, top = 5, 40001, 9
    print("[gpu-case] logprob captured", flush=True)
    logits, targets, dlogp, dentropy = make(tokens, vocab, "bf16", seed=7)
    spec = bns.make_logprob(tokens, vocab, "bf16", top=top)

    def buffers():
        return dict(logp=torch.empty(tokens, device="cuda"), entropy=torch.empty(tokens, device="cuda"), stats=torch.empty(tokens, 2, device="cuda"),
                    top_ids=torch.empty(tokens, top, dtype=torch.int64, device="cuda"), top_logp=torch.empty(tokens, top, device="cuda"),
                    space=torch.empty(bns.bns_logprob_workspace_bytes(spec), dtype=torch.uint8, device="cuda"), out=torch.empty(tokens, vocab, dtype=torch.bfloat16, device="cuda"))

    x, t, g, h = logits.cuda(), targets.cuda(), dlogp.cuda(), dentropy.cuda()

    def both(b):
        bns.bns_logprob_forward(spec, x, t, b["logp"], b["entropy"], b["stats"], b["top_ids"], b["top_logp"], b["space"])
        bns.bns_logprob_backward(spec, x, t, b["stats"], b["entropy"], g, h, b["out"])

    captured, eager = buffers(), buffers()
    both(captured)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(captured)
    side = torch.cuda.Stream()
    for turn in range(4):
        x.copy_(make(tokens, vocab, "bf16", seed=20 + turn)[0])
        captured["space"].fill_(turn)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            both(eager)
        graph.replay()
        torch.cuda.synchronize()
        for n in captured:
            if n != "space":
                assert torch.equal(captured[n], eager[n]), n
