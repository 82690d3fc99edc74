"""Softmax cross entropy from hidden states, without the logits, on the GPU against its definition in 64 bits (lm_reference).

Tolerances.  A logit is a sum of `width` products (six times as many in 32 bits) in fp32: off by at most n 2^-24 of the sum of their magnitudes, A, plus 2^-22 A for
the parts of an fp32 product that are dropped and the splits' own rounding.  lse and a token's loss are off by as much, plus a few units of
2^-24 of (1 + |lse|) for the exponentials and the logarithm; a probability by twice that, relative.  g is rounded to the operands' type (2^-8;
in 32 bits three parts hold it), and so is each gradient at the end; between, a sum of n terms in fp32 again."""
import pytest
import torch

import lm_reference as ref
from lm_reference import HALF_ULP, TYPES, Rows, vector, written
from paper_1810_10962_amd import bns

pytestmark = pytest.mark.gpu


# Kernels of the forward pass's logits, the backward pass's and the gradients' products: see "head_logits" and the options behind it.
PATHS = {"few": (1, 1, 1), "few_direct": (1, 1, 2), "direct64": (2, 2, 2), "direct64_few": (2, 2, 1), "direct128": (3, 3, 3), "laid_out256": (4, 4, 4), "laid_out128": (5, 5, 5),
         "mixed": (5, 1, 4), "mixed2": (4, 3, 5), "divided64": (2, 2, 2, 1), "halved64": (2, 2, 2, 3), "auto": (0, 0, 0)}
OPTIONS = ("head_logits", "head_logits_backward", "head_gradients", "head_groups")


@pytest.fixture(params=PATHS)
def path(request):
    for name, value in zip(OPTIONS, PATHS[request.param]):
        bns.bns_set_option(name, value)
    yield request.param
    for name in OPTIONS:
        bns.bns_set_option(name, 0)


def make(tokens, width, vocab, dtype, seed=0, ignored=0.2):
    g = torch.Generator().manual_seed(seed * 7919 + tokens * 31 + width * 7 + vocab)
    rnd = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    weight = (rnd(vocab, width) * 2 / width ** 0.5).to(TYPES[dtype])
    hidden = rnd(tokens, width).to(TYPES[dtype])
    targets = torch.randint(0, vocab, (tokens,), generator=g)
    skip = torch.rand(tokens, generator=g) < ignored
    targets = torch.where(skip, torch.tensor([-100, -1, vocab, 2 ** 40])[torch.randint(0, 4, (tokens,), generator=g)], targets)
    return hidden, weight, targets, 0.2 + torch.rand(tokens, generator=g)


def assert_within(got, want, bound, what):
    off = (got.double().cpu() - want).abs() - bound
    assert bool((off <= 0).all()), f"{what}: worst excess {off.max().item():.3e} over {bound.max().item():.3e}"


def check_forward(loss, lse, hidden, weight, targets, dtype):
    h, w = hidden.double(), weight.double()
    want_loss, want_lse, *_ = ref.head(h, w, targets, torch.ones(len(h), dtype=torch.float64))
    terms = h.shape[1] * (6 if dtype == "f32" else 1)
    z_off = (terms + 4) * 2.0 ** -24 * (h.abs() @ w.abs().T).amax(1)
    bound = 2 * z_off + 16 * 2.0 ** -24 * (1 + want_lse.abs()) + len(w) ** 0.5 * 2.0 ** -24
    assert_within(lse, want_lse, bound, "lse")
    assert_within(loss, want_loss, bound, "loss")
    return z_off, bound


def check_backward(dh, dw, hidden, weight, targets, dloss, dtype):
    h, w, d = hidden.double(), weight.double(), dloss.double()
    _, lse, p, g, want_dh, want_dw = ref.head(h, w, targets, d)
    kept = (targets >= 0) & (targets < len(w))
    terms = h.shape[1] * (6 if dtype == "f32" else 1)
    z_off = (terms + 4) * 2.0 ** -24 * (h.abs() @ w.abs().T).amax(1, keepdim=True)
    p_off = p * (3 * z_off + 64 * 2.0 ** -24 * (1 + lse.abs()[:, None] + (h @ w.T).abs()))
    g_off = torch.where(kept[:, None], d[:, None] * p_off, torch.zeros_like(p)) + g.abs() * (HALF_ULP[dtype] if dtype == "bf16" else 2.0 ** -23)
    more = 6 if dtype == "f32" else 1
    kh = torch.where(kept[:, None], h, torch.zeros_like(h))
    bound_h = g_off @ w.abs() + (more * len(w) ** 0.5 * 4 + 8) * 2.0 ** -24 * (g.abs() @ w.abs())
    bound_w = g_off.T @ kh.abs() + (more * len(h) ** 0.5 * 4 + 8) * 2.0 ** -24 * (g.abs().T @ kh.abs())
    assert_within(dh, want_dh, bound_h * 1.01 + HALF_ULP[dtype] * want_dh.abs() * 1.01 + 1e-36, "dhidden")
    assert_within(dw, want_dw, bound_w * 1.01 + HALF_ULP[dtype] * want_dw.abs() * 1.01 + 1e-36, "dweight")


def run(hidden, weight, targets, dloss, dtype, pad=0, piece=0):
    tokens, width, vocab = *hidden.shape, len(weight)
    head = bns.make_head(tokens, width, vocab, dtype, piece=piece, hidden_stride=width + pad if pad else 0, weight_stride=width + 2 * pad if pad else 0)
    ws = Rows(torch.zeros(1, bns.bns_head_workspace_bytes(head) // 4), dtype=torch.float32, written=True)
    ws.t.fill_(float("nan"))                                # nothing in the workspace is taken for granted
    h, w, t = Rows(hidden, width + pad if pad else 0), Rows(weight, width + 2 * pad if pad else 0), targets.cuda()
    loss, lse = written(tokens), written(tokens)
    bns.bns_head_forward(head, h, w, t, loss, lse, ws)
    dh, dw = Rows(torch.zeros(tokens, width), dtype=TYPES[dtype], written=True), Rows(torch.zeros(vocab, width), dtype=TYPES[dtype], written=True)
    kept = lse.t[0].clone()
    ws.t.fill_(float("nan"))
    bns.bns_head_backward(head, h, w, t, kept, vector(dloss), dh, dw, ws)
    ws.check()
    return loss.check()[0], lse.check()[0], dh.check(), dw.check()


SHAPES = [(1, 1, 1), (1, 64, 2), (3, 8, 257), (5, 100, 1000), (16, 128, 300), (64, 192, 513), (65, 64, 256), (130, 200, 255), (257, 320, 1030), (300, 77, 700), (40, 1000, 5003),
          (511, 512, 2049), (30, 72, 1500)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens,width,vocab", SHAPES)
def test_loss_and_gradients(tokens, width, vocab, dtype, path):
    for pad, piece in [(0, 0), (3, 256), (8, 512)]:
        print(f"[gpu-case] head {tokens}x{width}x{vocab} {dtype} {path} pad={pad} piece={piece}", flush=True)
        hidden, weight, targets, dloss = make(tokens, width, vocab, dtype)
        loss, lse, dh, dw = run(hidden, weight, targets, dloss, dtype, pad, piece)
        check_forward(loss, lse, hidden, weight, targets, dtype)
        check_backward(dh, dw, hidden, weight, targets, dloss, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens", [7, 100])
def test_tokens_that_are_left_out_may_hold_anything(tokens, dtype, path):
    hidden, weight, targets, dloss = make(tokens, 128, 600, dtype, seed=1, ignored=0.4)
    out = (targets < 0) | (targets >= 600)
    assert bool(out.any()) and not bool(out.all())
    hidden[out] = float("nan")
    hidden[out.nonzero()[0], 3:] = float("inf")
    dloss[out] = float("nan")
    print(f"[gpu-case] head masked NaN {tokens} {dtype}", flush=True)
    loss, lse, dh, dw = run(hidden, weight, targets, dloss, dtype)
    clean, cleand = torch.where(out[:, None], torch.zeros((), dtype=hidden.dtype), hidden), torch.where(out, torch.zeros(()), dloss)
    assert bool((loss.cpu()[out] == 0).all()) and bool((dh.cpu()[out] == 0).all())
    check_forward(loss.cpu()[~out], lse.cpu()[~out], clean[~out], weight, targets[~out], dtype)
    check_backward(dh, dw, clean, weight, targets, cleand, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_no_token_is_kept_or_there(dtype, path):
    print(f"[gpu-case] head without tokens {dtype}", flush=True)
    hidden, weight, targets, dloss = make(9, 64, 300, dtype, ignored=1.1)
    loss, lse, dh, dw = run(hidden, weight, targets, dloss, dtype)
    assert bool((loss == 0).all()) and bool((dh == 0).all()) and bool((dw == 0).all()) and bool(torch.isfinite(lse).all())
    head = bns.make_head(0, 64, 300, dtype)
    none = torch.empty(0, 64, dtype=TYPES[dtype], device="cuda")
    ws = torch.empty(bns.bns_head_workspace_bytes(head), dtype=torch.uint8, device="cuda")
    dw = Rows(torch.zeros(300, 64), dtype=TYPES[dtype], written=True)
    e = torch.empty(0, device="cuda")
    bns.bns_head_forward(head, none, weight.cuda(), torch.empty(0, dtype=torch.int64, device="cuda"), e, e, ws)
    bns.bns_head_backward(head, none, weight.cuda(), torch.empty(0, dtype=torch.int64, device="cuda"), e, e, none, dw, ws)
    assert bool((dw.check() == 0).all())


def test_large_logits_and_a_sure_model(path):
    """Logits of a few hundred, all probability on the target: a loss of zero, not of NaN, and gradients that vanish."""
    tokens, width, vocab = 64, 64, 700
    weight = torch.zeros(vocab, width)
    weight[torch.arange(vocab), torch.arange(vocab) % width] = 20.0
    weight[width:] *= -1
    targets = torch.arange(tokens) % width
    hidden = 20.0 * torch.eye(width)[targets]
    dloss = torch.ones(tokens)
    for dtype in ("f32", "bf16"):
        print(f"[gpu-case] head sure {dtype}", flush=True)
        loss, lse, dh, dw = run(hidden.to(TYPES[dtype]), weight.to(TYPES[dtype]), targets, dloss, dtype)
        assert bool((loss.abs() < 1e-3).all()) and bool(((lse - 400).abs() < 1e-3).all())
        assert float(dh.float().abs().max()) < 1e-3 and float(dw.float().abs().max()) < 1e-3


def test_same_bits_from_run_to_run_and_in_a_graph(path):
    hidden, weight, targets, dloss = make(200, 256, 3000, "bf16", seed=5)
    head = bns.make_head(200, 256, 3000, "bf16", piece=1024)
    h, w, t, d = hidden.cuda(), weight.cuda(), targets.cuda(), dloss.cuda()
    ws = torch.empty(bns.bns_head_workspace_bytes(head), dtype=torch.uint8, device="cuda")
    loss, lse, dh, dw = torch.empty(200, device="cuda"), torch.empty(200, device="cuda"), torch.empty_like(h), torch.empty_like(w)

    def step():
        bns.bns_head_forward(head, h, w, t, loss, lse, ws)
        bns.bns_head_backward(head, h, w, t, lse, d, dh, dw, ws)

    print("[gpu-case] head in a graph", flush=True)
    step()
    want = [x.clone() for x in (loss, lse, dh, dw)]
    step()
    assert all(torch.equal(a, b) for a, b in zip(want, (loss, lse, dh, dw)))
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step()
    for i in range(3):
        for x in (loss, lse, dh, dw):
            x.fill_(float(i))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (loss, lse, dh, dw))), f"replay {i}"


def test_gradient_against_differences():
    """The loss's own change along a direction, central difference with step 2^-6: third order about h^2 of the gradient's size, 3e-4; rounding 1e-6 / h."""
    tokens, width, vocab, h = 50, 96, 400, 2.0 ** -6
    hidden, weight, targets, dloss = make(tokens, width, vocab, "f32", seed=6)
    g = torch.Generator().manual_seed(9)
    dh, dw = torch.randn(tokens, width, generator=g), torch.randn(vocab, width, generator=g) / width ** 0.5
    print("[gpu-case] head gradient against differences", flush=True)
    _, _, gh, gw = run(hidden, weight, targets, dloss, "f32")

    def value(step):
        loss, *_ = run(hidden + step * dh, weight + step * dw, targets, dloss, "f32")
        return float((loss.double().cpu() * dloss.double()).sum())

    slope = float((gh.double().cpu() * dh.double()).sum() + (gw.double().cpu() * dw.double()).sum())
    measured = (value(h) - value(-h)) / (2 * h)
    size = float(gh.double().cpu().norm() * dh.double().norm() / width ** 0.5 + gw.double().cpu().norm() * dw.double().norm() / vocab ** 0.5)
    assert abs(slope - measured) < 5e-3 * size


@pytest.mark.parametrize("tokens,width,vocab,dtype,stride", [(5, 1024, 115000, "bf16", 1024), (20, 500, 115011, "f32", 512), (3, 1000, 120000, "bf16", 1001), (17, 1001, 60001, "f32", 1001)])
def test_a_matrix_beyond_the_cache(tokens, width, vocab, dtype, stride):
    """More than 224 MB of weights (rows of whole cache lines or not), read once."""
    hidden, weight, targets, _ = make(tokens, width, vocab, dtype, seed=6)
    print(f"[gpu-case] head beyond the cache {tokens}x{width}x{vocab} {dtype} stride={stride}", flush=True)
    spec = bns.make_head(tokens, width, vocab, dtype, weight_stride=stride)
    ws = torch.full((bns.bns_head_workspace_bytes(spec),), 255, dtype=torch.uint8, device="cuda")
    w = Rows(weight, stride)
    loss, lse = written(tokens), written(tokens)
    bns.bns_head_forward(spec, hidden.cuda(), w, targets.cuda(), loss, lse, ws)
    check_forward(loss.check()[0], lse.check()[0], hidden, weight, targets, dtype)
