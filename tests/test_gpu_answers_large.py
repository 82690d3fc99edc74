"""A step on a model's own answers beyond 2^31 elements: indices have to be as wide."""
import math

import pytest
import torch

import answers_reference as ref
from paper_1810_10962_amd import bns

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def fill(t, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    flat = t.reshape(-1)
    for at in range(0, flat.numel(), 1 << 28):
        flat[at:at + (1 << 28)].normal_(generator=g)
    return t


def test_many_tokens_of_queries():
    """2^31 elements and some, in place, forward and backward: what calls on some of the tokens leave, bit by bit (heads are independent)."""
    tokens, heads, width, chunk = (1 << 31) // (16 * 128) + 1000, 16, 128, 500
    print(f"[gpu-case] qk of {tokens} tokens", flush=True)
    q = fill(torch.empty(tokens, heads, width, dtype=torch.bfloat16, device="cuda"), 1)
    weight, turns = 1 + 0.1 * torch.randn(width, device="cuda"), 10000.0 ** (-torch.arange(64, dtype=torch.float64, device="cuda") / 64)
    positions = torch.arange(tokens, device="cuda")
    places = [0, tokens // 2, tokens - chunk]
    before = [q[at:at + chunk].clone() for at in places]
    few, many = (bns.make_qk(n, heads, 0, width, rotated=width) for n in (chunk, tokens))
    workspace, dw = torch.empty(bns.bns_qk_workspace_bytes(many), dtype=torch.uint8, device="cuda"), torch.empty(width, device="cuda")
    dk = torch.empty(width, device="cuda")
    x = q.clone()
    bns.bns_qk_forward(many, q, None, weight, None, positions, turns, q, None)
    for at, b in zip(places, before):
        out = torch.empty_like(b)
        bns.bns_qk_forward(few, b, None, weight, None, positions[at:at + chunk], turns, out, None)
        assert torch.equal(q[at:at + chunk], out), at
    wanted = []
    for at, b in zip(places, before):
        dx = torch.empty_like(b)
        bns.bns_qk_backward(few, b, None, weight, None, positions[at:at + chunk], turns, q[at:at + chunk], None, dx, None, dk, None, workspace)
        wanted.append(dx)
    bns.bns_qk_backward(many, x, None, weight, None, positions, turns, q, None, q, None, dw, None, workspace)
    for at, want in zip(places, wanted):
        assert torch.equal(q[at:at + chunk], want), at


def test_the_weight_s_gradient_of_many_tokens():
    """2^31 elements and some, the gradient along the result itself, so that no term has another's sign and a part that is missing shows: g = weight x^ and its rounding.
    Terms: x^ 16 u, g (|g_a| + |g_b|) (5 + 3 u and an angle's 2^-51 of 10^6, the reference's); their sum 1025 in turn in a lane, then 32, 16 and 32 in turn."""
    tokens, heads, width = (1 << 31) // (16 * 128) + 1000, 16, 128
    print(f"[gpu-case] qk weight's gradient of {tokens} tokens", flush=True)
    x = fill(torch.empty(tokens, heads, width, dtype=torch.bfloat16, device="cuda"), 4)
    weight, turns = 1 + 0.1 * torch.randn(width, device="cuda"), 10000.0 ** (-torch.arange(64, dtype=torch.float64, device="cuda") / 64)
    positions, spec = torch.arange(tokens, device="cuda"), bns.make_qk(tokens, heads, 0, width, rotated=width)
    dy, dw = torch.empty_like(x), torch.empty(width, device="cuda")
    bns.bns_qk_forward(spec, x, None, weight, None, positions, turns, dy, None)
    want, off = (torch.zeros(width, dtype=torch.float64, device="cuda") for _ in range(2))
    for at in range(0, tokens, 1 << 15):
        part = slice(at, at + (1 << 15))
        _, dw_part, g, r = ref.qk_backward(x[part].double(), weight.double(), positions[part], turns, dy[part].double(), width, False, 1e-6)
        want += dw_part
        xh = (x[part].double() * r).abs()
        off += (xh * ref.beside(g, width, False)).sum((0, 1)) * (8 * U + 2.0 ** -51 * 1e6) + (xh * g.abs()).sum((0, 1)) * (17 + 1025 + 80) * U
    bns.bns_qk_backward(spec, x, None, weight, None, positions, turns, dy, None, dy, None, dw, None,
                        torch.empty(bns.bns_qk_workspace_bytes(spec), dtype=torch.uint8, device="cuda"))
    assert float(((dw.double() - want).abs() - off).max()) <= 0 and float((off / want).max()) < 1 / 2048       # (a block's part is 1 / 512)


@pytest.mark.parametrize("kind", ["token", "head"])
def test_far_apart(kind):
    """Strides that pass 2^31 elements between neighbours, with bytes beyond 2^33 (a long head-major cache)."""
    tokens, heads, width = 3, 3, 64
    step = (1 << 31) + 24
    print(f"[gpu-case] qk strides {kind}", flush=True)
    whole = torch.empty(2 * step + 3 * width, dtype=torch.bfloat16, device="cuda")
    strides = (step, width) if kind == "token" else (width, step)
    k = whole.as_strided((tokens, heads, width), (*strides, 1))
    x = torch.randn(tokens, heads, width).bfloat16()
    k.copy_(x)
    weight, turns = torch.rand(width) + 0.5, 100.0 ** (-torch.arange(32, dtype=torch.float64) / 32)
    positions = torch.tensor([5, 1000, 77])
    spec = bns.make_qk(tokens, 0, heads, width, k=strides, k_out=strides)
    bns.bns_qk_forward(spec, None, k, None, weight.cuda(), positions.cuda(), turns.cuda(), None, k)
    want, v = ref.qk_forward(x.double(), weight.double(), positions, turns, width, False, 1e-6)
    off = ref.beside(v, width, False) * 30 * U + 2.0 ** -8 * want.abs()         # (test_gpu_qk: 17 + 5 + 3 u and an angle's 2^-51 of 1000)
    assert float(((k.double().cpu() - want).abs() - off).max()) <= 0


def test_many_logits():
    """2^31 logits and some: rows at both ends and in the middle against their definition, backward in place."""
    vocab, chunk = 131072, 4
    tokens = (1 << 31) // vocab + 40
    print(f"[gpu-case] logprob {tokens} x {vocab}", flush=True)
    logits = fill(torch.empty(tokens, vocab, dtype=torch.bfloat16, device="cuda"), 2)
    targets = torch.randint(0, vocab, (tokens,), device="cuda")
    logp, entropy, stats = torch.empty(tokens, device="cuda"), torch.empty(tokens, device="cuda"), torch.empty(tokens, 2, device="cuda")
    ids, top_logp = torch.empty(tokens, 5, dtype=torch.int64, device="cuda"), torch.empty(tokens, 5, device="cuda")
    spec = bns.make_logprob(tokens, vocab, top=5)
    bns.bns_logprob_forward(spec, logits, targets, logp, entropy, stats, ids, top_logp, torch.empty(bns.bns_logprob_workspace_bytes(spec), dtype=torch.uint8, device="cuda"))
    dlogp, dentropy = torch.randn(tokens, device="cuda"), torch.randn(tokens, device="cuda")
    rows = [slice(at, at + chunk) for at in (0, tokens // 2, tokens - chunk)]
    kept = [logits[r].double() for r in rows]
    bns.bns_logprob_backward(spec, logits, targets, stats, entropy, dlogp, dentropy, logits)
    for r, z in zip(rows, kept):
        all_logp = torch.log_softmax(z, 1)
        p = all_logp.exp()
        given, h = all_logp.gather(1, targets[r, None])[:, 0], -(p * all_logp).sum(1)
        # sums of 131072 positive terms, 512 a thread in turn, then ten steps: 525 u relative, that is absolute for their logarithm; a few u of the values
        assert float((logp[r] - given).abs().max()) <= 600 * U * (1 + float(given.abs().max()))
        assert float((entropy[r] - h).abs().max()) <= 1200 * U * (1 + float(h.abs().max()))
        assert torch.equal(ids[r], torch.sort(z, dim=1, descending=True, stable=True).indices[:, :5])
        assert float((top_logp[r] - all_logp.gather(1, ids[r])).abs().max()) <= 600 * U * 20
        hit = torch.zeros_like(p).scatter_(1, targets[r, None], 1.0)
        want = dlogp[r, None] * (hit - p) - dentropy[r, None] * p * (all_logp + h[:, None])
        off = 2.0 ** -8 * want.abs() + 2000 * U * p * (dlogp[r, None].abs() + dentropy[r, None].abs() * 20) + 4 * U * hit * dlogp[r, None].abs() + 1e-37
        assert float(((logits[r].double() - want).abs() - off).max()) <= 0


def test_a_large_gradient():
    """One gradient of 2^31 elements and some beside a small one: fp64 sums, so that norm and factor have the few roundings of their last steps."""
    n = (1 << 31) + 12345
    print(f"[gpu-case] clip {n}", flush=True)
    grads = [fill(torch.empty(n, dtype=torch.bfloat16, device="cuda"), 3), torch.randn(1001, device="cuda")]
    squares = sum(float(part.double().pow(2).sum()) for g in grads for part in g.split(1 << 26))
    parts = [slice(0, 5000), slice(n // 2, n // 2 + 5000), slice(n - 5000, n)]
    before = [grads[0][p].double() for p in parts] + [grads[1].double()]
    gradients = bns.make_gradients(grads, grads)
    norm = torch.empty(1, device="cuda")
    bns.bns_grads_clip(gradients, 10.0, norm, torch.empty(bns.bns_grads_workspace_bytes(gradients), dtype=torch.uint8, device="cuda"))
    assert abs(float(norm) - math.sqrt(squares)) <= 2 * U * math.sqrt(squares)
    factor = 10.0 / (math.sqrt(squares) + 1e-6)
    for got, b, half in zip([grads[0][p] for p in parts] + [grads[1]], before, [2.0 ** -8] * 3 + [U]):
        assert float(((got.double() - b * factor).abs() - (half + 5 * U) * (b * factor).abs()).max()) <= 1e-40
