"""What the calls of a step on a model's own answers refuse, before anything is enqueued: made-up addresses that are never dereferenced suffice, no GPU is needed."""
import ctypes as C

import pytest
import torch

from paper_1810_10962_amd import bns

Q, K, QO, KO, DQ, DK, W, P, F, V, WS = (i << 28 for i in range(1, 12))
NULL = 0
ROW = 8 * 64                # bytes of a token: 4 heads of 64 bf16


def qk_forward(q=Q, k=K, qw=W, kw=W + 4096, p=P, f=F, qo=QO, ko=KO, tokens=8, q_heads=4, k_heads=2, width=64, **kw_):
    spec = bns.make_qk(tokens, q_heads, k_heads, width, **kw_)
    return bns.load().bns_qk_forward(C.byref(spec), q, k, qw, kw, p, f, qo, ko, None)


def qk_backward(q=Q, k=K, qw=W, kw=W + 4096, p=P, f=F, go=QO, gko=KO, dq=DQ, dk=DK, dqw=V, dkw=V + 4096, ws=WS, short=0, tokens=8, q_heads=4, k_heads=2, width=64, **kw_):
    spec = bns.make_qk(tokens, q_heads, k_heads, width, **kw_)
    n = max(0, bns.bns_qk_workspace_bytes(spec) - short)
    return bns.load().bns_qk_backward(C.byref(spec), q, k, qw, kw, p, f, go, gko, dq, dk, dqw, dkw, ws, n, None)


BOTH = [dict(p=NULL), dict(f=NULL), dict(qw=W + 2), dict(kw=W + 1), dict(kw=W + 1, weight_dtype="bf16"), dict(p=P + 4), dict(f=F + 4), dict(q=Q + 1), dict(k=K + 1), dict(tokens=-1), dict(q_heads=-1), dict(k_heads=-3),
        dict(width=0), dict(width=-64), dict(rotated=-2), dict(rotated=3), dict(rotated=66), dict(interleaved=2), dict(dtype=2), dict(weight_dtype=-1), dict(eps=-1.0),
        dict(eps=float("nan")), dict(eps=float("inf")), dict(q=Q, dtype="f32", k=K + 2)]
STRIDES = [(-1, 0), (0, -1), (255, 64), (256, 63), (64, 300), (1, 64), (64, 64), (63, 8 * 64), (64, 7 * 64)]


@pytest.mark.parametrize("call", [qk_forward, qk_backward])
@pytest.mark.parametrize("kw", BOTH + [{n: s} for n in ("q", "q_out", "dq") for s in STRIDES])
def test_qk_refuses(call, kw):
    kw = dict(kw)
    strides = {n: kw.pop(n) for n in ("q", "q_out", "dq") if isinstance(kw.get(n), tuple)}
    if strides:         # (q is a pointer above and a stride of the description below)
        name, value = next(iter(strides.items()))
        spec = bns.make_qk(8, 4, 2, 64, **{name: value})
        lib = bns.load()
        if call is qk_forward:
            assert lib.bns_qk_forward(C.byref(spec), Q, K, W, W, P, F, QO, KO, None) == bns.BNS_EINVAL
        else:
            assert lib.bns_qk_backward(C.byref(spec), Q, K, W, W, P, F, QO, KO, DQ, DK, V, V, WS, 1 << 30, None) == bns.BNS_EINVAL
        assert bns.bns_qk_workspace_bytes(spec) == 0
        return
    assert call(**kw) == bns.BNS_EINVAL


@pytest.mark.parametrize("kw", [dict(q=NULL), dict(k=NULL), dict(qo=NULL), dict(ko=NULL), dict(qo=QO + 1), dict(ko=KO + 1), dict(qo=K), dict(ko=Q), dict(ko=QO), dict(qo=KO + 64),
                                dict(qo=Q + 2), dict(qo=Q + 8 * ROW - 2), dict(ko=K + 256)])
def test_qk_forward_refuses(kw):
    assert qk_forward(**kw) == bns.BNS_EINVAL


def test_in_place_with_other_strides_is_refused():
    lib = bns.load()
    spec = bns.make_qk(8, 4, 2, 64, q=(512, 64), q_out=(256, 64))
    assert lib.bns_qk_forward(C.byref(spec), Q, K, W, W, P, F, Q, KO, None) == bns.BNS_EINVAL
    spec = bns.make_qk(8, 4, 2, 64, q_out=(64, 8 * 64))         # head-major on token-major
    assert lib.bns_qk_forward(C.byref(spec), Q, K, W, W, P, F, Q, KO, None) == bns.BNS_EINVAL


@pytest.mark.parametrize("kw", [dict(q=NULL), dict(k=NULL), dict(go=NULL), dict(gko=NULL), dict(dq=NULL), dict(dk=NULL), dict(dqw=NULL), dict(dkw=NULL), dict(ws=NULL), dict(qw=NULL),
                                dict(kw=NULL), dict(ws=WS + 8), dict(dqw=V + 2), dict(go=QO + 1), dict(dq=Q), dict(dk=K), dict(dq=K), dict(dk=QO), dict(dk=DQ + 64), dict(dq=QO + 2)])
def test_qk_backward_refuses(kw):
    assert qk_backward(**kw) == bns.BNS_EINVAL


def test_weight_gradients_that_overlap_are_refused():
    for off in (0, 4, 63 * 4):
        assert qk_backward(dqw=V, dkw=V + off) == qk_backward(dqw=V + off, dkw=V) == bns.BNS_EINVAL


def test_qk_limits():
    for kw in (dict(tokens=2 ** 31), dict(q_heads=2 ** 20), dict(k_heads=2 ** 20), dict(width=513, rotated=0)):
        assert qk_forward(**kw) == qk_backward(**kw) == bns.BNS_EUNSUPPORTED
    for strides in (dict(q=(2 ** 48, 64)), dict(k=(64, 2 ** 60)), dict(q_out=(2 ** 47, 64)), dict(dk=(2 ** 62, 2 ** 61))):
        assert bns.bns_qk_workspace_bytes(bns.make_qk(8, 4, 2, 64, **strides)) == 0
        spec = bns.make_qk(8, 4, 2, 64, **strides)
        assert bns.load().bns_qk_forward(C.byref(spec), Q, K, W, W, P, F, QO, KO, None) == bns.BNS_EUNSUPPORTED
    assert qk_backward(short=1) == bns.BNS_EWORKSPACE
    assert bns.load().bns_qk_forward(None, Q, K, W, W, P, F, QO, KO, None) == bns.BNS_EINVAL and bns.load().bns_qk_workspace_bytes(None) == 0


def logprob(call, x=Q, t=P, logp=V, h=V + 4096, st=V + 8192, ids=NULL, top_logp=NULL, ws=WS, short=0, g=V + 12288, gh=V + 16384, dx=DQ, tokens=8, vocab=100, **kw):
    spec = bns.make_logprob(tokens, vocab, **kw)
    if call == "forward":
        return bns.load().bns_logprob_forward(C.byref(spec), x, t, logp, h, st, ids, top_logp, ws, max(0, bns.bns_logprob_workspace_bytes(spec) - short), None)
    return bns.load().bns_logprob_backward(C.byref(spec), x, t, st, h, g, gh, dx, None)


@pytest.mark.parametrize("call", ["forward", "backward"])
@pytest.mark.parametrize("kw", [dict(x=NULL), dict(t=NULL), dict(x=Q + 1), dict(x=Q + 2, dtype="f32"), dict(t=P + 4), dict(h=V + 2), dict(st=V + 1), dict(tokens=-1), dict(vocab=0), dict(vocab=-1), dict(top=-1),
                                dict(top=101), dict(dtype=2), dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=float("nan")), dict(temperature=float("inf")),
                                dict(logits_stride=99), dict(dlogits_stride=-1)])
def test_logprob_refuses(call, kw):
    assert logprob(call, **kw) == bns.BNS_EINVAL


@pytest.mark.parametrize("kw", [dict(logp=NULL), dict(logp=V + 2), dict(ws=NULL), dict(ws=WS + 8), dict(ids=K), dict(top_logp=K), dict(top=4), dict(top=4, ids=K), dict(top=4, top_logp=K),
                                dict(top=4, ids=K + 4, top_logp=QO), dict(top=4, ids=K, top_logp=QO + 2)])
def test_logprob_forward_refuses(kw):
    assert logprob("forward", **kw) == bns.BNS_EINVAL


@pytest.mark.parametrize("kw", [dict(st=NULL), dict(h=NULL), dict(g=NULL), dict(g=V + 2), dict(gh=V + 1), dict(dx=NULL), dict(dx=DQ + 1), dict(dx=Q + 16), dict(dx=Q, dlogits_stride=200)])
def test_logprob_backward_refuses(kw):
    assert logprob("backward", **kw) == bns.BNS_EINVAL


def test_logprob_limits():
    for kw in (dict(tokens=2 ** 31), dict(vocab=2 ** 30), dict(top=129, vocab=1000), dict(logits_stride=2 ** 31), dict(dlogits_stride=2 ** 40), dict(temperature=1e-7), dict(temperature=1e7)):
        assert logprob("forward", **kw) == logprob("backward", **kw) == bns.BNS_EUNSUPPORTED
        assert bns.bns_logprob_workspace_bytes(bns.make_logprob(**{**dict(tokens=8, vocab=100), **kw})) == 0
    for kw in (dict(), dict(tokens=1, vocab=131072), dict(tokens=1, vocab=131072, top=128, ids=K, top_logp=QO)):
        assert logprob("forward", short=1, **kw) == bns.BNS_EWORKSPACE
    lib = bns.load()
    assert lib.bns_logprob_forward(None, Q, P, V, V, V, None, None, WS, 1 << 20, None) == bns.BNS_EINVAL and lib.bns_logprob_workspace_bytes(None) == 0
    assert lib.bns_logprob_backward(None, Q, P, V, V, V, V, DQ, None) == bns.BNS_EINVAL


def gradients(*entries):
    return (bns.bns_gradient * max(1, len(entries)))(*(bns.bns_gradient(*e) for e in entries)), len(entries)


def grads(call, list_, count=None, squares=V, norm=V + 4096, ws=WS, short=0, max_norm=1.0):
    array, n = gradients(*list_)
    n = n if count is None else count
    lib = bns.load()
    size = max(0, lib.bns_grads_workspace_bytes(n) - short)
    if call == "norm":
        return lib.bns_grads_norm(array, n, squares, norm, ws, size, None)
    if call == "scale":
        return lib.bns_grads_scale(array, n, squares, max_norm, norm, ws, size, None)
    return lib.bns_grads_clip(array, n, max_norm, norm, ws, size, None)


GOOD = (Q, QO, 1000, 0, 0)


@pytest.mark.parametrize("call", ["norm", "scale", "clip"])
@pytest.mark.parametrize("entry", [(NULL, QO, 5, 0, 0), (Q, QO, -1, 0, 0), (Q, QO, 5, 2, 0), (Q, QO, 5, -1, 0), (Q, QO, 5, 0, 1), (Q + 2, QO, 5, 0, 0), (Q + 1, QO, 5, 1, 0)])
def test_gradients_are_checked(call, entry):
    assert grads(call, [entry]) == grads(call, [(K, KO, 10, 1, 0), entry]) == bns.BNS_EINVAL


@pytest.mark.parametrize("call", ["scale", "clip"])
@pytest.mark.parametrize("list_", [[(Q, NULL, 5, 0, 0)], [(Q, QO + 2, 5, 0, 0)], [(Q, QO + 1, 5, 1, 0)], [(Q, Q + 4, 5, 0, 0)], [(Q, Q - 4, 5, 0, 0)], [(Q, QO, 5, 0, 0), (K, QO, 5, 0, 0)],
                                   [(Q, QO, 5, 0, 0), (K, QO + 16, 5, 0, 0)], [(Q, K, 5, 0, 0), (K, KO, 5, 0, 0)], [(Q, KO, 5, 0, 0), (K, Q + 8, 5, 1, 0)], [(Q, Q, 5, 0, 0)] * 2,
                                   [(Q, Q, 100, 0, 0), (Q + 396, Q + 396, 5, 1, 0)], [(Q + 4 * i, QO + 3 * 4 * i, 1, 0, 0) for i in range(1000)] + [(K, QO + 12 * 500, 1, 0, 0)]])
def test_results_that_overlap_are_refused(call, list_):
    assert grads(call, list_) == bns.BNS_EINVAL


def test_gradients_at_addresses_that_do_not_fit_a_word_are_refused():
    for call in ("norm", "scale", "clip"):
        for at in (2 ** 48, 2 ** 48 - 16, 2 ** 63, 2 ** 64 - 64):
            assert grads(call, [(at, at, 5, 0, 0)]) == bns.BNS_EUNSUPPORTED
    for call in ("scale", "clip"):
        assert grads(call, [(Q, 2 ** 48, 5, 0, 0)]) == bns.BNS_EUNSUPPORTED


def test_arguments_of_gradients():
    for call in ("norm", "scale", "clip"):
        assert grads(call, [GOOD], ws=NULL) == grads(call, [GOOD], ws=WS + 8) == grads(call, [GOOD], norm=V + 2) == grads(call, [GOOD], count=-1) == bns.BNS_EINVAL
        assert grads(call, [GOOD], short=1) == grads(call, [(Q, QO + 4 * i, 1, 0, 0) for i in range(200)], short=1) == bns.BNS_EWORKSPACE
        assert grads(call, [(Q, QO, 2 ** 40, 0, 0)]) == bns.BNS_EUNSUPPORTED
        assert grads(call, [(Q + (i << 42), Q + (i << 42), 2 ** 40 - 1, 0, 0) for i in range(9)]) == bns.BNS_EUNSUPPORTED
        assert grads(call, [GOOD], count=65537) == bns.BNS_EUNSUPPORTED
    for call in ("norm", "scale"):
        assert grads(call, [GOOD], squares=NULL) == grads(call, [GOOD], squares=V + 4) == bns.BNS_EINVAL
    for call in ("scale", "clip"):
        for max_norm in (-1.0, float("nan"), float("inf")):
            assert grads(call, [GOOD], max_norm=max_norm) == bns.BNS_EINVAL
    assert grads("clip", [GOOD], norm=NULL) == bns.BNS_EINVAL
    assert bns.load().bns_grads_clip(None, 1, 1.0, V, WS, 1 << 20, None) == bns.BNS_EINVAL
    lib = bns.load()
    assert lib.bns_grads_workspace_bytes(-1) == lib.bns_grads_workspace_bytes(65537) == 0 < lib.bns_grads_workspace_bytes(0) < lib.bns_grads_workspace_bytes(65536)


def test_nothing_to_do():
    before = bns.bns_get_option("launch_count")
    assert qk_forward(tokens=0, q=NULL, k=NULL, qo=NULL, ko=NULL, p=NULL) == bns.BNS_OK
    assert qk_forward(q_heads=0, k_heads=0, q=NULL, k=NULL, qo=NULL, ko=NULL, qw=NULL, kw=NULL, p=NULL, f=NULL) == bns.BNS_OK
    assert qk_backward(q_heads=0, k_heads=0, q=NULL, k=NULL, go=NULL, gko=NULL, dq=NULL, dk=NULL, qw=NULL, kw=NULL, dqw=NULL, dkw=NULL) == bns.BNS_OK
    for call in ("forward", "backward"):
        assert logprob(call, tokens=0, x=NULL, t=P, logp=V, dx=NULL) == bns.BNS_OK
    assert bns.bns_get_option("launch_count") == before


def test_the_binding_checks_gradients():
    a, b = torch.zeros(4, 6), torch.zeros(24)
    assert bns.make_gradients([a, b], [b, a]).count == 2 and bns.make_gradients([]).count == 0
    for grads_, outs in (([a.double()], None), ([a.t()], None), ([a], [a.bfloat16()]), ([a], [torch.zeros(5)]), ([a], []), ([a], [torch.zeros(6, 4).t()])):
        with pytest.raises(ValueError):
            bns.make_gradients(grads_, outs)


def test_gradients_with_the_channels_last():
    """Weights of convolutions in the order of N x H x W x C tensors: dense, so that their elements are taken as they lie, where the results have the same order."""
    a = torch.zeros(4, 6, 3, 3).to(memory_format=torch.channels_last)
    b, solid = torch.zeros(2, 4, 3, 3, 3).to(memory_format=torch.channels_last_3d), torch.zeros(4, 6, 3, 3)
    assert bns.make_gradients([a, b, solid]).count == 3
    got = bns.make_gradients([a, b], [torch.empty_like(a), b])
    assert got.array[0].elements == a.numel() and got.array[0].grad == a.data_ptr() and got.array[1].out == b.data_ptr()
    point = torch.zeros(4, 6, 1, 1).to(memory_format=torch.channels_last)          # (in either order)
    assert bns.make_gradients([point], [torch.zeros(24)]).count == 1
    for grads_, outs in (([a], [solid]), ([solid], [a]), ([a], [torch.zeros(a.numel())]), ([a], [torch.zeros(4, 3, 6, 3).to(memory_format=torch.channels_last)]),
                         ([a[:, :, :2]], None), ([a[:, ::2]], None), ([a.expand(2, 4, 6, 3, 3)], None), ([solid.permute(1, 0, 2, 3)], None)):
        with pytest.raises(ValueError):
            bns.make_gradients(grads_, outs)
