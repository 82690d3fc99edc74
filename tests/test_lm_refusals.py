"""What the language-model calls refuse, before anything is enqueued: made-up addresses that are never dereferenced suffice, no GPU is needed."""
import ctypes as C

import pytest

from paper_1810_10962_amd import bns

X, R, S, Y, W, V, WS = 0x10000000, 0x20000000, 0x30000000, 0x40000000, 0x50000000, 0x60000000, 0x70000000
NULL = 0


def rms_forward(x=X, r=R, w=W, s=S, y=Y, scales=NULL, rstd=V, rows=8, width=64, **kw):
    spec = kw.pop("spec", None) or bns.make_rms(rows, width, **kw)
    return bns.load().bns_rms_forward(C.byref(spec), x, r, w, s, y, scales, rstd, None)


def rms_backward(x=X, w=W, rstd=V, dy=Y, dsum=R, dx=S, dw=V + 4096, ws=WS, short=0, rows=8, width=64, **kw):
    spec = bns.make_rms(rows, width, **kw)
    return bns.load().bns_rms_backward(C.byref(spec), x, w, rstd, dy, dsum, dx, dw, ws, max(0, bns.bns_rms_workspace_bytes(spec) - short), None)


def head(call, h=X, w=W, t=V, lse=V + 4096, loss=V + 8192, dh=S, dw=Y, ws=WS, short=0, tokens=8, width=64, vocab=100, **kw):
    spec = bns.make_head(tokens, width, vocab, **kw)
    n = max(0, bns.bns_head_workspace_bytes(spec) - short)
    if call == "forward":
        return bns.load().bns_head_forward(C.byref(spec), h, w, t, loss, lse, ws, n, None)
    return bns.load().bns_head_backward(C.byref(spec), h, w, t, lse, loss, dh, dw, ws, n, None)


def distill(call, z=X, ids=R, u=W, dloss=V, loss=V + 4096, lse=V + 8192, dz=Y, tokens=8, vocab=100, k=4, **kw):
    spec = bns.make_distill(tokens, vocab, k, **kw)
    if call == "forward":
        return bns.load().bns_distill_forward(C.byref(spec), z, ids, u, dloss, loss, lse, dz, None)
    return bns.load().bns_distill_backward(C.byref(spec), z, ids, u, lse, dloss, dz, None)


@pytest.mark.parametrize("kw", [
    dict(x=NULL), dict(w=NULL), dict(y=NULL), dict(r=NULL), dict(x=X + 4), dict(r=R + 8), dict(s=S + 2), dict(y=Y + 1), dict(w=W + 4),
    dict(rows=-1), dict(width=0), dict(width=-64), dict(dtype=2), dict(dtype=-1), dict(weight_dtype=7), dict(out=2), dict(eps=-1e-6),
    dict(eps=float("nan")), dict(eps=float("inf")), dict(group=32), dict(pow2_scales=True), dict(scales=V + 4096), dict(out="e4m3"),
    dict(out="e4m3", scales=V + 4096, group=16), dict(out="e4m3", scales=V + 4096, group=-32), dict(out="e4m3", scales=V + 4096, group=96),
    dict(x_stride=63), dict(residual_stride=-1), dict(sum_stride=1), dict(y_stride=63),
    dict(s=X + 64), dict(s=R + 128), dict(s=X, x_stride=128), dict(y=R), dict(y=S), dict(y=X + 16), dict(y=X, s=X),
    dict(y=X, out="e4m3", scales=V + 4096)])
def test_rms_forward_refuses(kw):
    assert rms_forward(**kw) == bns.BNS_EINVAL


@pytest.mark.parametrize("kw", [
    dict(x=NULL), dict(w=NULL), dict(rstd=NULL), dict(dy=NULL), dict(dx=NULL), dict(dw=NULL), dict(ws=NULL), dict(x=X + 4), dict(dy=Y + 2), dict(dsum=R + 4),
    dict(dx=S + 8), dict(ws=WS + 8), dict(dx=X), dict(dx=Y + 16), dict(dx=R + 128), dict(x_stride=3), dict(width=0), dict(rows=-2), dict(eps=-1.0)])
def test_rms_backward_refuses(kw):
    assert rms_backward(**kw) == bns.BNS_EINVAL


@pytest.mark.parametrize("call", ["forward", "backward"])
@pytest.mark.parametrize("kw", [
    dict(h=NULL), dict(w=NULL), dict(t=NULL), dict(lse=NULL), dict(loss=NULL), dict(ws=NULL), dict(h=X + 2), dict(w=W + 8), dict(ws=WS + 4), dict(tokens=-1), dict(width=0),
    dict(vocab=0), dict(vocab=-5), dict(dtype=3), dict(piece=-1), dict(hidden_stride=63), dict(weight_stride=-64)])
def test_head_refuses(call, kw):
    assert head(call, **kw) == bns.BNS_EINVAL


@pytest.mark.parametrize("kw", [dict(dh=NULL), dict(dw=NULL), dict(dh=S + 4), dict(dw=Y + 8), dict(dh=X), dict(dh=W + 16), dict(dw=W), dict(dw=X + 32), dict(dw=S + 512)])
def test_head_backward_refuses(kw):
    assert head("backward", **kw) == bns.BNS_EINVAL


@pytest.mark.parametrize("call", ["forward", "backward"])
@pytest.mark.parametrize("kw", [
    dict(z=NULL), dict(ids=NULL), dict(u=NULL), dict(lse=NULL), dict(z=X + 2), dict(ids=R + 8), dict(u=W + 4), dict(dz=Y + 4), dict(tokens=-1), dict(vocab=0), dict(k=0),
    dict(k=-1), dict(dtype=2), dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=float("nan")), dict(temperature=float("inf")), dict(logits_stride=99),
    dict(dlogits_stride=-100), dict(dz=X + 16), dict(dz=X, dlogits_stride=200), dict(dz=R), dict(dz=W), dict(dloss=NULL)])
def test_distill_refuses(call, kw):
    assert distill(call, **kw) == bns.BNS_EINVAL


def test_distill_needs_its_outputs():
    assert distill("forward", loss=NULL) == bns.BNS_EINVAL
    assert distill("backward", dz=NULL) == bns.BNS_EINVAL


def test_beyond_the_limits():
    big = dict(x=NULL, r=NULL, w=NULL, s=NULL, y=NULL)      # (the limits come before the pointers)
    for kw in (dict(rows=2 ** 31), dict(width=16385), dict(x_stride=2 ** 31), dict(y_stride=2 ** 40)):
        assert rms_forward(**{**big, **kw}) == bns.BNS_EUNSUPPORTED
    for kw in (dict(tokens=2 ** 20 + 1), dict(width=65537), dict(vocab=2 ** 24), dict(hidden_stride=2 ** 31), dict(weight_stride=2 ** 31)):
        assert head("forward", **kw) == head("backward", **kw) == bns.BNS_EUNSUPPORTED
        assert bns.bns_head_workspace_bytes(bns.make_head(**{**dict(tokens=8, width=64, vocab=100), **kw})) == 0
    for kw in (dict(tokens=2 ** 31), dict(vocab=2 ** 30), dict(k=1025), dict(logits_stride=2 ** 31), dict(dlogits_stride=2 ** 33)):
        assert distill("forward", **kw) == distill("backward", **kw) == bns.BNS_EUNSUPPORTED
    assert bns.bns_rms_workspace_bytes(bns.make_rms(4, 20000)) == 0
    lib = bns.load()
    assert lib.bns_rms_forward(None, X, R, W, S, Y, None, V, None) == bns.BNS_EINVAL
    assert lib.bns_head_forward(None, X, W, V, V, V, WS, 1 << 30, None) == bns.BNS_EINVAL
    assert lib.bns_distill_backward(None, X, R, W, V, V, Y, None) == bns.BNS_EINVAL
    assert lib.bns_head_workspace_bytes(None) == 0 and lib.bns_rms_workspace_bytes(None) == 0


def test_small_workspaces():
    assert rms_backward(short=1) == bns.BNS_EWORKSPACE
    for call in ("forward", "backward"):
        assert head(call, short=1) == bns.BNS_EWORKSPACE
        assert head(call, short=1, dtype="f32", width=100, tokens=3000, vocab=50000) == bns.BNS_EWORKSPACE


def test_nothing_to_do():
    """Matrices without rows: null pointers are fine, and nothing is launched where there is nothing to write."""
    before = bns.bns_get_option("launch_count")
    assert rms_forward(rows=0, x=NULL, r=NULL, s=NULL, y=NULL) == bns.BNS_OK
    assert head("forward", tokens=0, h=NULL, t=NULL, loss=NULL, lse=NULL) == bns.BNS_OK
    for call in ("forward", "backward"):
        assert distill(call, tokens=0, z=NULL, ids=NULL, u=NULL, dz=NULL, loss=NULL, lse=NULL) == bns.BNS_OK
    assert bns.bns_get_option("launch_count") == before


def test_workspace_grows_with_the_piece_and_stays_modest():
    """The logits of 4096 tokens and 131072 words in 32 bits would be 2 GiB."""
    size = lambda **kw: bns.bns_head_workspace_bytes(bns.make_head(4096, 4096, 131072, **kw))  # noqa: E731
    assert size(piece=256) < size(piece=4096) < size(piece=65536)
    assert size() < 1 << 30


def test_the_binding_raises():
    class T:
        nbytes = 0

        def data_ptr(self):
            return NULL

        def get_device(self):
            return -1

        device = "cpu"

    with pytest.raises(bns.BnsError) as e:
        old, bns._stream = bns._stream, lambda t: 0
        try:
            bns.bns_rms_forward(bns.make_rms(4, 64), T(), None, T(), None, T(), None, None)
        finally:
            bns._stream = old
    assert e.value.status == bns.BNS_EINVAL
