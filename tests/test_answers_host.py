"""Host code of the calls of a step on a model's own answers under AddressSanitizer and UndefinedBehaviorSanitizer, on a machine without a GPU: see
tests/host_checks/answers_harness.cpp.  And the marshalling of their calls through the extension against ctypes."""
import ctypes as C
import inspect
import os
import shutil
import subprocess
import types

import pytest

from paper_1810_10962_amd import bns

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SAN = ["-fsanitize=address,undefined", "-fno-sanitize-recover=all"]
ENV = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")


@pytest.fixture(scope="module")
def harness(tmp_path_factory):
    gxx = shutil.which("g++")
    if not gxx:
        pytest.skip("g++ not found")
    exe = str(tmp_path_factory.mktemp("san") / "answers_harness")
    r = subprocess.run([gxx, "-std=c++17", "-O1", "-g", "-Wall", "-Werror", *SAN, os.path.join(ROOT, "tests", "host_checks", "answers_harness.cpp"), "-o", exe],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    return exe


def _run(*cmd):
    r = subprocess.run(cmd, capture_output=True, text=True, env=ENV)
    assert r.returncode == 0, f"exit {r.returncode}\n{r.stdout[-2000:]}\n{r.stderr[-4000:]}"
    return [int(v) for v in r.stdout.split()[1::2]]


def test_descriptions_of_extreme_values(harness):
    accepted, rejected = _run(harness)
    assert accepted > 100 and rejected > 10 ** 5


def test_overlaps_are_what_they_mean(harness):
    checked, apart, lists, fine = _run(harness, "overlaps")
    assert checked > 10 ** 5 and 0 < apart < checked and lists > 10 ** 5 and 0 < fine < lists


def test_structures_have_the_sizes_of_the_header(tmp_path):
    text = '#include "bns.h"\n#include <stdio.h>\nint main(void) { printf("%zu %zu %zu %zu", sizeof(bns_head_strides), sizeof(bns_qk), sizeof(bns_logprob), sizeof(bns_gradient)); }\n'
    (tmp_path / "s.c").write_text(text)
    subprocess.run(["gcc", "-std=c99", "-I" + os.path.join(ROOT, "include"), str(tmp_path / "s.c"), "-o", str(tmp_path / "s")], check=True)
    sizes = [int(v) for v in subprocess.run([str(tmp_path / "s")], capture_output=True, text=True, check=True).stdout.split()]
    assert sizes == [C.sizeof(s) for s in (bns.bns_head_strides, bns.bns_qk, bns.bns_logprob, bns.bns_gradient)]


class Tensor:
    def __init__(self, address, nbytes=0):
        self.address, self.nbytes, self.count = address, nbytes, 77

    def data_ptr(self):
        return self.address

    def get_device(self):
        return -1


SPECS = {"qk": bns.make_qk(5, 3, 1, 64, "f32", rotated=32, interleaved=True, eps=0.5, q=(300, 70), dk=(64, 400)),
         "logprob": bns.make_logprob(7, 1000, "f32", top=9, temperature=3.0, dlogits_stride=1001)}


@pytest.mark.parametrize("through", ["extension", "ctypes"])
@pytest.mark.parametrize("name", bns._EVERY_STEP_ANSWERS)
def test_arguments_reach_the_library(name, through, monkeypatch):
    received = []

    def stand_in(which):
        restype, argtypes = bns._PROTOS["bns_" + which]
        return C.CFUNCTYPE(restype, *argtypes)(lambda *a: received.append([bytes(x.contents) if isinstance(x, C._Pointer) else x for x in a]) or bns.BNS_EWORKSPACE)

    bns.load()
    try:
        keep = {n: stand_in(n) for n in bns._EVERY_STEP_ANSWERS}
        bns._call.bind_answers(bns.bns_qk, bns.bns_logprob, *(C.cast(keep[n], C.c_void_p).value for n in bns._EVERY_STEP_ANSWERS))
        monkeypatch.setattr(bns, "_lib", types.SimpleNamespace(bns_status_string=bns._lib.bns_status_string, **{"bns_" + n: f for n, f in keep.items()}))
        if through == "ctypes":
            monkeypatch.setattr(bns, "_call", bns._NoExtension)
        monkeypatch.setattr(bns, "_stream", lambda t: 0x7fff12345678)
        given, wanted = [], []
        for i, p in enumerate(inspect.signature(getattr(bns, "bns_" + name)).parameters):
            if p in SPECS:
                given.append(SPECS[p])
                wanted.append(bytes(SPECS[p]))
            elif p in ("k_weight", "dk_weight", "top_ids"):
                given.append(None)
                wanted.append(None)
            elif p == "max_norm":
                given.append(0.25)
                wanted.append(0.25)
            else:
                given.append(Tensor(2 ** 47 + 4096 * i, 12345))
                wanted.append(2 ** 47 + 4096 * i)
            if p == "workspace":
                wanted.append(12345)
            if p == "gradients":
                wanted.append(77)
        with pytest.raises(bns.BnsError) as e:
            getattr(bns, "bns_" + name)(*given)
        assert e.value.status == bns.BNS_EWORKSPACE and received == [wanted + [0x7fff12345678]]
        if name.startswith(("qk", "logprob")):
            with pytest.raises(Exception):
                getattr(bns, "bns_" + name)(SPECS["logprob" if name.startswith("qk") else "qk"], *given[1:])      # another operator's description
            assert len(received) == 1
    finally:
        monkeypatch.undo()
        bns.load(reload=True)


def test_a_call_goes_to_the_device_of_its_tensors(monkeypatch):
    """Tensors on another device than the current one: that one is current while the call is made."""
    import torch
    current, seen = [0], []

    class On:
        def __init__(self, device):
            self.device = device

        def __enter__(self):
            self.before, current[0] = current[0], self.device

        def __exit__(self, *_):
            current[0] = self.before

    class There(Tensor):
        def get_device(self):
            return 3

    monkeypatch.setattr(bns, "_current_device", lambda: current[0])
    monkeypatch.setattr(torch.cuda, "device", On)
    monkeypatch.setattr(bns, "_stream", lambda t: 1)
    monkeypatch.setattr(bns, "_calls", lambda: types.SimpleNamespace(grads_norm=lambda *a: seen.append(current[0]) or 0))
    bns.bns_grads_norm(Tensor(0), There(16), None, There(32, 9))
    assert seen == [3] and current == [0]
