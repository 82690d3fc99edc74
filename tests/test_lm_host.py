"""Host code of the language-model operators under AddressSanitizer and UndefinedBehaviorSanitizer, on a machine without a GPU: see
tests/host_checks/lm_harness.cpp.  And the marshalling of their calls through the extension against ctypes."""
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
    exe = str(tmp_path_factory.mktemp("san") / "lm_harness")
    r = subprocess.run([gxx, "-std=c++17", "-O1", "-g", "-Wall", "-Werror", *SAN, os.path.join(ROOT, "tests", "host_checks", "lm_harness.cpp"), "-o", exe],
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
    checked, apart = _run(harness, "overlaps")
    assert checked > 10 ** 5 and 0 < apart < checked


class Tensor:
    def __init__(self, address, nbytes=0):
        self.address, self.nbytes = address, nbytes

    def data_ptr(self):
        return self.address


SPECS = {"rms": bns.make_rms(5, 64, "f32", out="e4m3", group=32, pow2_scales=True, eps=0.5, x_stride=70), "head": bns.make_head(6, 64, 1000, "f32", piece=512),
         "distill": bns.make_distill(7, 1000, 9, "f32", temperature=3.0)}


@pytest.mark.parametrize("through", ["extension", "ctypes"])
@pytest.mark.parametrize("name", bns._EVERY_STEP_LM)
def test_arguments_reach_the_library(name, through, monkeypatch):
    received = []

    def stand_in(which):
        restype, argtypes = bns._PROTOS["bns_" + which]
        return C.CFUNCTYPE(restype, *argtypes)(lambda *a: received.append([bytes(x.contents) if isinstance(x, C._Pointer) else x for x in a]) or bns.BNS_EWORKSPACE)

    bns.load()
    try:
        keep = {n: stand_in(n) for n in bns._EVERY_STEP_LM}
        bns._call.bind_lm(bns.bns_rms, bns.bns_head, bns.bns_distill, *(C.cast(keep[n], C.c_void_p).value for n in bns._EVERY_STEP_LM))
        monkeypatch.setattr(bns, "_lib", types.SimpleNamespace(bns_status_string=bns._lib.bns_status_string, **{"bns_" + n: f for n, f in keep.items()}))
        if through == "ctypes":
            monkeypatch.setattr(bns, "_call", bns._NoExtension)
        monkeypatch.setattr(bns, "_stream", lambda t: 0x7fff12345678)
        given, wanted = [], []
        for i, p in enumerate(inspect.signature(getattr(bns, "bns_" + name)).parameters):
            if p in SPECS:
                given.append(SPECS[p])
                wanted.append(bytes(SPECS[p]))
            elif p in ("residual", "dsum", "scales"):
                given.append(None)
                wanted.append(None)
            else:
                given.append(Tensor(2 ** 47 + 4096 * i, 12345))
                wanted.append(2 ** 47 + 4096 * i)
            if p == "workspace":
                wanted.append(12345)
        with pytest.raises(bns.BnsError) as e:
            getattr(bns, "bns_" + name)(*given)
        assert e.value.status == bns.BNS_EWORKSPACE and received == [wanted + [0x7fff12345678]]
        with pytest.raises(Exception):
            getattr(bns, "bns_" + name)(SPECS["rms" if "rms" not in name else "head"], *given[1:])      # another operator's description
        assert len(received) == 1
    finally:
        monkeypatch.undo()
        bns.load(reload=True)
