"""What the host plans for window attention's backward pass (no GPU needed): the calls of
test_gpu_window_variants.py reach the kernels that they are there for."""
import os
import shutil
import subprocess

import pytest

from tests.test_build_flags import _builder
from tests.test_gpu_window_variants import VARIANTS

DRIVER = r"""
#include <cstdio>
#include "ops_internal.h"
using namespace bsa_ops;
int main() {
  int B, H, Hkv, Nq, Nkv, d, left, right, sinks;
  while (std::scanf("%d %d %d %d %d %d %d %d %d", &B, &H, &Hkv, &Nq, &Nkv, &d, &left, &right, &sinks) == 9) {
    WindowArgs a{};
    a.B = B, a.H = H, a.Hkv = Hkv, a.group = H / Hkv, a.Nq = Nq, a.Nkv = Nkv;
    a.left = left < 0 ? kFar : left, a.right = right < 0 ? kFar : right, a.sinks = sinks < Nkv ? sinks : Nkv;
    plan_backward(&a, d);
    std::printf("deep %d slices %d sink_slices %d\n", a.deep, a.slices, a.sink_slices);
  }
}
"""


def test_variants_of_the_backward_calls(tmp_path):
    b, gxx = _builder(), shutil.which("g++")
    if gxx is None:
        pytest.skip("g++ not available")
    try:
        rocm = os.path.dirname(os.path.dirname(b.hipcc()))
    except RuntimeError:
        pytest.skip("hipcc not available")
    obj = os.path.join(b.BUILD, "window_bwd.o")
    sources = [os.path.join(b.CSRC, f) for f in ("window_bwd.hip", "window_common.h", "ops_internal.h")]
    if not os.path.exists(obj) or os.path.getmtime(obj) < max(map(os.path.getmtime, sources)):
        os.makedirs(b.BUILD, exist_ok=True)
        b._compile("window_bwd.hip")
    (tmp_path / "plan.cpp").write_text(DRIVER)
    exe = str(tmp_path / "plan")
    cmd = [gxx, "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(rocm, "include"), "-I", b.CSRC,
           str(tmp_path / "plan.cpp"), obj, "-o", exe, "-L", os.path.join(rocm, "lib"), "-lamdhip64",
           "-Wl,-rpath," + os.path.join(rocm, "lib")]
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout
    lines = "".join("%d %d %d %d %d %d %d %d %d\n" % c[:9] for c, _ in VARIANTS.values())
    out = subprocess.run([exe], input=lines, stdout=subprocess.PIPE, text=True, check=True, timeout=60).stdout.splitlines()
    assert len(out) == len(VARIANTS)
    for (name, (_, want)), line in zip(VARIANTS.items(), out):
        w = line.split()
        got = dict(zip(w[::2], map(int, w[1::2])))
        assert {k: got[k] for k in want} == want, (name, line)
