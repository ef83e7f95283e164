"""Launches and sizes of the layer norm on the CPU: tests/sanitize/norm_driver.cpp, linked with the translation unit, under AddressSanitizer and
UndefinedBehaviorSanitizer."""
import os

import pytest

from test_sanitizers import CSRC, ENV, HIPCC, ROCM_INCLUDE, ROOT, SAN, _run


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not found")
def test_sizes_to_the_limits_and_each_row_in_one_launch(tmp_path):
    host_san = []
    for f in SAN:
        host_san += ["-Xarch_host", f]
    common = ["-std=c++17", "-I", os.path.join(ROOT, "include"), "-I", CSRC]
    objs = []
    # only the host's side is compiled; the image with the kernels, whose address the driver's registration never looks at, is not there
    for src, extra in ((os.path.join(CSRC, "rocket_layer_norm.hip"), ["--offload-arch=gfx950", "--offload-host-only"]),
                       (os.path.join(ROOT, "tests", "sanitize", "norm_driver.cpp"), ["-x", "c++", "-D__HIP_PLATFORM_AMD__", "-I", ROCM_INCLUDE])):
        obj = str(tmp_path / (os.path.basename(src) + ".o"))
        _run([HIPCC] + extra + common + host_san + ["-c", src, "-o", obj])
        objs.append(obj)
    exe = str(tmp_path / "norm_driver")
    _run([HIPCC, "--offload-arch=gfx950"] + host_san + ["-Wl,--unresolved-symbols=ignore-in-object-files"] + objs + ["-o", exe])
    assert "norm driver: ok" in _run([exe], env=ENV)
