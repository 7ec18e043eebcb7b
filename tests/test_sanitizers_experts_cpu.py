"""The host code of layers with experts, and of norms of queries and keys, under
AddressSanitizer and UndefinedBehaviorSanitizer (CPU): every source of libmxq built
with the sanitizers on its host code only, linked with
tests/sanitize/experts_host_driver.cpp, which runs the size queries, the argument
checks and, for valid arguments, the path up to the kernel launch (refused by the
runtime without a device)."""
import concurrent.futures as cf
import os

import pytest

from paper_2607_17733_amd import build as hip_build
from test_sanitizers_cpu import CSRC, FLAGS, HIPCC, HOST_SAN, ROOT, _run


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not installed")
def test_experts_host_paths_under_sanitizers(tmp_path):
    def compile_one(src):
        path = src if os.path.isabs(src) else os.path.join(CSRC, src)
        obj = os.path.join(tmp_path, os.path.basename(src) + ".o")
        _run([HIPCC] + FLAGS + HOST_SAN + ["-c", path, "-o", obj])
        return obj

    driver = os.path.join(ROOT, "tests", "sanitize", "experts_host_driver.cpp")
    sources = sorted(hip_build.SOURCES, key=lambda s: not s.startswith("attn"))   # the longest first
    with cf.ThreadPoolExecutor(max_workers=8) as ex:
        objs = list(ex.map(compile_one, sources + [driver]))
    exe = os.path.join(tmp_path, "experts_driver")
    _run([HIPCC, "--offload-arch=gfx950"] + HOST_SAN + ["-o", exe] + objs)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=1",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1", HIP_VISIBLE_DEVICES="")
    r = _run([exe], env=env, timeout=300)
    assert "experts host driver: ok" in r.stdout
