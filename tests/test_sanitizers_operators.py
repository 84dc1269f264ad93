"""Host code of rotary positions, eviction and cross attention under AddressSanitizer and
UndefinedBehaviorSanitizer (CPU only), driven by tests/sanitize/operators_main.cpp; built as
test_sanitizers builds the rest (HIP sources with the sanitizers on their host side)."""
import os
from concurrent.futures import ThreadPoolExecutor

import pytest

from paper_2603_29494_amd.build import SOURCES
from test_sanitizers import CLANG, CSRC, HIPCC, HOST_SAN, INC, ROCM, ROOT, SAN, run


@pytest.mark.skipif(not (os.path.exists(HIPCC) and os.path.exists(CLANG)),
                    reason="ROCm compilers not available")
def test_operators_under_sanitizers(tmp_path):
    d = str(tmp_path)
    inc = ["-I" + INC, "-I" + CSRC]
    hip = ["-std=c++17", "-O1", "-g"] + inc
    host = [CLANG, "-D__HIP_PLATFORM_AMD__", "-I" + os.path.join(ROCM, "include")] + hip + SAN
    kernels = [HIPCC, "-x", "hip", "--offload-arch=gfx950", "-Xclang", "-target-feature", "-Xclang",
               "-packed-fp32-ops"] + hip + HOST_SAN
    sources = [os.path.join(ROOT, "tests", "sanitize", "operators_main.cpp")]
    sources += [os.path.join(CSRC, s) for s in SOURCES]
    objects = [os.path.basename(s) + ".o" for s in sources]
    jobs = [(kernels if s.endswith(".hip") else host) + ["-c", s, "-o", o]
            for s, o in zip(sources, objects)]
    with ThreadPoolExecutor(max_workers=8) as ex:
        list(ex.map(lambda c: run(c, d), jobs))
    run([HIPCC, "--offload-arch=gfx950"] + HOST_SAN[:4] + objects + ["-o", "operators_san"], d)
    out = run([os.path.join(d, "operators_san")], d)
    assert out.strip().endswith("ok"), out
