"""The argument checks and sizes of the 4-bit matrices, the 4-bit cache and the log probabilities under AddressSanitizer and
UndefinedBehaviorSanitizer (CPU only, no GPU needed), built as in test_host_sanitizers."""
import os
import subprocess

import pytest

from tests.test_host_sanitizers import BUILD, CSRC, DEVICE_OBJECTS, ENV, FLAGS, HOST_SOURCES, ROOT, SAN, hipcc, run

OWN = ["mx4_abi.cpp", "paged_abi.cpp", "logprobs_abi.cpp", "logprobs.hip"]
BUILT = [s + ".o" for s in ("mx4.hip", "mx4_gemm.hip", "paged.hip", "q4.hip")]


@pytest.fixture(scope="module")
def objects():
    """The library's other objects as the ordinary build leaves them."""
    objs = [os.path.join(BUILD, o) for o in DEVICE_OBJECTS + BUILT + [s + ".o" for s in HOST_SOURCES]]
    if not all(os.path.exists(o) for o in objs):
        from paper_2503_05130_amd import build as B
        B.build()
    return objs


def test_entry_points_clean_under_sanitizers(tmp_path, objects):
    own = []
    for src in OWN + [os.path.join(ROOT, "tests", "c", "sanitize_mx4.cpp")]:
        own.append(str(tmp_path / (os.path.basename(src) + ".o")))
        kind = ["-x", "hip"] if src in OWN and src.endswith(".cpp") else []
        run([hipcc()] + FLAGS + SAN + kind + ["-c", os.path.join(CSRC, src), "-o", own[-1]])
    exe = str(tmp_path / "sanitize_mx4")
    run([hipcc(), "--offload-arch=gfx950"] + SAN[:4] + own + objects + ["-o", exe])
    res = subprocess.run([exe], capture_output=True, text=True, env=ENV, timeout=600)
    print(res.stdout, res.stderr)
    assert res.returncode == 0, res.stderr[-4000:]
    assert "4-bit host sanitizer checks passed" in res.stdout
