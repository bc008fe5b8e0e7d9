"""The argument checks of the paged cache's and the 4-bit product's entry points, and the host code that sizes and splits,
under AddressSanitizer and UndefinedBehaviorSanitizer (CPU only, no GPU needed), built as in test_host_sanitizers."""
import os
import subprocess

import pytest

from tests.test_host_sanitizers import BUILD, CSRC, DEVICE_OBJECTS, ENV, FLAGS, HOST_SOURCES, ROOT, SAN, hipcc, run

OWN = ["paged_abi.cpp", "paged.hip", "q4.hip"]


@pytest.fixture(scope="module")
def objects():
    """The library's other objects as the ordinary build leaves them."""
    objs = [os.path.join(BUILD, o) for o in DEVICE_OBJECTS + [s + ".o" for s in HOST_SOURCES]]
    if not all(os.path.exists(o) for o in objs):
        from paper_2503_05130_amd import build as B
        B.build()
    return objs


def test_paged_entry_points_clean_under_sanitizers(tmp_path, objects):
    own = []
    for src in OWN + [os.path.join(ROOT, "tests", "c", "sanitize_paged.cpp")]:
        own.append(str(tmp_path / (os.path.basename(src) + ".o")))
        kind = ["-x", "hip"] if src in OWN and src.endswith(".cpp") else []
        run([hipcc()] + FLAGS + SAN + kind + ["-c", os.path.join(CSRC, src), "-o", own[-1]])
    exe = str(tmp_path / "sanitize_paged")
    run([hipcc(), "--offload-arch=gfx950"] + SAN[:4] + own + objects + ["-o", exe])
    res = subprocess.run([exe], capture_output=True, text=True, env=ENV, timeout=600)
    print(res.stdout, res.stderr)
    assert res.returncode == 0, res.stderr[-4000:]
    assert "paged host sanitizer checks passed" in res.stdout
