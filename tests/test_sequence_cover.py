"""The cut of the paged attention over workgroups, under AddressSanitizer and
UndefinedBehaviorSanitizer (CPU only, no device code; tests/sanitize/seq_cover_driver.cpp)."""
import os
import shutil
import subprocess

import pytest

from tests import test_sanitizers as san


def test_splits_cover_every_key_tile_once(tmp_path):
    if "libclang_rt.asan" in os.environ.get("LD_PRELOAD", ""):
        pytest.skip("the whole suite runs under a sanitizer already; a second runtime cannot load")
    hipcc = shutil.which("hipcc")
    if not (hipcc and os.path.exists(san.CLANGXX)):
        pytest.skip("ROCm clang and hipcc are needed for the sanitizer builds")
    objs = []
    for src in (os.path.join(san.CSRC, "na_seq_api.cpp"), os.path.join(san.SAN, "seq_cover_driver.cpp")):
        objs.append(str(tmp_path / (os.path.basename(src) + ".o")))
        san._run([hipcc] + san.HIP_HOST_ONLY + san.HOST_SAN_FLAGS + ["-c", src, "-o", objs[-1]])
    san._run([san.CLANGXX] + san.SAN_FLAGS + objs + ["-o", str(tmp_path / "driver")])
    res = subprocess.run([str(tmp_path / "driver")], capture_output=True, text=True,
                         env={**os.environ, **san.RUN_ENV}, timeout=300)
    assert res.returncode == 0, res.stdout + res.stderr
    words = res.stdout.split()
    assert words[:2] == ["ok", "cover"], res.stdout
    assert int(words[2]) > 10 ** 6 and int(words[3]) > 10 ** 5  # checks, tiles that were split
