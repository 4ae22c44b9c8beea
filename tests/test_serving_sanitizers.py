"""AddressSanitizer and UndefinedBehaviorSanitizer over the host code of the cache operators for long
contexts (CPU only, no device code): na_long_api.cpp through valid, invalid and extreme problems,
with launchers that check what each kernel would be handed (tests/sanitize/long_driver.cpp)."""
import concurrent.futures
import os
import shutil
import subprocess

import pytest

from tests import test_sanitizers as san


def test_long_driver_is_clean(tmp_path):
    if "libclang_rt.asan" in os.environ.get("LD_PRELOAD", ""):
        pytest.skip("the whole suite runs under a sanitizer already; a second runtime cannot load")
    hipcc = shutil.which("hipcc")
    if not (hipcc and os.path.exists(san.CLANGXX)):
        pytest.skip("ROCm clang and hipcc are needed for the sanitizer builds")
    objs, compiles = [], []
    for src in (os.path.join(san.CSRC, "na_long_api.cpp"), os.path.join(san.SAN, "long_driver.cpp")):
        objs.append(str(tmp_path / (os.path.basename(src) + ".o")))
        compiles.append([hipcc] + san.HIP_HOST_ONLY + san.HOST_SAN_FLAGS + ["-c", src, "-o", objs[-1]])
    with concurrent.futures.ThreadPoolExecutor(2) as ex:
        list(ex.map(san._run, compiles))
    san._run([san.CLANGXX] + san.SAN_FLAGS + objs + ["-o", str(tmp_path / "long_driver")])
    res = subprocess.run([str(tmp_path / "long_driver")], capture_output=True, text=True,
                         env={**os.environ, **san.RUN_ENV}, timeout=300)
    assert res.returncode == 0, res.stdout + res.stderr
    words = res.stdout.split()
    assert words[:2] == ["ok", "long"], res.stdout
    assert int(words[2]) > 100000 and int(words[3]) > 10000  # checks, stubbed launches


def test_long_limits_driver_is_clean(tmp_path):
    """Grids, cuts and workspaces at the ends of what the checks accept."""
    if "libclang_rt.asan" in os.environ.get("LD_PRELOAD", ""):
        pytest.skip("the whole suite runs under a sanitizer already; a second runtime cannot load")
    hipcc = shutil.which("hipcc")
    if not (hipcc and os.path.exists(san.CLANGXX)):
        pytest.skip("ROCm clang and hipcc are needed for the sanitizer builds")
    objs, compiles = [], []
    for src in (os.path.join(san.CSRC, "na_long_api.cpp"),
                os.path.join(san.SAN, "long_limits_driver.cpp")):
        objs.append(str(tmp_path / (os.path.basename(src) + ".o")))
        compiles.append([hipcc] + san.HIP_HOST_ONLY + san.HOST_SAN_FLAGS + ["-c", src, "-o", objs[-1]])
    with concurrent.futures.ThreadPoolExecutor(2) as ex:
        list(ex.map(san._run, compiles))
    san._run([san.CLANGXX] + san.SAN_FLAGS + objs + ["-o", str(tmp_path / "limits")])
    res = subprocess.run([str(tmp_path / "limits")], capture_output=True, text=True,
                         env={**os.environ, **san.RUN_ENV}, timeout=300)
    assert res.returncode == 0, res.stdout + res.stderr
    assert res.stdout.split()[:2] == ["ok", "limits"], res.stdout
