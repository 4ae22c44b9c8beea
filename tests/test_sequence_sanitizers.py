"""AddressSanitizer and UndefinedBehaviorSanitizer over the host code of the sequence operators
(CPU only, no device code): na_seq_api.cpp through valid, invalid and extreme problems, with
launchers that check what each kernel would be handed (tests/sanitize/seq_driver.cpp)."""
import concurrent.futures
import os
import shutil
import subprocess

import pytest

from tests import test_sanitizers as san


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    if "libclang_rt.asan" in os.environ.get("LD_PRELOAD", ""):
        pytest.skip("the whole suite runs under a sanitizer already; a second runtime cannot load")
    hipcc = shutil.which("hipcc")
    if not (hipcc and os.path.exists(san.CLANGXX)):
        pytest.skip("ROCm clang and hipcc are needed for the sanitizer builds")
    out = tmp_path_factory.mktemp("seq_sanitize")
    objs = []
    compiles = []
    for src in (os.path.join(san.CSRC, "na_seq_api.cpp"), os.path.join(san.SAN, "seq_driver.cpp")):
        objs.append(str(out / (os.path.basename(src) + ".o")))
        compiles.append([hipcc] + san.HIP_HOST_ONLY + san.HOST_SAN_FLAGS + ["-c", src, "-o", objs[-1]])
    with concurrent.futures.ThreadPoolExecutor(2) as ex:
        list(ex.map(san._run, compiles))
    san._run([san.CLANGXX] + san.SAN_FLAGS + objs + ["-o", str(out / "seq_driver")])
    return out / "seq_driver"


def test_sequence_driver_is_clean(driver):
    res = subprocess.run([str(driver)], capture_output=True, text=True,
                         env={**os.environ, **san.RUN_ENV}, timeout=300)
    assert res.returncode == 0, res.stdout + res.stderr
    words = res.stdout.split()
    assert words[:2] == ["ok", "sequence"], res.stdout
    assert int(words[2]) > 100000 and int(words[3]) > 10000  # checks, stubbed launches
