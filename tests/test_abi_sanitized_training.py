"""The host code of the gated recurrence, the loss on logits and the gradients' norm under AddressSanitizer and
UndefinedBehaviorSanitizer: their source files, with the sanitizers on the host code only, linked with abi_training_check.cpp
and run on the CPU.  No GPU is used."""
import concurrent.futures as cf
import os
import subprocess

import pytest

from tests.test_abi_sanitized import CSRC, FLAGS, ROOT, SAN, _hipcc, _run


@pytest.mark.slow
def test_host_code_is_clean_under_asan_and_ubsan(tmp_path):
    hipcc = _hipcc()
    if hipcc is None:
        pytest.skip("hipcc not found")
    names = ("gatedrec", "ppo_logits", "adamw", "abi_misc")
    objs = [str(tmp_path / (n + ".o")) for n in names]
    check = str(tmp_path / "abi_training_check.o")
    with cf.ThreadPoolExecutor(8) as ex:
        futs = [ex.submit(_run, [hipcc, *FLAGS, *SAN, "-c", os.path.join(CSRC, n + ".hip"), "-o", o]) for n, o in zip(names, objs)]
        futs.append(ex.submit(_run, [hipcc, "-O1", "-g", "-std=c++17", *SAN, "-I", os.path.join(ROOT, "include"), "-c",
                                     os.path.join(ROOT, "tests", "abi_training_check.cpp"), "-o", check]))
        for f in futs:
            f.result()
    exe = str(tmp_path / "abi_training_check")
    _run([hipcc, "--offload-arch=gfx950", *SAN, *objs, check, "-o", exe])
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=1", UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1",
               HIP_VISIBLE_DEVICES="")
    res = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
    assert res.returncode == 0, (res.stdout + res.stderr)[-6000:]
    assert "checks passed" in res.stdout
