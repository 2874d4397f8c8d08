"""The host side of the operators around drafting under AddressSanitizer and UndefinedBehaviorSanitizer (CPU only; nothing of the
kind runs on the GPU): planning and argument validation, which return before anything is launched."""
import os
import shutil

import pytest

from tests.test_sanitizers import HERE, SAN_ENV, _run


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="hipcc is needed to build the library's host side")
def test_drafting_validation_under_sanitizers(tmp_path):
    from paper_2502_20704_amd import build as hip_build

    exe = str(tmp_path / "drafting_san")
    flags = [f for f in hip_build.FLAGS if f not in ("-shared", "-O3")]
    cmd = ["hipcc", "-O1", "-g", *flags, "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
           "-Xarch_host", "-fno-sanitize-recover=all", "-o", exe, os.path.join(HERE, "drafting_driver.cpp"), hip_build.SRC_DRAFTING]
    r = _run(cmd)
    assert r.returncode == 0, "the sanitizer build of the host side failed"
    r = _run([exe], env=SAN_ENV, timeout=300)
    assert r.returncode == 0 and "0 unexpected results" in r.stdout
    assert "ERROR: AddressSanitizer" not in r.stdout and "runtime error" not in r.stdout
