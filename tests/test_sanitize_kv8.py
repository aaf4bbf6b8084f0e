"""The 8-bit cache's argument checks under AddressSanitizer and
UndefinedBehaviorSanitizer, with stand-ins for the launches that check what is let
through (CPU only; ``sanitize/kv8_driver.cpp``)."""
import os

from tests.test_sanitize import CSRC, HERE, ROOT, SAN, _check_clean, _env, _run, pytestmark  # noqa: F401


def test_kv8_host_under_sanitizers(tmp_path):
    exe = str(tmp_path / "kv8_driver")
    _run(["g++", "-std=c++17", *SAN, "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
          "-I" + os.path.join(ROOT, "include"), "-I" + CSRC, os.path.join(CSRC, "kv8_host.cpp"),
          os.path.join(CSRC, "jfkv_host.cpp"), os.path.join(HERE, "stubs.cpp"),
          os.path.join(HERE, "kv8_driver.cpp"), "-o", exe])
    _check_clean(_run([exe], timeout=300, env=_env()), "checks passed")
