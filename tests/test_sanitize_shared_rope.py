"""Argument checks of the rotary positions and of the attention of requests that share
prefixes under AddressSanitizer and UndefinedBehaviorSanitizer, with stand-ins for the
launches that check what is let through (CPU only; ``sanitize/shared_rope_driver.cpp``)."""
import os

import pytest

base = pytest.importorskip("tests.test_sanitize")
pytestmark = base.pytestmark


def test_hosts_under_sanitizers(tmp_path):
    exe = str(tmp_path / "shared_rope_driver")
    src = [os.path.join(base.CSRC, n) for n in ("rope_host.cpp", "kv8_shared_host.cpp", "jfkv_host.cpp")]
    src += [os.path.join(base.HERE, n) for n in ("stubs.cpp", "shared_rope_driver.cpp")]
    base._run(["g++", "-std=c++17", *base.SAN, "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
               "-I" + os.path.join(base.ROOT, "include"), "-I" + base.CSRC, *src, "-o", exe])
    base._check_clean(base._run([exe], timeout=300, env=base._env()), "checks passed")
