"""How blocks of an append to the 8-bit cache share its work, checked on the CPU under
AddressSanitizer and UndefinedBehaviorSanitizer (``sanitize/append_grid_driver.cpp``)."""
import os

import pytest

base = pytest.importorskip("tests.test_sanitize")
pytestmark = base.pytestmark


def test_every_block_has_a_place_of_its_own(tmp_path):
    exe = str(tmp_path / "append_grid_driver")
    base._run(["g++", "-std=c++17", *base.SAN, "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
               "-I" + base.CSRC, os.path.join(base.HERE, "append_grid_driver.cpp"), "-o", exe])
    base._check_clean(base._run([exe], timeout=300, env=base._env()), "checks passed")
