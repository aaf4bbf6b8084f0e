"""The plan of the attention of requests that share prefixes, carried out on the CPU for
thousands of batches, under AddressSanitizer and UndefinedBehaviorSanitizer
(``sanitize/shared_plan_driver.cpp``): every step in one segment, every record that the
join reads written by one block."""
import os

import pytest

base = pytest.importorskip("tests.test_sanitize")
pytestmark = base.pytestmark


def test_every_record_that_is_joined_has_been_written(tmp_path):
    exe = str(tmp_path / "shared_plan_driver")
    base._run(["g++", "-std=c++17", *base.SAN, "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
               "-I" + os.path.join(base.ROOT, "include"), "-I" + base.CSRC,
               os.path.join(base.HERE, "shared_plan_driver.cpp"), "-o", exe])
    base._check_clean(base._run([exe], timeout=300, env=base._env()), "checks passed")
